// rbq_sparse_decode_kv8 / rbq_dense_decode_kv8: the decode attention of
// decode.hip over a cache of 8-bit rows (e4m3 or int8, one scale per block of
// tokens, KV head and tensor), plus a window of recent rows in bf16 or fp32.
//
//   logit_t = <q, c_t> sm_scale ks(t),   out = sum_t p_t vs(t) c'_t / sum_t p_t
//
// The scales never touch the rows: ks multiplies the finished product of a row,
// vs its probability. Codes of either format are exact in bf16, so a row costs its
// conversion and nothing else: the products are those of the codes, accumulated in
// fp32, with the queries and the weighted probabilities in three bf16 parts (24
// bits; fp32 outputs keep fp32's accuracy, two parts would leave 2^-17).
//
// The split over the keys and the row lists are decode.hip's, by rules of their own
// (decode_kv8_splits); a wave takes groups of 32 rows (the bytes of 16 rows in bf16) so
// that the softmax's cross-lane steps and the second product serve twice the rows:
//   logits  v_mfma_f32_16x16x32_bf16 on two tiles of 16 rows: A = rows (lane (x, j)
//           holds row x, dimensions 64 i + 16 j .. +16: each lane's 16 bytes are one
//           load), B = the queries in the same order of dimensions
//   values  one v_mfma_f32_16x16x32_bf16 per 16 columns and part over all 32 rows:
//           C's layout gives a lane rows 4j .. 4j+3 of both tiles, which is the k
//           order of A (its probabilities) and of B (its columns of those rows)
// The split's scales (at most 128 pairs) are staged in LDS beside its row list.
// Window rows take the same path in blocks of their own (or behind the last splits' rows),
// 16 rows at a time; fp32 rows are split into three bf16 parts as the queries are (an array of 32
// or 48 bytes per lane stays in scratch memory or LDS there; no registers are spilled).
// Bound by the bytes where rows follow each other: 128K rows of 8 heads, 268 MB, 46 us
// (5.9 TB/s) and 4 of the join. Scattered rows of 128 bytes make 4.6 TB/s (a fifth of 128K
// per head: 37.7 us, 6 of them before the first row arrives), few rows the chain search,
// list, rows, join (64K rows of D = 64, 2 %: 9.6 and 3.1 us).
#include "decode_rows_dev.h"

namespace rbq {

rbq_status launch_decode_kv8(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const float* q,
                             const Kv8Cache& cache, int32_t n, const int32_t* sel_idx, const int32_t* sel_count,
                             const Kv8Window& win, float sm_scale, float* out, float* lse, void* ws, bool sparse,
                             hipStream_t stream, const unsigned long long* sel_mask, int32_t mask_words,
                             const int32_t* seq_n, const int32_t* seq_w) {
  const int G = heads_q / heads_kv;
  const DecodeSplits sp = decode_kv8_splits(batch, heads_kv, n, win.w, sparse, seq_n != nullptr, seq_w != nullptr);
  Call a = make_call(batch, heads_q, heads_kv, head_dim, q, n, sel_idx, sel_count, win, sm_scale, ws, sparse, stream,
                     sel_mask, mask_words, seq_n, seq_w, sp);
  a.K = static_cast<const char*>(cache.K8);
  a.V = static_cast<const char*>(cache.V8);
  a.k_scale = cache.k_scale;
  a.v_scale = cache.v_scale;
  a.bshift = __builtin_ctz(unsigned(cache.block));
  a.cap = cache.cap;
  const bool f32 = win.dtype == RBQ_F32 && win.w > 0, i8 = cache.dtype == RBQ_I8;
  rbq_status st;
#define RBQ_KV8(D)                                                                                          \
  (i8 ? (f32 ? launch_kind<RBQ_I8, RBQ_F32, D>(sparse, G, a) : launch_kind<RBQ_I8, RBQ_BF16, D>(sparse, G, a)) \
      : (f32 ? launch_kind<RBQ_E4M3, RBQ_F32, D>(sparse, G, a) : launch_kind<RBQ_E4M3, RBQ_BF16, D>(sparse, G, a)))
  st = head_dim == 64 ? RBQ_KV8(64) : RBQ_KV8(128);
#undef RBQ_KV8
  if (st != RBQ_OK) return st;
  if (head_dim == 64) launch_join<64>(batch * heads_q, sp.total(), a.part, out, lse, stream);
  else launch_join<128>(batch * heads_q, sp.total(), a.part, out, lse, stream);
  return hipGetLastError() == hipSuccess ? RBQ_OK : RBQ_EDEVICE;
}

}  // namespace rbq
