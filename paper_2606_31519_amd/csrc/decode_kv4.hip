// rbq_sparse_decode_kv4 / rbq_dense_decode_kv4: the decode attention over a cache of
// 4-bit rows (kv4.hip), plus a window of recent rows in bf16 or fp32.
//
//   fp4   k = 2^e c with e per group of D / 4 dimensions: the conversion to bf16 takes the
//         exponent along and is exact, so a row costs its conversion
//   int4  k = s c + m per row:  <q, k> = s <q, c> + m sum(q),
//         out = (sum_t (p_t s_t) c_t + sum_t p_t m_t) / sum_t p_t
//         the codes are exact in bf16; m's part of a logit is one product beside the row's,
//         m's part of the sums one accumulator per head. (As 16 + c, the codes' own bits, they
//         need no conversion, but 16 s then leaves with m: rel. error 3.3e-6, so 6e-7.)
//
// The kernel is the 8-bit cache's (decode_rows_dev.h) with rows of a quarter of bf16's
// bytes: K and V of a row lie in one record, so that a listed row is one line of 128 bytes
// (gathered from two arrays, 59 % of 1M rows took 50.6 us instead of 38.8, a fifth 26.4
// instead of 19.2). A lane of the logits product takes a quarter of a row, one load of 16
// bytes at D = 128 and one exponent; the words of four rows are loaded by the four lanes of a
// quad and spread from there.
// Bound by memory while rows stream (5.3 TB/s), by latency around that: of the
// 37.1 us of 128K rows x 8 heads (143 MB) the rows take 27, starting a block 0.9, joining its
// waves 1.7, the second kernel with its launch 4.6; of the 33.8 us with a fifth of them listed
// (88 MB with the lists) the rows take 19, reading a list 4.7. Four waves a SIMD: five spill,
// and three that load further ahead are slower.
#include "decode_rows_dev.h"

namespace rbq {

rbq_status launch_decode_kv4(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const float* q,
                             const Kv4Cache& cache, int32_t n, const int32_t* sel_idx, const int32_t* sel_count,
                             const Kv8Window& win, float sm_scale, float* out, float* lse, void* ws, bool sparse,
                             hipStream_t stream, const unsigned long long* sel_mask, int32_t mask_words,
                             const int32_t* seq_n, const int32_t* seq_w) {
  const int G = heads_q / heads_kv;
  const DecodeSplits sp =
      decode_kv4_splits(batch, heads_q, heads_kv, head_dim, n, win.w, sparse, seq_n != nullptr, seq_w != nullptr);
  Call a = make_call(batch, heads_q, heads_kv, head_dim, q, n, sel_idx, sel_count, win, sm_scale, ws, sparse, stream,
                     sel_mask, mask_words, seq_n, seq_w, sp);
  a.K = static_cast<const char*>(cache.KV4);
  a.k_scale = reinterpret_cast<const float*>(cache.par);
  a.cap = cache.cap;
  a.turns = !sparse && !a.ragged && kv4_one_round(batch, heads_q, heads_kv, head_dim, sp);
  const bool f32 = win.dtype == RBQ_F32 && win.w > 0, i4 = cache.dtype == RBQ_I4;
  rbq_status st;
#define RBQ_KV4(D)                                                                                          \
  (i4 ? (f32 ? launch_kind<RBQ_I4, RBQ_F32, D>(sparse, G, a) : launch_kind<RBQ_I4, RBQ_BF16, D>(sparse, G, a)) \
      : (f32 ? launch_kind<RBQ_FP4, RBQ_F32, D>(sparse, G, a) : launch_kind<RBQ_FP4, RBQ_BF16, D>(sparse, G, a)))
  st = head_dim == 64 ? RBQ_KV4(64) : RBQ_KV4(128);
#undef RBQ_KV4
  if (st != RBQ_OK) return st;
  if (head_dim == 64) launch_join<64>(batch * heads_q, sp.total(), a.part, out, lse, stream);
  else launch_join<128>(batch * heads_q, sp.total(), a.part, out, lse, stream);
  return hipGetLastError() == hipSuccess ? RBQ_OK : RBQ_EDEVICE;
}

}  // namespace rbq
