// Host-side argument checks and workspace sizing. No HIP calls: everything
// here runs (and is tested) without a GPU.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "rbq_internal.h"

namespace rbq {

namespace {
constexpr int64_t kMaxRows = int64_t(1) << 31;
constexpr int64_t kMaxStride = int64_t(1) << 23;   // elements: 64 rows of it are addressed with 32-bit byte offsets
constexpr int64_t kCus = 256;                      // compute units of the GPU
// Blocks of a round of the decode over an 8-bit cache: 4 per compute unit, as many as run at once at D = 128 in
// groups of up to 8 heads. (By the compiler's report, with a bf16 window, 5 or 6 do at D = 64, 4 sparse in groups
// of 16; at D = 128 in groups of 16 dense 3, sparse 2. A planned round is 0.7 to 0.8, 1.3 and 2 of the GPU's
// there: no plans of their own are made for them, and none were measured.)
constexpr int64_t kKv8Resident = 4 * kCus;
// a required device pointer: present, and 16-byte aligned (the kernels use 16-byte vector loads)
bool bad_ptr(const void* p) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
}  // namespace

rbq_status check_heads(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim) {
  if (batch <= 0 || heads_q <= 0 || heads_kv <= 0 || head_dim <= 0) return RBQ_EINVAL;
  if (heads_q % heads_kv != 0) return RBQ_EINVAL;
  if (head_dim % 32 != 0) return RBQ_EINVAL;
  if (int64_t(batch) * heads_q > 65535 * int64_t(1024)) return RBQ_EINVAL;
  if (int64_t(batch) * heads_kv > 65535) return RBQ_EINVAL;   // grid.y of the per-(b, kv-head) kernels
  if (heads_q / heads_kv > 16) return RBQ_EUNSUPPORTED;       // GQA group size handled by the kernels
  if (head_dim != kHeadDim && head_dim != 64) return RBQ_EUNSUPPORTED;   // D = 128, and 64 for the uniform calls
  return RBQ_OK;
}

size_t encode_workspace_bytes(int32_t batch, int32_t heads_kv, int32_t head_dim, int32_t n_new) {
  if (batch <= 0 || heads_kv <= 0 || head_dim <= 0 || n_new < 0) return 0;
  const int64_t chunks = (int64_t(n_new) + kCentroidChunk - 1) / kCentroidChunk;
  return align_up(size_t(batch) * heads_kv * (chunks > 0 ? chunks : 1) * head_dim * sizeof(float), 256);
}

rbq_status check_encode(int32_t batch, int32_t heads_kv, int32_t head_dim, const void* keys, int32_t keys_dtype,
                        int64_t keys_ld, int32_t n_new, int32_t offset, int32_t cap, const float* P,
                        const float* c_k, const uint32_t* codes, const void* kfac, uint32_t flags,
                        const void* ws, size_t ws_bytes) {
  rbq_status s = check_heads(batch, heads_kv, heads_kv, head_dim);
  if (s != RBQ_OK) return s;
  if (keys_dtype != RBQ_F32 && keys_dtype != RBQ_BF16) return RBQ_EUNSUPPORTED;
  if (n_new < 0 || offset < 0 || cap < 0 || keys_ld < n_new || keys_ld >= kMaxRows) return RBQ_EINVAL;
  if (int64_t(offset) + n_new > cap) return RBQ_EINVAL;
  if (flags & ~RBQ_ENCODE_SET_CENTROID) return RBQ_EINVAL;
  if ((flags & RBQ_ENCODE_SET_CENTROID) && n_new == 0) return RBQ_EINVAL;   // the mean of no keys
  if (bad_ptr(P) || bad_ptr(c_k) || bad_ptr(codes) || bad_ptr(kfac)) return RBQ_EINVAL;
  if (n_new > 0 && bad_ptr(keys)) return RBQ_EINVAL;
  if (flags & RBQ_ENCODE_SET_CENTROID) {
    if (bad_ptr(ws) || ws_bytes < encode_workspace_bytes(batch, heads_kv, head_dim, n_new)) return RBQ_EINVAL;
  }
  return RBQ_OK;
}

rbq_status check_quantize(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const float* q,
                          const float* P, const float* c_k, const uint32_t* qplanes, const float* qscal) {
  rbq_status s = check_heads(batch, heads_q, heads_kv, head_dim);
  if (s != RBQ_OK) return s;
  if (bad_ptr(q) || bad_ptr(P) || bad_ptr(c_k) || bad_ptr(qplanes) || bad_ptr(qscal)) return RBQ_EINVAL;
  return RBQ_OK;
}

rbq_status check_score(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t n, int32_t cap,
                       const uint32_t* codes, const void* kfac, const uint32_t* qplanes, const void* qscal,
                       const void* out) {
  rbq_status s = check_heads(batch, heads_q, heads_kv, head_dim);
  if (s != RBQ_OK) return s;
  if (n < 0 || cap < 0 || n > cap) return RBQ_EINVAL;
  if (n > 0 && (bad_ptr(codes) || bad_ptr(kfac) || bad_ptr(qplanes) || bad_ptr(qscal) || bad_ptr(out)))
    return RBQ_EINVAL;
  return RBQ_OK;
}

ToppPlan topp_plan(int32_t n) {
  const int64_t subs = n > 0 ? (int64_t(n) + kSelSub - 1) / kSelSub : 1;
  ToppPlan pl;
  pl.spb = int32_t((subs + kSelMaxParts - 1) / kSelMaxParts);
  pl.parts = int32_t((subs + pl.spb - 1) / pl.spb);
  return pl;
}

ToppWorkspace topp_workspace(void* base, int64_t rows, int32_t n) {
  const ToppPlan pl = topp_plan(n);
  ToppWorkspace w{};
  size_t off = 0;
  char* b = static_cast<char*>(base);
  w.part1 = reinterpret_cast<unsigned char*>(b + off);
  off = align_up(off + size_t(rows) * pl.parts * kSelPart1Bytes, 256);
  w.part2 = reinterpret_cast<unsigned char*>(b + off);
  off = align_up(off + size_t(rows) * pl.parts * kSelPart2Bytes, 256);
  w.state = reinterpret_cast<uint32_t*>(b + off);
  off = align_up(off + size_t(rows) * kSelStateWords * sizeof(uint32_t), 256);
  w.bytes = off;
  return w;
}

rbq_status check_topp(int32_t batch, int32_t heads_q, int32_t n, const float* scores, float p, float sm_scale,
                      const int32_t* sel_idx, const int32_t* sel_count, const void* ws, size_t ws_bytes) {
  if (batch <= 0 || heads_q <= 0 || n < 0) return RBQ_EINVAL;
  if (int64_t(batch) * heads_q > 65535) return RBQ_EINVAL;
  // a row's softmax masses are summed as 2^-40 fixed-point integers of at most
  // 2^40 each in 64 bits: exact only below 2^24 keys per row
  if (n >= kToppMaxKeys) return RBQ_EUNSUPPORTED;
  if (!(p > 0.0f) || !(p <= 1.0f)) return RBQ_EINVAL;                  // also rejects NaN
  if (!std::isfinite(sm_scale) || !(sm_scale > 0.0f)) return RBQ_EINVAL;
  if (bad_ptr(sel_count)) return RBQ_EINVAL;
  if (n > 0 && (bad_ptr(scores) || bad_ptr(sel_idx))) return RBQ_EINVAL;
  if (n > 0 && p < 1.0f) {
    if (bad_ptr(ws) || ws_bytes < topp_workspace(nullptr, int64_t(batch) * heads_q, n).bytes) return RBQ_EINVAL;
  }
  return RBQ_OK;
}

DecodeSplits decode_splits(int32_t batch, int32_t heads_kv, int32_t n, int32_t w, bool tail_window, bool sparse,
                           bool ragged) {
  DecodeSplits s;
  s.fold_s0 = 0;
  s.fold_wq = 0;
  // halve the chunk until the grid has kDecodeMinBlocks blocks or the chunk is 256
  const int64_t groups = int64_t(batch) * heads_kv;
  s.chunk = kDecodeChunk;
  while (s.chunk > 256 && groups * ((int64_t(n) + s.chunk - 1) / s.chunk) < kDecodeMinBlocks) s.chunk /= 2;
  s.idx_splits = n > 0 ? int32_t((int64_t(n) + s.chunk - 1) / s.chunk) : 0;
  s.win_splits = w > 0 ? int32_t((int64_t(w) + kDecodeWinChunk - 1) / kDecodeWinChunk) : 0;
  if (tail_window && s.idx_splits > 0 && w > 0) {
    if (ragged) {
      const int cap = kDecodeListCap - s.chunk;   // window rows a split's list can still take
      if ((int64_t(w) + cap - 1) / cap <= s.idx_splits) {
        s.fold_wq = cap;
        s.win_splits = 0;
      }
    } else if (sparse) {
      const int64_t wq = (int64_t(w) + s.idx_splits - 1) / s.idx_splits;
      if (wq <= kDecodeFoldMax) {
        s.fold_wq = int32_t(wq);
        s.win_splits = 0;
      }
    } else if (int64_t(n) - int64_t(s.idx_splits - 1) * s.chunk + w <= s.chunk) {
      s.fold_s0 = s.idx_splits - 1;
      s.fold_wq = w;
      s.win_splits = 0;
    }
  }
  if (s.total() == 0) s.win_splits = 1;   // one empty split keeps the combine step uniform
  return s;
}

size_t decode_workspace_bytes(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t n,
                              int32_t w) {
  if (batch <= 0 || heads_q <= 0 || heads_kv <= 0 || head_dim <= 0 || n < 0 || w < 0) return 0;
  const DecodeSplits s = decode_splits(batch, heads_kv, n, w);
  return align_up(size_t(batch) * heads_q * s.total() * (head_dim + 2) * sizeof(float), 256);
}

rbq_status check_decode(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const float* q,
                        const void* K, const void* V, int32_t kv_dtype, int32_t cap, int32_t n, bool sparse,
                        const int32_t* sel_idx, const int32_t* sel_count, const void* K_loc, const void* V_loc,
                        int64_t loc_ld, int32_t w, float sm_scale, const float* out, const void* ws,
                        size_t ws_bytes) {
  rbq_status s = check_heads(batch, heads_q, heads_kv, head_dim);
  if (s != RBQ_OK) return s;
  if (kv_dtype != RBQ_F32 && kv_dtype != RBQ_BF16) return RBQ_EUNSUPPORTED;
  const int32_t G = heads_q / heads_kv;
  if (G & (G - 1)) return RBQ_EUNSUPPORTED;   // the decode kernels are built for G in {1, 2, 4, 8, 16}
  if (n < 0 || cap < 0 || n > cap || w < 0 || w > RBQ_MAX_WINDOW) return RBQ_EINVAL;
  if (!std::isfinite(sm_scale) || !(sm_scale > 0.0f)) return RBQ_EINVAL;
  if (bad_ptr(q) || bad_ptr(out)) return RBQ_EINVAL;
  if (n > 0 && (bad_ptr(K) || bad_ptr(V))) return RBQ_EINVAL;
  if (sparse && (bad_ptr(sel_count) || (n > 0 && bad_ptr(sel_idx)))) return RBQ_EINVAL;
  if (w > 0 && (bad_ptr(K_loc) || bad_ptr(V_loc) || loc_ld < w || loc_ld >= kMaxRows)) return RBQ_EINVAL;
  // rows of one (sequence, KV head) are addressed with 32-bit byte offsets
  const int64_t row_bytes = int64_t(head_dim) * (kv_dtype == RBQ_BF16 ? 2 : 4);
  if (int64_t(n) * row_bytes >= (int64_t(1) << 31) || int64_t(w) * row_bytes >= (int64_t(1) << 31)) return RBQ_EINVAL;
  if (bad_ptr(ws) || ws_bytes < decode_workspace_bytes(batch, heads_q, heads_kv, head_dim, n, w)) return RBQ_EINVAL;
  return RBQ_OK;
}

namespace {
// blocks of a dense call over the 8-bit cache that are planned for: those of `blocks` in whole rounds
int64_t kv8_round_blocks(int64_t blocks) {
  return std::max<int64_t>((blocks + kKv8Resident / 2) / kKv8Resident, 1) * kKv8Resident;
}
}  // namespace

DecodeSplits decode_kv8_splits(int32_t batch, int32_t heads_kv, int32_t n, int32_t w, bool sparse, bool ragged,
                               bool own_windows) {
  DecodeSplits s = decode_splits(batch, heads_kv, n, w);
  if (ragged || n <= 0) return s;
  const int64_t groups = int64_t(batch) * heads_kv;
  auto take = [&](int64_t chunk) {
    s.chunk = int32_t(chunk);
    s.idx_splits = int32_t((int64_t(n) + chunk - 1) / chunk);
  };
  if (sparse) {
    take(kDecodeChunk);
    while (s.chunk > kDecodeMinChunk && groups * s.idx_splits < kKv8SparseBlocks) take(s.chunk / 2);
    if (groups * s.idx_splits < kCus) take(kDecodeMinChunk / 2);
    if (!own_windows && s.win_splits <= s.idx_splits && groups * s.idx_splits <= kKv8Resident &&
        groups * s.total() > kKv8Resident) {
      s.fold_s0 = s.idx_splits - s.win_splits;
      s.fold_wq = kDecodeWinChunk;
      s.win_splits = 0;
    }
    return s;
  }
  if (groups * n < kKv8Resident * kDecodeMinChunk) {
    if (groups * s.idx_splits < kCus) take(kDecodeMinChunk / 2);
    return s;
  }
  const int64_t splits = kv8_round_blocks(groups * s.total()) / groups - s.win_splits;
  if (splits < 1) return s;
  const int64_t chunk = ((int64_t(n) + splits - 1) / splits + 63) / 64 * 64;
  take(std::max<int64_t>(std::min<int64_t>(chunk, kKv8DenseChunk), kDecodeMinChunk));
  return s;
}

int64_t kv4_places(int32_t heads_q, int32_t heads_kv, int32_t head_dim) {
  return head_dim == kHeadDim && heads_q / heads_kv == 16 ? 3 * kCus : kKv8Resident;
}

DecodeSplits decode_kv4_splits(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t n, int32_t w,
                               bool sparse, bool ragged, bool own_windows) {
  DecodeSplits s = decode_kv8_splits(batch, heads_kv, n, w, sparse, ragged, own_windows);
  const int64_t groups = int64_t(batch) * heads_kv;
  if (sparse || ragged || groups * n < kKv8Resident * kDecodeMinChunk) return s;
  const int64_t places = kv4_places(heads_q, heads_kv, head_dim), splits = places / groups - s.win_splits;
  if (20 * splits * groups < 17 * places) return s;
  const int64_t chunk = ((int64_t(n) + splits - 1) / splits + 63) / 64 * 64;
  s.chunk = int32_t(std::max<int64_t>(chunk, kDecodeMinChunk));
  s.idx_splits = int32_t((int64_t(n) + s.chunk - 1) / s.chunk);
  return s;
}

namespace {
size_t decode_states_bytes(int32_t batch, int32_t heads_q, int32_t head_dim, int64_t splits) {
  return size_t(batch) * heads_q * splits * (size_t(head_dim) + 2) * sizeof(float);
}
}  // namespace

size_t decode_kv8_workspace_bytes(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t n,
                                  int32_t w, bool step) {
  if (batch <= 0 || heads_q <= 0 || heads_kv <= 0 || head_dim <= 0 || n < 0 || w < 0) return 0;
  // sparse: chunks that do not depend on the window, and its splits beside them
  int64_t total = decode_kv8_splits(batch, heads_kv, n, w, true, false, true).total();
  if (!step) {
    // ragged: the same; dense: of its own, or of a shorter window's the most that whole rounds leave
    const int64_t groups = int64_t(batch) * heads_kv, ragged = decode_splits(batch, heads_kv, n, w).total();
    total = std::max<int64_t>({total, ragged, decode_kv8_splits(batch, heads_kv, n, w, false, false, false).total()});
    if (groups * n >= kKv8Resident * kDecodeMinChunk) total = std::max(total, kv8_round_blocks(groups * ragged) / groups);
  }
  return align_up(decode_states_bytes(batch, heads_q, head_dim, total), 256);
}

size_t decode_kv4_workspace_bytes(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t n,
                                  int32_t w, bool step) {
  // the 8-bit cache's splits, or, of a dense call with any window, at most a round of blocks
  const size_t as_kv8 = decode_kv8_workspace_bytes(batch, heads_q, heads_kv, head_dim, n, w, step);
  if (as_kv8 == 0 || step) return as_kv8;
  const int64_t groups = int64_t(batch) * heads_kv;
  int64_t dense = decode_kv4_splits(batch, heads_q, heads_kv, head_dim, n, w, false, false, false).total();
  if (groups * n >= kKv8Resident * kDecodeMinChunk) dense = std::max(dense, kv4_places(heads_q, heads_kv, head_dim) / groups);
  return std::max(as_kv8, align_up(decode_states_bytes(batch, heads_q, head_dim, dense), 256));
}

namespace {
bool bad_seq(const int32_t* p) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
rbq_status check_kv8_form(int32_t block, int32_t kv8_dtype) {
  if (kv8_dtype != RBQ_E4M3 && kv8_dtype != RBQ_I8) return RBQ_EUNSUPPORTED;
  if (block < 1 || (block & (block - 1)) != 0) return RBQ_EINVAL;
  if (block < kMinKv8Block || block > kMaxKv8Block) return RBQ_EUNSUPPORTED;
  return RBQ_OK;
}
}  // namespace

rbq_status check_quantize_kv(int32_t batch, int32_t heads_kv, int32_t head_dim, const void* K, const void* V,
                             int32_t dtype, int64_t ld, int32_t rows, int32_t offset, int32_t cap, int32_t block,
                             int32_t kv8_dtype, const void* K8, const void* V8, const float* k_scale,
                             const float* v_scale, const int32_t* seq_off, const int32_t* seq_rows) {
  rbq_status s = check_heads(batch, heads_kv, heads_kv, head_dim);
  if (s != RBQ_OK) return s;
  if (dtype != RBQ_F32 && dtype != RBQ_BF16) return RBQ_EUNSUPPORTED;
  if ((s = check_kv8_form(block, kv8_dtype)) != RBQ_OK) return s;
  if (rows < 0 || offset < 0 || cap < 0 || ld < rows || ld >= kMaxRows) return RBQ_EINVAL;
  if (int64_t(offset) + rows > cap) return RBQ_EINVAL;
  if ((int64_t(offset) + rows) * head_dim >= (int64_t(1) << 31)) return RBQ_EINVAL;   // as the calls that read them
  if (bad_seq(seq_off) || bad_seq(seq_rows)) return RBQ_EINVAL;
  if (rows > 0 && (bad_ptr(K) || bad_ptr(V) || bad_ptr(K8) || bad_ptr(V8) || bad_ptr(k_scale) || bad_ptr(v_scale)))
    return RBQ_EINVAL;
  return RBQ_OK;
}

rbq_status check_decode_kv8(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const float* q,
                            const Kv8Cache& c, int32_t n, bool sparse, const int32_t* sel_idx,
                            const int32_t* sel_count, const Kv8Window& win, float sm_scale, const float* out,
                            const void* ws, size_t ws_bytes, const int32_t* seq_n, const int32_t* seq_w) {
  rbq_status s = check_heads(batch, heads_q, heads_kv, head_dim);
  if (s != RBQ_OK) return s;
  if ((s = check_kv8_form(c.block, c.dtype)) != RBQ_OK) return s;
  if (win.w != 0 && win.dtype != RBQ_F32 && win.dtype != RBQ_BF16) return RBQ_EUNSUPPORTED;
  const int32_t G = heads_q / heads_kv;
  if (G & (G - 1)) return RBQ_EUNSUPPORTED;   // the decode kernels are built for G in {1, 2, 4, 8, 16}
  if (n < 0 || c.cap < 0 || n > c.cap || win.w < 0 || win.w > RBQ_MAX_WINDOW) return RBQ_EINVAL;
  if (!std::isfinite(sm_scale) || !(sm_scale > 0.0f)) return RBQ_EINVAL;
  if (bad_ptr(q) || bad_ptr(out) || bad_seq(seq_n) || bad_seq(seq_w)) return RBQ_EINVAL;
  if (n > 0 && (bad_ptr(c.K8) || bad_ptr(c.V8) || bad_ptr(c.k_scale) || bad_ptr(c.v_scale))) return RBQ_EINVAL;
  if (sparse && (bad_ptr(sel_count) || (n > 0 && bad_ptr(sel_idx)))) return RBQ_EINVAL;
  if (win.w > 0 && (bad_ptr(win.K) || bad_ptr(win.V) || win.ld < win.w || win.ld >= kMaxRows)) return RBQ_EINVAL;
  // rows of one (sequence, KV head) are addressed with 32-bit byte offsets
  if (int64_t(n) * head_dim >= (int64_t(1) << 31)) return RBQ_EINVAL;
  // (what this form of the call needs: rbq_workspace_bytes gives the largest of the forms')
  const int64_t splits = decode_kv8_splits(batch, heads_kv, n, win.w, sparse, seq_n != nullptr, seq_w != nullptr).total();
  if (bad_ptr(ws) || ws_bytes < decode_states_bytes(batch, heads_q, head_dim, splits)) return RBQ_EINVAL;
  // a ragged batch's blocks are numbered along one dimension of the grid
  if ((seq_n || seq_w) && int64_t(batch) * heads_kv * splits >= (int64_t(1) << 24)) return RBQ_EUNSUPPORTED;
  return RBQ_OK;
}

namespace {
rbq_status check_kv4_form(int32_t kv4_dtype) {
  return kv4_dtype == RBQ_FP4 || kv4_dtype == RBQ_I4 ? RBQ_OK : RBQ_EUNSUPPORTED;
}
}  // namespace

rbq_status check_quantize_kv4(int32_t batch, int32_t heads_kv, int32_t head_dim, const void* K, const void* V,
                              int32_t dtype, int64_t ld, int32_t rows, int32_t offset, const Kv4Cache& c,
                              const int32_t* seq_off, const int32_t* seq_rows) {
  rbq_status s = check_heads(batch, heads_kv, heads_kv, head_dim);
  if (s != RBQ_OK) return s;
  if (dtype != RBQ_F32 && dtype != RBQ_BF16) return RBQ_EUNSUPPORTED;
  if ((s = check_kv4_form(c.dtype)) != RBQ_OK) return s;
  if (rows < 0 || offset < 0 || c.cap < 0 || ld < rows || ld >= kMaxRows) return RBQ_EINVAL;
  if (int64_t(offset) + rows > c.cap) return RBQ_EINVAL;
  if ((int64_t(offset) + rows) * head_dim >= (int64_t(1) << 31)) return RBQ_EINVAL;   // as the calls that read them
  if (bad_seq(seq_off) || bad_seq(seq_rows)) return RBQ_EINVAL;
  if (rows > 0 && (bad_ptr(K) || bad_ptr(V) || bad_ptr(c.KV4) || bad_ptr(c.par))) return RBQ_EINVAL;
  return RBQ_OK;
}

rbq_status check_decode_kv4(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const float* q,
                            const Kv4Cache& c, int32_t n, bool sparse, const int32_t* sel_idx,
                            const int32_t* sel_count, const Kv8Window& win, float sm_scale, const float* out,
                            const void* ws, size_t ws_bytes, const int32_t* seq_n, const int32_t* seq_w) {
  rbq_status s = check_kv4_form(c.dtype);
  if (s != RBQ_OK) return s;
  // the same call over another cache: a row's record takes the bytes that K's row takes there
  const float* par = reinterpret_cast<const float*>(c.par);
  const Kv8Cache as{c.KV4, c.KV4, par, par, RBQ_E4M3, kMinKv8Block, c.cap};
  s = check_decode_kv8(batch, heads_q, heads_kv, head_dim, q, as, n, sparse, sel_idx, sel_count, win, sm_scale, out, ws,
                       ws_bytes, seq_n, seq_w);
  if (s != RBQ_OK) return s;
  // (the splits of dense calls are its own)
  const DecodeSplits sp =
      decode_kv4_splits(batch, heads_q, heads_kv, head_dim, n, win.w, sparse, seq_n != nullptr, seq_w != nullptr);
  return ws_bytes < decode_states_bytes(batch, heads_q, head_dim, sp.total()) ? RBQ_EINVAL : RBQ_OK;
}

namespace {
// Time of a prompt call in us, but for what every choice takes, with the keys in chunks of
// `kchunk`: the steps of 64 keys that a block takes one after the other, by the blocks of a
// compute unit (the longest sequence's length stands for the others': with many, for half of
// theirs), and the states' way through memory and the joining kernel.
double prefill_cost(int64_t blocks, int32_t batch, int64_t rows, int32_t head_dim, int64_t max_k, int32_t dtype,
                    int64_t kchunk) {
  const int64_t splits = (max_k + kchunk - 1) / kchunk;
  const double per_cu = double(blocks * splits) * (0.5 + 1.0 / (batch + 1.0)) / kCus;
  double step;
  if (dtype == RBQ_F32) step = head_dim == 64 ? 2.8 + 2.4 * std::ceil(per_cu) : 2.4 + 9.0 * std::ceil(per_cu);
  else step = (head_dim == 64 ? 0.7 : 1.0) * (per_cu <= 1.0 ? 1.2 : 1.5 * std::max(1.0, per_cu / 2.0));
  const double states = splits > 1 ? 3.5 + 0.27e-6 * double(rows * splits) * (head_dim + 2) * sizeof(float) : 0.0;
  return double(kchunk / 64) * step + states;
}
}  // namespace

namespace {
// Rows (token, head of the group) a sequence up to which chunks over a 4-bit cache take the
// kernel of few rows, two blocks per compute unit (us, in brackets in tiles of 128 rows): 32 / 8 heads of 128, fp4,
// 8 x 7 tokens over up to 8000 rows 20.1 (30.3), 8 tokens over 30000 22.8 (30.0), 128 tokens 92.6 (120), 256 tokens
// 168 (157), 512 over 8000 99.8 (98.6), 2001 over 30011 1243 (1054). (A batch goes by its mean: a long chunk beside many
// single tokens takes that, 2000 tokens and 63 single ones over 1000 to 30000 rows each 1019 us, apart 664 and 286.)
// fp32 takes it, whatever the rows, unless more keys are the chunk's own than are cached: 1000 tokens of 32 / 8 heads
// over 8000 rows 409 us (1508), 1000 of 4 / 1 over none 35.4 (35.2), 2500 180 (112); at D = 64, where it is the faster
// one there too (16.9 and 24.0, 55.5 and 59.2), no rule of its own is made.
constexpr int64_t kFewRows = 512, kFewOwn = 1024;
bool few_rows(int64_t rows, int32_t batch, int32_t max_k, int32_t total_q, int32_t dtype) {
  const int64_t ends = std::min<int64_t>(batch, total_q);
  if (dtype == RBQ_F32) return total_q <= ends * std::max<int64_t>(max_k - total_q, kFewOwn);
  return rows <= kFewRows * ends;
}
}  // namespace

PrefillPlan prefill_plan(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t max_k, int32_t total_q,
                         int32_t dtype, bool kv4) {
  const int64_t rows = int64_t(total_q) * (heads_q / heads_kv);
  PrefillPlan p;
  if (kv4 && few_rows(rows, batch, max_k, total_q, dtype)) {
    p.rows = 32;
    const int64_t ends = std::min<int64_t>(batch, total_q);
    p.tiles = int32_t(rows / p.rows + ends);
    // (sequences end in a tile half full, and have, of several, half the longest one's keys)
    const double blocks = double(std::max<int64_t>(rows / p.rows + ends / 2, ends)) * heads_kv * (0.5 + 1.0 / (batch + 1.0));
    const int64_t want = std::min<int64_t>(std::max<int64_t>(int64_t(2 * kCus / blocks), 1), 64);   // (the joining kernel's most)
    const int64_t kchunk = std::max<int64_t>(((int64_t(max_k) + want - 1) / want + 63) / 64 * 64, 128);
    p.kchunk = int32_t(std::min<int64_t>(kchunk, (int64_t(1) << 31) - 64));
    p.splits = std::max<int32_t>(int32_t((int64_t(max_k) + p.kchunk - 1) / p.kchunk), 1);
    return p;
  }
  p.rows = 128;
  // every sequence with tokens may end in a tile of its own
  const int64_t ends = std::min<int64_t>(batch, total_q);
  p.tiles = int32_t(rows / p.rows + ends);
  const int64_t blocks = std::max<int64_t>((rows + p.rows - 1) / p.rows, ends) * heads_kv;
  auto chunk_of = [&](int64_t splits) { return std::max<int64_t>(((int64_t(max_k) + splits - 1) / splits + 63) / 64 * 64, 64); };
  int64_t kchunk = chunk_of(1);
  if (blocks < kCus) {
    double best = prefill_cost(blocks, batch, int64_t(total_q) * heads_q, head_dim, max_k, dtype, kchunk);
    for (int64_t want : {2, 3, 4, 5, 6, 8, 10, 12, 14, 17, 20, 24, 28, 34, 40, 48, 64}) {   // (the joining kernel weighs a split per lane: 64)
      const int64_t c = chunk_of(want);
      const double t = prefill_cost(blocks, batch, int64_t(total_q) * heads_q, head_dim, max_k, dtype, c);
      if (t < 0.97 * best) {
        best = t;
        kchunk = c;
      }
    }
  }
  p.kchunk = int32_t(std::min<int64_t>(kchunk, (int64_t(1) << 31) - 64));
  p.splits = std::max<int32_t>(int32_t((int64_t(max_k) + p.kchunk - 1) / p.kchunk), 1);
  return p;
}

size_t prefill_workspace_bytes(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t max_k,
                               int32_t total_q, bool kv4) {
  if (batch <= 0 || heads_q <= 0 || heads_kv <= 0 || head_dim <= 0 || max_k < 0 || total_q <= 0) return 0;
  if (heads_q % heads_kv != 0) return 0;
  size_t need = 0;
  for (int32_t dtype : {RBQ_F32, RBQ_BF16}) {
    const PrefillPlan p = prefill_plan(batch, heads_q, heads_kv, head_dim, max_k, total_q, dtype, kv4);
    if (p.splits > 1) need = std::max(need, size_t(total_q) * heads_q * p.splits * (size_t(head_dim) + 2) * sizeof(float));
  }
  return align_up(need, 256);
}

rbq_status check_prefill(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const PrefillArgs& a) {
  rbq_status s = check_heads(batch, heads_q, heads_kv, head_dim);
  if (s != RBQ_OK) return s;
  if (a.cache != nullptr) {
    if ((s = check_kv4_form(a.cache->dtype)) != RBQ_OK) return s;
    if (a.cached < 0 || a.cache->cap < 0 || a.cached > a.cache->cap || a.total_q < 0 || bad_seq(a.seq_n)) return RBQ_EINVAL;
    if (int64_t(a.cached) * head_dim >= (int64_t(1) << 31)) return RBQ_EINVAL;   // as the decode calls
    if (a.cached > 0 && (bad_ptr(a.cache->KV4) || bad_ptr(a.cache->par))) return RBQ_EINVAL;
  }
  if (a.dtype != RBQ_F32 && a.dtype != RBQ_BF16) return RBQ_EUNSUPPORTED;
  const int64_t align = a.dtype == RBQ_BF16 ? 8 : 4;   // elements of 16 bytes
  if (a.total_q < 0 || a.max_k < 0 || a.kv_rows < 0) return RBQ_EINVAL;
  if (a.q_ld < int64_t(heads_q) * head_dim || a.q_ld % align != 0) return RBQ_EINVAL;
  if (a.kv_ld < head_dim || a.kv_ld % align != 0 || a.kv_head < 0 || a.kv_head % align != 0 || a.kv_seq < 0 ||
      a.kv_seq % align != 0)
    return RBQ_EINVAL;
  if (a.q_ld >= kMaxStride || a.kv_ld >= kMaxStride) return RBQ_EUNSUPPORTED;
  if (!std::isfinite(a.sm_scale) || !(a.sm_scale > 0.0f)) return RBQ_EINVAL;
  if (a.total_q == 0) return RBQ_OK;
  // the rows of a sequence (tokens times heads of a group) and the grid are 32-bit numbers
  const int64_t rows = int64_t(a.total_q) * (heads_q / heads_kv);
  const int64_t tile = prefill_plan(batch, heads_q, heads_kv, head_dim, a.max_k, a.total_q, a.dtype, a.cache != nullptr).rows;
  if (rows >= kMaxRows - 256 || (rows / tile + std::min<int64_t>(batch, a.total_q)) * heads_kv >= (int64_t(1) << 24))
    return RBQ_EUNSUPPORTED;
  if (bad_ptr(a.q) || bad_ptr(a.out) || bad_ptr(a.cu_q) || bad_ptr(a.cu_k)) return RBQ_EINVAL;
  if (a.kv_rows > 0 && a.max_k > 0 && (bad_ptr(a.K) || bad_ptr(a.V))) return RBQ_EINVAL;
  const bool kv4 = a.cache != nullptr;
  const PrefillPlan p = prefill_plan(batch, heads_q, heads_kv, head_dim, a.max_k, a.total_q, a.dtype, kv4);
  if (p.splits > 1 &&
      (bad_ptr(a.ws) || a.ws_bytes < prefill_workspace_bytes(batch, heads_q, heads_kv, head_dim, a.max_k, a.total_q, kv4)))
    return RBQ_EINVAL;
  return RBQ_OK;
}

// Keys per lane of the score kernel: enough blocks to cover the 256 CUs
// several times over, as many keys in flight per lane as that allows.
int score_keys_per_lane(int32_t batch, int32_t heads_kv, int32_t n) {
  const int64_t kv_keys = int64_t(batch) * heads_kv * n;
  if (kv_keys >= int64_t(kScoreThreads) * 4 * 2048) return 4;
  if (kv_keys >= int64_t(kScoreThreads) * 2 * 1024) return 2;
  return 1;
}
int topp_mask_words(int32_t n) {
  return n > 0 ? int((int64_t(n) + kSelSub - 1) / kSelSub * (kSelSub / 64)) : 0;
}

StepWorkspace step_workspace(void* base, int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                             int32_t n, int32_t w, bool kv8) {
  StepWorkspace s{};
  const int64_t rows = int64_t(batch) * heads_q;
  char* b = static_cast<char*>(base);
  size_t off = 0;
  s.decode = b + off;
  off = align_up(off + (kv8 ? decode_kv8_workspace_bytes(batch, heads_q, heads_kv, head_dim, n, w, true)
                            : decode_workspace_bytes(batch, heads_q, heads_kv, head_dim, n, w)), 256);
  s.topp = b + off;
  s.topp_bytes = topp_workspace(nullptr, rows, n).bytes;
  off = align_up(off + s.topp_bytes, 256);
  s.masks = reinterpret_cast<unsigned long long*>(b + off);
  off = align_up(off + size_t(rows) * topp_mask_words(n) * sizeof(unsigned long long), 256);
  s.bytes = off;
  return s;
}

}  // namespace rbq

extern "C" {

size_t rbq_workspace_bytes(int32_t op, int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                           int32_t n, int32_t w) {
  if (batch <= 0 || heads_q <= 0 || heads_kv <= 0 || head_dim <= 0 || n < 0 || w < 0) return 0;
  switch (op) {
    case RBQ_OP_ENCODE:
      return rbq::encode_workspace_bytes(batch, heads_kv, head_dim, n);
    case RBQ_OP_TOPP:
      return rbq::topp_workspace(nullptr, int64_t(batch) * heads_q, n).bytes;
    case RBQ_OP_SPARSE_DECODE:
    case RBQ_OP_DENSE_DECODE:
      return rbq::decode_workspace_bytes(batch, heads_q, heads_kv, head_dim, n, w);
    case RBQ_OP_DECODE_KV8:
      return rbq::decode_kv8_workspace_bytes(batch, heads_q, heads_kv, head_dim, n, w);
    case RBQ_OP_DECODE_KV4:
      return rbq::decode_kv4_workspace_bytes(batch, heads_q, heads_kv, head_dim, n, w);
    case RBQ_OP_PREFILL:
      return rbq::prefill_workspace_bytes(batch, heads_q, heads_kv, head_dim, n, w);
    case RBQ_OP_PREFILL_KV4: {
      const int64_t keys = rbq::prefill_kv4_keys(n, w);
      return keys < rbq::kMaxRows - 64
                 ? rbq::prefill_workspace_bytes(batch, heads_q, heads_kv, head_dim, int32_t(keys), w, true) : 0;
    }
    case RBQ_OP_DECODE_STEP:
    case RBQ_OP_DECODE_STEP_KV8:
    case RBQ_OP_DECODE_STEP_KV4:
      if (heads_q % heads_kv != 0) return 0;
      return rbq::step_workspace(nullptr, batch, heads_q, heads_kv, head_dim, n, w, op != RBQ_OP_DECODE_STEP).bytes;
    default:
      return 0;
  }
}

size_t rbq_index_bytes(int32_t batch, int32_t heads_kv, int32_t head_dim, int32_t cap) {
  if (batch <= 0 || heads_kv <= 0 || head_dim <= 0 || cap < 0 || head_dim % 32 != 0) return 0;
  return size_t(batch) * heads_kv * size_t(cap) * (size_t(head_dim) / 8 + 2 * sizeof(float));
}

const char* rbq_status_string(rbq_status s) {
  switch (s) {
    case RBQ_OK: return "ok";
    case RBQ_EINVAL: return "invalid argument";
    case RBQ_EUNSUPPORTED: return "unsupported shape, dtype or size";
    case RBQ_EDEVICE: return "HIP runtime error";
    default: return "unknown status";
  }
}

int32_t rbq_version(void) { return 100; }

}  // extern "C"
