// rbq_quantize_kv4 / rbq_dequantize_kv4: rows of K and V into and out of the 4-bit
// cache, one record of D bytes (D / 2 of K's codes, D / 2 of V's) and one pair of
// 32-bit words per row and KV head. A row stands by itself: writing it touches no other.
//
//   fp4   a group of D / 4 dimensions has s = 2^e with the smallest e that keeps its
//         largest magnitude within 7 (which 6, the largest code, is nearest to); x / s
//         is exact and the code is its one rounding
//   int4  a row has a base m, its smallest value rounded down to bf16, and a step s, a
//         fifteenth of what is left, rounded up: every finite value lies within half a
//         step of a code
//
// Bound by the bytes of the rows and the records: K and V of 130816 tokens x 8 heads x 128 in
// bf16, 678 MB either way, written in 125 us (5.4 TB/s) and read back in 104 (6.5; stores that
// the caches keep 121, one row a thread 110). (Two rows a thread write the same in 122, but 16 x
// 256 rows in 8.3 us instead of 7.8.)
#include <type_traits>

#include "kv4_dev.h"

namespace rbq {
namespace {

constexpr int kThreads4 = 256;
constexpr float kLeast = 1.17549435e-38f;   // 2^-126, the least scale and step
constexpr float kMost = 8.50705917e37f;     // 2^126: int4 takes finite values beyond as this
constexpr float kRound = 12582912.f;        // 1.5 * 2^23: adding it rounds to a whole number, kept in the low bits
constexpr int kTake = 16;                   // values of a row and tensor that a thread takes
constexpr int kRowsR = 2;                   // rows that a thread reads back

// The rows of one call: sequence b's rows [off, off + cnt) of the cache.
struct Span {
  int off, cnt;
};
__device__ __forceinline__ Span span_of(int b, int offset, int rows, const int32_t* seq_off, const int32_t* seq_rows) {
  return Span{seq_off ? min(max(seq_off[b], 0), offset) : offset, seq_rows ? min(max(seq_rows[b], 0), rows) : rows};
}

// v combined by op with the lanes that hold the other values: of one group of a row (2 or 1
// lanes), or of a row and tensor (8 or 4 lanes)
template <int LANES, class Op>
__device__ __forceinline__ float lanes_reduce(float v, Op op) {
  if constexpr (LANES >= 2) v = op(v, RBQ_DPP(v, 0xB1));
  if constexpr (LANES >= 4) v = op(v, RBQ_DPP(v, 0x4E));
  if constexpr (LANES >= 8) v = op(v, RBQ_DPP(v, 0x141));
  return v;
}
__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }
__device__ __forceinline__ float bf16_up(float x) {   // x >= 0
  return __uint_as_float((__float_as_uint(x) + 0xFFFFu) & 0xFFFF0000u);
}
__device__ __forceinline__ float bf16_down(float x) {   // |x| <= 2^126
  const uint32_t u = __float_as_uint(x);
  return __uint_as_float((int32_t(u) < 0 ? u + 0xFFFFu : u) & 0xFFFF0000u);
}

// 16 values of fp4: their codes, and their group's exponent byte
template <int LANES>
__device__ __forceinline__ u32x2 encode_fp4(const float* x, uint32_t& byte) {
  uint32_t amax = 0u;
#pragma unroll
  for (int i = 0; i < kTake; ++i) {
    const uint32_t u = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    amax = max(amax, u < 0x7F800000u ? u : 0u);   // (the order of magnitudes is the order of the bits)
  }
  if constexpr (LANES >= 2) amax = max(amax, RBQ_DPP_U32(amax, 0xB1));
  // amax = m 2^x with m in [1, 2); 7 = 1.75 * 2^2, so e = x - 2, one more above m = 1.75
  const int e = int(amax >> 23) - 127 - 2 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  const int ec = min(max(e, -126), 125);
  byte = amax == 0u ? 0u : uint32_t(ec + 127);
  const float r = __uint_as_float(uint32_t(127 - ec) << 23);
  u32x2 w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t v = 0u;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      float y[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float t = x[8 * h + 2 * p + i] * r;   // exact: r is a power of two
        y[i] = amax != 0u && t == t ? fminf(fmaxf(t, -6.f), 6.f) : 0.f;
      }
      // (the byte's place is a literal)
      v = p == 0   ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[0], y[1], 1.f, 0)
          : p == 1 ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[0], y[1], 1.f, 1)
          : p == 2 ? __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[0], y[1], 1.f, 2)
                   : __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[0], y[1], 1.f, 3);
    }
    w[h] = v;
  }
  return w;
}

// 16 values of int4: their codes, and their row's word
template <int LANES>
__device__ __forceinline__ u32x2 encode_i4(const float* x, uint32_t& word) {
  float lo = INFINITY, hi = -INFINITY;
#pragma unroll
  for (int i = 0; i < kTake; ++i) {
    const bool f = is_finite(x[i]);
    const float v = fminf(fmaxf(x[i], -kMost), kMost);
    lo = f ? fminf(lo, v) : lo;
    hi = f ? fmaxf(hi, v) : hi;
  }
  lo = lanes_reduce<LANES>(lo, [](float a, float b) { return fminf(a, b); });
  hi = lanes_reduce<LANES>(hi, [](float a, float b) { return fmaxf(a, b); });
  if (lo > hi) lo = hi = 0.f;   // no finite value
  const float m = bf16_down(lo), d = hi - m;
  const float s = d > 0.f ? bf16_up(fmaxf(d / 15.f, kLeast)) : 0.f;
  const float r = s > 0.f ? 1.f / s : 0.f;
  word = __float_as_uint(s) >> 16 | __float_as_uint(m);
  u32x2 w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t v = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float y = x[8 * h + i] == x[8 * h + i] ? x[8 * h + i] : 0.f;
      const float t = fmaf(y - m, r, kRound);   // one rounding, to a whole number
      const uint32_t c = __float_as_uint(t == t ? fminf(fmaxf(t, kRound), kRound + 15.f) : kRound) & 15u;
      v |= c << nibble_shift<RBQ_I4>(i);
    }
    w[h] = v;
  }
  return w;
}

// Grid (row pieces, (b, kv head)): a thread takes 16 values of a row of K or of V; the lanes of a
// row follow each other, K's before V's, so that a wave's codes leave as whole records.
template <int DT, int FMT, int D>
__global__ __launch_bounds__(kThreads4) void quantize_kv4_kernel(
    const char* __restrict__ K, const char* __restrict__ V, int64_t ld, int n_new, int offset, int cap,
    char* __restrict__ KV4, uint32_t* __restrict__ par, int Hkv, const int32_t* __restrict__ seq_off,
    const int32_t* __restrict__ seq_new) {
  constexpr int kEl = DT == RBQ_BF16 ? 2 : 4, kLanes = D / kTake;   // lanes of a row and tensor
  const int bh = blockIdx.y, b = bh / Hkv;
  const Span sp = span_of(b, offset, n_new, seq_off, seq_new);
  const int row = int(blockIdx.x) * (kThreads4 / (2 * kLanes)) + threadIdx.x / (2 * kLanes);
  const int l = threadIdx.x % (2 * kLanes), piece = l % kLanes;
  const bool isv = l >= kLanes;
  if (row >= sp.cnt) return;   // (all lanes of a row alike)
  const u32x4* src = reinterpret_cast<const u32x4*>((isv ? V : K) + ((int64_t(bh) * ld + row) * D + piece * kTake) * kEl);
  float x[kTake];
#pragma unroll
  for (int i = 0; i < kTake * kEl / 16; ++i) {
    const u32x4 v = __builtin_nontemporal_load(src + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (DT == RBQ_BF16) {
        x[8 * i + 2 * k] = bf16_lo(v[k]);
        x[8 * i + 2 * k + 1] = bf16_hi(v[k]);
      } else {
        x[4 * i + k] = __uint_as_float(v[k]);
      }
    }
  }
  const int64_t at = int64_t(bh) * cap + sp.off + row;
  uint32_t word;
  u32x2 codes;
  if constexpr (FMT == RBQ_FP4) {
    uint32_t byte;
    codes = encode_fp4<D / 4 / kTake>(x, byte);
    // the row's four bytes: of lanes 0, 2, 4, 6 of eight, or of the four lanes
    word = byte << (8 * (piece * kTake / (D / 4)));
    if constexpr (D == 64) word |= RBQ_DPP_U32(word, 0xB1);
    word |= RBQ_DPP_U32(word, 0x4E);
    if constexpr (D == 128) word |= RBQ_DPP_U32(word, 0x141);
  } else {
    codes = encode_i4<kLanes>(x, word);
  }
  *reinterpret_cast<u32x2*>(KV4 + at * D + l * (kTake / 2)) = codes;
  if (piece == 0) par[2 * at + isv] = word;
}

// Grid (row pieces, (b, kv head)): a thread takes 8 dimensions of kRowsR rows of K or of V, whose
// values leave past the caches.
template <int DT, int FMT, int D>
__global__ __launch_bounds__(kThreads4) void dequantize_kv4_kernel(
    const char* __restrict__ KV4, const uint32_t* __restrict__ par, int cap, int n_rows, int offset, char* __restrict__ K,
    char* __restrict__ V, int64_t ld, int Hkv, const int32_t* __restrict__ seq_off,
    const int32_t* __restrict__ seq_rows) {
  constexpr int kEl = DT == RBQ_BF16 ? 2 : 4, kWords = D / 8, kStep = kThreads4 / (2 * kWords);
  const int bh = blockIdx.y, b = bh / Hkv;
  const Span sp = span_of(b, offset, n_rows, seq_off, seq_rows);
  const int row0 = int(blockIdx.x) * (kStep * kRowsR) + threadIdx.x / (2 * kWords);
  const int l = threadIdx.x % (2 * kWords), piece = l % kWords;
  const bool isv = l >= kWords;
  if (row0 >= sp.cnt) return;
  uint32_t w[kRowsR], word[kRowsR];
#pragma unroll
  for (int u = 0; u < kRowsR; ++u) {   // (behind the last row: that one again)
    const int64_t at = int64_t(bh) * cap + sp.off + min(row0 + u * kStep, sp.cnt - 1);
    w[u] = *reinterpret_cast<const uint32_t*>(KV4 + at * D + 4 * l);
    word[u] = par[2 * at + isv];
  }
#pragma unroll
  for (int u = 0; u < kRowsR; ++u) {
    if (row0 + u * kStep >= sp.cnt) break;
    const f32x2 sc = row_scale<FMT>(word[u], piece * 8 / (D / 4));
    char* dst = (isv ? V : K) + ((int64_t(bh) * ld + row0 + u * kStep) * D + piece * 8) * kEl;
    if constexpr (DT == RBQ_BF16) {
      __builtin_nontemporal_store(word_bf16<FMT>(w[u], sc), reinterpret_cast<u32x4*>(dst));
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = code_value<FMT>(w[u] >> nibble_shift<FMT>(4 * h + i) & 15u, sc);
        __builtin_nontemporal_store(v, reinterpret_cast<f32x4*>(dst) + h);
      }
    }
  }
}

// The instance of a (type, format, head dimension)
template <class F>
void pick(int32_t dtype, int32_t fmt, int32_t head_dim, F f) {
  auto dim = [&](auto dt, auto fm) {
    if (head_dim == 64) f(dt, fm, std::integral_constant<int, 64>{});
    else f(dt, fm, std::integral_constant<int, 128>{});
  };
  auto form = [&](auto dt) {
    if (fmt == RBQ_FP4) dim(dt, std::integral_constant<int, RBQ_FP4>{});
    else dim(dt, std::integral_constant<int, RBQ_I4>{});
  };
  if (dtype == RBQ_BF16) form(std::integral_constant<int, RBQ_BF16>{});
  else form(std::integral_constant<int, RBQ_F32>{});
}
}  // namespace

rbq_status launch_quantize_kv4(int32_t batch, int32_t heads_kv, int32_t head_dim, const void* K, const void* V,
                               int32_t dtype, int64_t ld, int32_t n_new, int32_t offset, int32_t cap, int32_t kv4_dtype,
                               void* KV4, uint32_t* par, const int32_t* seq_off, const int32_t* seq_new,
                               hipStream_t stream) {
  if (n_new == 0) return RBQ_OK;
  const int rows = kThreads4 / (2 * (head_dim / kTake));
  const dim3 grid(uint32_t((int64_t(n_new) + rows - 1) / rows), batch * heads_kv);
  pick(dtype, kv4_dtype, head_dim, [&](auto dt, auto fm, auto d) {
    quantize_kv4_kernel<decltype(dt)::value, decltype(fm)::value, decltype(d)::value><<<grid, kThreads4, 0, stream>>>(
        static_cast<const char*>(K), static_cast<const char*>(V), ld, n_new, offset, cap, static_cast<char*>(KV4), par,
        heads_kv, seq_off, seq_new);
  });
  return hipGetLastError() == hipSuccess ? RBQ_OK : RBQ_EDEVICE;
}

rbq_status launch_dequantize_kv4(int32_t batch, int32_t heads_kv, int32_t head_dim, const void* KV4, const uint32_t* par,
                                 int32_t kv4_dtype, int32_t cap, int32_t n_rows, int32_t offset, void* K, void* V,
                                 int32_t dtype, int64_t ld, const int32_t* seq_off, const int32_t* seq_rows,
                                 hipStream_t stream) {
  if (n_rows == 0) return RBQ_OK;
  const int rows = kRowsR * kThreads4 / (2 * (head_dim / 8));
  const dim3 grid(uint32_t((int64_t(n_rows) + rows - 1) / rows), batch * heads_kv);
  pick(dtype, kv4_dtype, head_dim, [&](auto dt, auto fm, auto d) {
    dequantize_kv4_kernel<decltype(dt)::value, decltype(fm)::value, decltype(d)::value><<<grid, kThreads4, 0, stream>>>(
        static_cast<const char*>(KV4), par, cap, n_rows, offset, static_cast<char*>(K), static_cast<char*>(V), ld, heads_kv,
        seq_off, seq_rows);
  });
  return hipGetLastError() == hipSuccess ? RBQ_OK : RBQ_EDEVICE;
}

}  // namespace rbq
