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
// bf16, 678 MB either way, written in 115 us (5.9 TB/s) and read back in 104 (6.5; stores that
// the caches keep 121, one row a thread 110). Writing has its arithmetic beside the bytes: with a
// look at each value for infinities and NaN (now for a wave's at once, and the values' own way
// only where there is one) 16 values took 210 (fp4) to 400 (int4) vector instructions, and the
// rows above 125 us, 16 x 256 of int4 7.5 instead of 5.6. (Two rows a thread were no faster then,
// and 16 x 256 rows slower by 0.5.)
#include <type_traits>

#include "kv4_dev.h"

namespace rbq {
namespace {

constexpr int kThreads4 = 256;
constexpr float kLeast = 1.17549435e-38f;   // 2^-126, the least scale and step
constexpr float kMost = 8.50705917e37f;     // 2^126: int4 takes finite values beyond as this
constexpr float kRound = 12582912.f;        // 1.5 * 2^23: adding it rounds to a whole number, kept in the low bits
constexpr uint32_t kRoundBits = 0x4B400000u;   // its bits
constexpr int kTake = 16;                   // values of a row and tensor that a thread takes
constexpr int kRowsR = 2;                   // rows that a thread reads back

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

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

// A thread's 16 values as they were loaded.
template <int DT>
struct Taken {
  static constexpr int kWords = DT == RBQ_BF16 ? kTake / 2 : kTake;
  uint32_t w[kWords];
  __device__ __forceinline__ void values(float* x) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (DT == RBQ_BF16) {
        x[2 * i] = bf16_lo(w[i]);
        x[2 * i + 1] = bf16_hi(w[i]);
      } else {
        x[i] = __uint_as_float(w[i]);
      }
    }
  }
  // the bits of the largest magnitude (their order is the magnitudes', NaN's above infinity's)
  __device__ __forceinline__ uint32_t amax() const {
    if constexpr (DT == RBQ_BF16) {
      u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7FFF7FFFu);
#pragma unroll
      for (int i = 1; i < kWords; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
      return uint32_t(max(m.x, m.y)) << 16;
    } else {
      uint32_t m = 0u;
#pragma unroll
      for (int i = 0; i < kWords; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
      return m;
    }
  }
  // the smallest and the largest, NaN below or above all (as whole numbers, whose order the values'
  // is once negative ones' lower bits are turned)
  __device__ __forceinline__ f32x2 extremes() const {
    if constexpr (DT == RBQ_BF16) {
      auto turn = [](i16x2 v) { return v ^ ((v >> 15) & i16x2{0x7FFF, 0x7FFF}); };
      i16x2 lo = turn(__builtin_bit_cast(i16x2, w[0])), hi = lo;
#pragma unroll
      for (int i = 1; i < kWords; ++i) {
        const i16x2 v = turn(__builtin_bit_cast(i16x2, w[i]));
        lo = __builtin_elementwise_min(lo, v);
        hi = __builtin_elementwise_max(hi, v);
      }
      const uint32_t r = __builtin_bit_cast(uint32_t, turn(i16x2{min(lo.x, lo.y), max(hi.x, hi.y)}));
      return f32x2{bf16_lo(r), bf16_hi(r)};
    } else {
      auto turn = [](int32_t v) { return v ^ ((v >> 31) & 0x7FFFFFFF); };
      int32_t lo = turn(int32_t(w[0])), hi = lo;
#pragma unroll
      for (int i = 1; i < kWords; ++i) {
        lo = min(lo, turn(int32_t(w[i])));
        hi = max(hi, turn(int32_t(w[i])));
      }
      return f32x2{__uint_as_float(uint32_t(turn(lo))), __uint_as_float(uint32_t(turn(hi)))};
    }
  }
};

// e of a group whose largest magnitude is amax = m 2^x, m in [1, 2): 7 = 1.75 * 2^2, so x - 2,
// one more above m = 1.75
__device__ __forceinline__ int fp4_exponent(uint32_t amax) {
  const int e = int(amax >> 23) - 127 - 2 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, -126), 125);
}

// 16 values of fp4: their codes, and their group's exponent byte. Where a whole wave's are finite
// the conversion takes them as they are, scale and bounds with it.
template <int LANES, int DT>
__device__ __forceinline__ u32x2 encode_fp4(const Taken<DT>& raw, uint32_t& byte) {
  uint32_t top = raw.amax();
  if (__ballot(top >= 0x7F800000u) == 0ull) {
    if constexpr (LANES >= 2) top = max(top, RBQ_DPP_U32(top, 0xB1));
    const int ec = fp4_exponent(top);
    byte = top == 0u ? 0u : uint32_t(ec + 127);
    const float scale = __uint_as_float(uint32_t(ec + 127) << 23);
    u32x2 w;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      auto pair = [&](uint32_t v, int p, auto place) {
        if constexpr (DT == RBQ_BF16) {
          return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(v, __builtin_bit_cast(bf16x2_t, raw.w[4 * h + p]), scale,
                                                           decltype(place)::value);
        } else {
          return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, __uint_as_float(raw.w[8 * h + 2 * p]),
                                                          __uint_as_float(raw.w[8 * h + 2 * p + 1]), scale, decltype(place)::value);
        }
      };
      uint32_t v = pair(0u, 0, std::integral_constant<int, 0>{});
      v = pair(v, 1, std::integral_constant<int, 1>{});
      v = pair(v, 2, std::integral_constant<int, 2>{});
      v = pair(v, 3, std::integral_constant<int, 3>{});
      w[h] = top == 0u ? 0u : v;
    }
    return w;
  }
  float x[kTake];
  raw.values(x);
  uint32_t amax = 0u;
#pragma unroll
  for (int i = 0; i < kTake; ++i) {
    const uint32_t u = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    amax = max(amax, u < 0x7F800000u ? u : 0u);   // (the order of magnitudes is the order of the bits)
  }
  if constexpr (LANES >= 2) amax = max(amax, RBQ_DPP_U32(amax, 0xB1));
  const int ec = fp4_exponent(amax);
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

// A row's base, step and the step's reciprocal from its extremes
struct Line {
  float m, s, r;
};
__device__ __forceinline__ Line line_of(float lo, float hi) {
  Line a;
  a.m = bf16_down(lo);
  const float d = hi - a.m;
  a.s = d > 0.f ? bf16_up(fmaxf(d / 15.f, kLeast)) : 0.f;
  a.r = a.s > 0.f ? 1.f / a.s : 0.f;
  return a;
}

// 16 values of int4: their codes, and their row's word. Where a whole wave's are within 2^126 no
// code is beyond 0 .. 15: x lies between m and hi, and s is no less than d / 15.
template <int LANES, int DT>
__device__ __forceinline__ u32x2 encode_i4(const Taken<DT>& raw, uint32_t& word) {
  float x[kTake];
  raw.values(x);
  const f32x2 ends = raw.extremes();
  float lo = ends.x, hi = ends.y;
  auto least = [](float a, float b) { return fminf(a, b); };
  auto most = [](float a, float b) { return fmaxf(a, b); };
  u32x2 w;
  if (__ballot(!(lo >= -kMost && hi <= kMost)) == 0ull) {
    const Line a = line_of(lanes_reduce<LANES>(lo, least), lanes_reduce<LANES>(hi, most));
    word = __float_as_uint(a.s) >> 16 | __float_as_uint(a.m);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t v = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i)   // (what the numbers have beside their low bits is taken off the word)
        v += (__float_as_uint(fmaf(x[8 * h + i] - a.m, a.r, kRound)) << nibble_shift<RBQ_I4>(i)) -
             (kRoundBits << nibble_shift<RBQ_I4>(i));
      w[h] = v;
    }
    return w;
  }
  lo = INFINITY, hi = -INFINITY;
#pragma unroll
  for (int i = 0; i < kTake; ++i) {
    const bool f = is_finite(x[i]);
    const float v = fminf(fmaxf(x[i], -kMost), kMost);
    lo = f ? fminf(lo, v) : lo;
    hi = f ? fmaxf(hi, v) : hi;
  }
  lo = lanes_reduce<LANES>(lo, least);
  hi = lanes_reduce<LANES>(hi, most);
  if (lo > hi) lo = hi = 0.f;   // no finite value
  const Line a = line_of(lo, hi);
  word = __float_as_uint(a.s) >> 16 | __float_as_uint(a.m);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t v = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float y = x[8 * h + i] == x[8 * h + i] ? x[8 * h + i] : 0.f;
      const float t = fmaf(y - a.m, a.r, kRound);   // one rounding, to a whole number
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
  Taken<DT> x;
#pragma unroll
  for (int i = 0; i < kTake * kEl / 16; ++i) {
    const u32x4 v = __builtin_nontemporal_load(src + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) x.w[4 * i + k] = v[k];
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
