// rbq_quantize_kv / rbq_dequantize_kv: rows of K and V into and out of the 8-bit
// cache, one scale per (sequence, KV head, block of `block` tokens) and tensor.
//
//   e4m3: s = 2^e with the smallest e that keeps the block's largest magnitude
//         within 448; x / s is then exact and the code is its one rounding
//   int8: s = amax / 127, code = x (1/s) rounded once to a whole number
//
// A token block of one tensor is held in registers by a wave (below 4096 values) or
// by four: its new rows are read once, their largest magnitude is reduced, and the
// codes leave from the same registers, so the bytes are those of the rows and the
// codes, which bound it: K and V of 130816 tokens x 8 heads x 128 in bf16, 805 MB,
// 129 us (6.2 TB/s, a plain copy's rate on this GPU), and the same back 138; half as
// many tokens in fp32, 670 MB, 113 us. (With loads that the caches keep 162; 8 codes
// per lane and store 159; one wave for 4096 values 133, and 163 in fp32, whose loads of
// 16 values per lane do not follow each other; bounds by branches instead of by the
// buffers' ends 131 and 157.)
// A block that holds earlier rows keeps them: where the new rows need a
// larger scale, the held codes are read, multiplied by the ratio of the scales and
// written back (a rounding of at most half a step of the new scale).
#include "rbq_device.h"
#include "rbq_internal.h"

namespace rbq {
namespace {

constexpr int kQuantThreads = 256;
constexpr float kE4m3Max = 448.f, kI8Max = 127.f;
constexpr int kPast = 0x7FFFFF00;      // an offset past the end of every buffer here
constexpr float kRound = 12582912.f;   // 1.5 * 2^23: adding it rounds to a whole number, kept in the low bits

// bits of |x|, 0 for an infinity or NaN: the order of magnitudes is the order of the bits
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
  return u < 0x7F800000u ? u : 0u;
}

// scale of a block from the bits of its largest magnitude (0 for a block of zeros)
template <int FMT>
__device__ __forceinline__ float block_scale(uint32_t amax) {
  if (amax == 0u) return 0.f;
  if constexpr (FMT == RBQ_E4M3) {
    // amax = m 2^x with m in [1, 2); 448 = 1.75 * 2^8, so e = x - 8, one more above m = 1.75
    const int e = int(amax >> 23) - 127 - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return __uint_as_float(uint32_t(max(e, -126) + 127) << 23);   // (subnormal amax: the floor)
  }
  return fmaxf(__uint_as_float(amax) / kI8Max, 1.17549435e-38f);
}

// four codes of y r, each product rounded once; NaN (and an infinity in a block of zeros) gives 0
template <int FMT>
__device__ __forceinline__ uint32_t encode4(const float* x, float r) {
  if constexpr (FMT == RBQ_E4M3) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = x[i] * r;   // exact: r is a power of two
      y[i] = v == v ? fminf(fmaxf(v, -kE4m3Max), kE4m3Max) : 0.f;
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    return uint32_t(w);
  }
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float v = fmaf(x[i], r, kRound);
    b[i] = __float_as_uint(v == v ? fminf(fmaxf(v, kRound - kI8Max), kRound + kI8Max) : kRound);
  }
  const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000C0Cu);
  return lo | hi;
}

// the four values of a word of codes, without the scale
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, float* x) {
  if constexpr (FMT == RBQ_E4M3) {
    x[0] = __builtin_amdgcn_cvt_f32_fp8(int(w), 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8(int(w), 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8(int(w), 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8(int(w), 3);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = float(int8_t(w >> (8 * i)));
  }
}

// Values of a row that a thread takes at once: 16 in bf16, so that their codes leave 16
// bytes per lane, 4 in fp32, so that a wave's loads follow each other.
template <int DT>
constexpr int kTake = DT == RBQ_BF16 ? 16 : 4;
// kTake values of DT, 0 past the buffer's ends. (Read once: streamed past the caches.)
template <int DT>
__device__ __forceinline__ void load_values(__amdgpu_buffer_rsrc_t r, int off, u32x4* raw) {
#pragma unroll
  for (int i = 0; i < (DT == RBQ_BF16 ? 2 : 1); ++i)
    raw[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off + 16 * i, 0, 2));
}
template <int DT>
__device__ __forceinline__ void widen(const u32x4* raw, float* x) {
#pragma unroll
  for (int i = 0; i < kTake<DT>; ++i) {
    if constexpr (DT == RBQ_BF16) x[i] = i % 2 ? bf16_hi(raw[i / 8][i % 8 / 2]) : bf16_lo(raw[i / 8][i % 8 / 2]);
    else x[i] = __uint_as_float(raw[0][i]);
  }
}

// The rows of one call: sequence b's rows [off, off + cnt) of the cache.
struct Span {
  int off, cnt;
};
__device__ __forceinline__ Span span_of(int b, int offset, int rows, const int32_t* seq_off, const int32_t* seq_rows) {
  return Span{seq_off ? min(max(seq_off[b], 0), offset) : offset, seq_rows ? min(max(seq_rows[b], 0), rows) : rows};
}

// Grid (token blocks of a sequence / units per workgroup, (b, kv head), K or V).
// T threads take a token block of D-dimension rows, 16 CH values each.
template <int DT, int FMT, int T, int CH>
__global__ __launch_bounds__(kQuantThreads) void quantize_kv_kernel(
    const char* __restrict__ K, const char* __restrict__ V, int64_t ld, int n_new, int offset, int cap, int bshift,
    int dshift, char* __restrict__ K8, char* __restrict__ V8, float* __restrict__ k_scale, float* __restrict__ v_scale,
    int Hkv, const int32_t* __restrict__ seq_off, const int32_t* __restrict__ seq_new) {
  constexpr int kEl = DT == RBQ_BF16 ? 2 : 4, kRaw = DT == RBQ_BF16 ? 2 : 1;
  constexpr int kVals = kTake<DT>, kPieces = CH * 16 / kVals;
  constexpr int kUnits = kQuantThreads / T;
  __shared__ uint32_t red[kQuantThreads / kWave];
  const int bh = blockIdx.y, b = bh / Hkv;
  const Span sp = span_of(b, offset, n_new, seq_off, seq_new);
  const int t = threadIdx.x % T;   // (a unit is whole waves)
  const int blk = (sp.off >> bshift) + int(blockIdx.x) * kUnits + __builtin_amdgcn_readfirstlane(threadIdx.x / T);
  const int row0 = blk << bshift;
  const int end = sp.off + sp.cnt;
  if (row0 >= end) return;
  // value e of the token block; [first, last) are the new ones, those before them held. Loads and
  // stores of the others lie past the ends of the buffers: they give 0 and are dropped.
  const int first = max(sp.off - row0, 0) << dshift, last = min(end - row0, 1 << bshift) << dshift;
  const char* rows = (blockIdx.z ? V : K) + ((int64_t(bh) * ld + max(row0 - sp.off, 0)) << dshift) * kEl;
  const __amdgpu_buffer_rsrc_t src = make_rsrc(rows, uint32_t(last - first) * kEl);
  char* codes = (blockIdx.z ? V8 : K8) + ((int64_t(bh) * cap + row0) << dshift);
  const __amdgpu_buffer_rsrc_t dst = make_rsrc(codes + first, uint32_t(last - first));
  const int64_t sidx = int64_t(bh) * ((int64_t(cap) + (1 << bshift) - 1) >> bshift) + blk;
  float* scale = (blockIdx.z ? v_scale : k_scale) + sidx;
  const float old = row0 < sp.off ? *scale : 0.f;   // rows that the block holds already

  u32x4 raw[kPieces][kRaw];
#pragma unroll
  for (int c = 0; c < kPieces; ++c) {
    const int e = (c * T + t) * kVals;
    load_values<DT>(src, e >= first ? (e - first) * kEl : kPast, raw[c]);
  }
  uint32_t amax = 0u;
#pragma unroll
  for (int c = 0; c < kPieces; ++c) {
    float x[kVals];
    widen<DT>(raw[c], x);
#pragma unroll
    for (int i = 0; i < kVals; ++i) amax = max(amax, finite_bits(x[i]));
  }
  amax = wave_max_u32(amax);
  if constexpr (T > kWave) {
    if (lane_id() == 0) red[threadIdx.x / kWave] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kQuantThreads / kWave; ++w) amax = max(amax, red[w]);
  }
  const float s = fmaxf(block_scale<FMT>(amax), old);
  const float r = s > 0.f ? 1.f / s : 0.f;
#pragma unroll
  for (int c = 0; c < kPieces; ++c) {
    const int e = (c * T + t) * kVals, at = e >= first ? e - first : kPast;
    float x[kVals];
    widen<DT>(raw[c], x);
    if constexpr (kVals == 16) {
      const u32x4 now = {encode4<FMT>(x, r), encode4<FMT>(x + 4, r), encode4<FMT>(x + 8, r), encode4<FMT>(x + 12, r)};
      __builtin_amdgcn_raw_buffer_store_b128(now, dst, at, 0, 0);
    } else {
      __builtin_amdgcn_raw_buffer_store_b32(encode4<FMT>(x, r), dst, at, 0, 0);
    }
  }
  if (row0 < sp.off && s > old) {   // the held rows under the larger scale
    const float ratio = old / s;
    for (int e = 4 * t; e < first; e += 4 * T) {
      uint32_t* at = reinterpret_cast<uint32_t*>(codes + e);
      float x[4];
      decode4<FMT>(*at, x);
      *at = encode4<FMT>(x, ratio);
    }
  }
  if (t == 0) *scale = s;
}

// Grid (row pieces, (b, kv head), K or V): a thread takes 8 dimensions of a row.
template <int DT, int FMT>
__global__ __launch_bounds__(kQuantThreads) void dequantize_kv_kernel(
    const uint32_t* __restrict__ K8, const uint32_t* __restrict__ V8, const float* __restrict__ k_scale,
    const float* __restrict__ v_scale, int cap, int bshift, int dshift, int n_rows, int offset, char* __restrict__ K,
    char* __restrict__ V, int64_t ld, int Hkv, const int32_t* __restrict__ seq_off,
    const int32_t* __restrict__ seq_rows) {
  constexpr int kEl = DT == RBQ_BF16 ? 2 : 4;
  const int bh = blockIdx.y, b = bh / Hkv;
  const Span sp = span_of(b, offset, n_rows, seq_off, seq_rows);
  const int cshift = dshift - 3;
  const int64_t e = int64_t(blockIdx.x) * kQuantThreads + threadIdx.x;
  const int row = int(e >> cshift), dim = int(e & ((1 << cshift) - 1)) * 8;
  if (row >= sp.cnt) return;
  const int at = sp.off + row;   // cache row
  const uint32_t* src = (blockIdx.z ? V8 : K8) + ((int64_t(bh) * cap + at) << (dshift - 2)) + dim / 4;
  const int64_t nblk = (int64_t(cap) + (1 << bshift) - 1) >> bshift;
  const float s = (blockIdx.z ? v_scale : k_scale)[int64_t(bh) * nblk + (at >> bshift)];
  const u32x2 w = *reinterpret_cast<const u32x2*>(src);
  float x[8];
  decode4<FMT>(w.x, x);
  decode4<FMT>(w.y, x + 4);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= s;
  char* dst = (blockIdx.z ? V : K) + (((int64_t(bh) * ld + row) << dshift) + dim) * kEl;
  if constexpr (DT == RBQ_BF16) {
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    typedef float f32x8 __attribute__((ext_vector_type(8)));
    f32x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[i];
    *reinterpret_cast<u32x4*>(dst) = __builtin_bit_cast(u32x4, __builtin_convertvector(v, bf16x8));
  } else {
    reinterpret_cast<f32x4*>(dst)[0] = f32x4{x[0], x[1], x[2], x[3]};
    reinterpret_cast<f32x4*>(dst)[1] = f32x4{x[4], x[5], x[6], x[7]};
  }
}

int log2i(int x) { return __builtin_ctz(unsigned(x)); }

template <int DT, int FMT>
void launch_quantize_form(int pieces, dim3 grid, hipStream_t stream, const char* K, const char* V, int64_t ld, int n_new,
                          int offset, int cap, int bshift, int dshift, char* K8, char* V8, float* ks, float* vs,
                          int Hkv, const int32_t* seq_off, const int32_t* seq_new) {
#define RBQ_QUANT_FORM(T, CH)                                                                                     \
  quantize_kv_kernel<DT, FMT, T, CH><<<grid, kQuantThreads, 0, stream>>>(K, V, ld, n_new, offset, cap, bshift, dshift, \
                                                                         K8, V8, ks, vs, Hkv, seq_off, seq_new)
  switch (pieces) {   // of 16 values in a token block: 64 threads below 256, 256 from there on
    case 64: RBQ_QUANT_FORM(64, 1); break;
    case 128: RBQ_QUANT_FORM(64, 2); break;
    case 256: RBQ_QUANT_FORM(256, 1); break;
    case 512: RBQ_QUANT_FORM(256, 2); break;
    case 1024: RBQ_QUANT_FORM(256, 4); break;
    default: RBQ_QUANT_FORM(256, 8); break;
  }
#undef RBQ_QUANT_FORM
}
}  // namespace

rbq_status launch_quantize_kv(int32_t batch, int32_t heads_kv, int32_t head_dim, const void* K, const void* V,
                              int32_t dtype, int64_t ld, int32_t n_new, int32_t offset, int32_t cap, int32_t block,
                              int32_t kv8_dtype, void* K8, void* V8, float* k_scale, float* v_scale,
                              const int32_t* seq_off, const int32_t* seq_new, hipStream_t stream) {
  if (n_new == 0) return RBQ_OK;
  const int bshift = log2i(block), dshift = log2i(head_dim), pieces = block * head_dim / 16;
  const int units = pieces < 256 ? kQuantThreads / kWave : 1;
  // token blocks a sequence's rows can touch (ragged: from any place in the first)
  const int64_t first = seq_off ? 0 : offset >> bshift;
  const int64_t blocks =
      seq_off ? (int64_t(block) - 1 + n_new + block - 1) >> bshift : ((int64_t(offset) + n_new - 1) >> bshift) - first + 1;
  const dim3 grid((blocks + units - 1) / units, batch * heads_kv, 2);
  const char *k = static_cast<const char*>(K), *v = static_cast<const char*>(V);
  char *k8 = static_cast<char*>(K8), *v8 = static_cast<char*>(V8);
#define RBQ_QUANT(DT, FMT)                                                                                              \
  launch_quantize_form<DT, FMT>(pieces, grid, stream, k, v, ld, n_new, offset, cap, bshift, dshift, k8, v8, k_scale, \
                                v_scale, heads_kv, seq_off, seq_new)
  if (dtype == RBQ_BF16) {
    if (kv8_dtype == RBQ_E4M3) RBQ_QUANT(RBQ_BF16, RBQ_E4M3);
    else RBQ_QUANT(RBQ_BF16, RBQ_I8);
  } else {
    if (kv8_dtype == RBQ_E4M3) RBQ_QUANT(RBQ_F32, RBQ_E4M3);
    else RBQ_QUANT(RBQ_F32, RBQ_I8);
  }
#undef RBQ_QUANT
  return hipGetLastError() == hipSuccess ? RBQ_OK : RBQ_EDEVICE;
}

rbq_status launch_dequantize_kv(int32_t batch, int32_t heads_kv, int32_t head_dim, const void* K8, const void* V8,
                                int32_t kv8_dtype, int32_t block, const float* k_scale, const float* v_scale,
                                int32_t cap, int32_t n_rows, int32_t offset, void* K, void* V, int32_t dtype,
                                int64_t ld, const int32_t* seq_off, const int32_t* seq_rows, hipStream_t stream) {
  if (n_rows == 0) return RBQ_OK;
  const int bshift = log2i(block), dshift = log2i(head_dim);
  const int64_t pieces = int64_t(n_rows) << (dshift - 3);
  const dim3 grid((pieces + kQuantThreads - 1) / kQuantThreads, batch * heads_kv, 2);
#define RBQ_DEQUANT(DT, FMT)                                                                                         \
  dequantize_kv_kernel<DT, FMT><<<grid, kQuantThreads, 0, stream>>>(                                                 \
      static_cast<const uint32_t*>(K8), static_cast<const uint32_t*>(V8), k_scale, v_scale, cap, bshift, dshift, n_rows, \
      offset, static_cast<char*>(K), static_cast<char*>(V), ld, heads_kv, seq_off, seq_rows)
  if (dtype == RBQ_BF16) {
    if (kv8_dtype == RBQ_E4M3) RBQ_DEQUANT(RBQ_BF16, RBQ_E4M3);
    else RBQ_DEQUANT(RBQ_BF16, RBQ_I8);
  } else {
    if (kv8_dtype == RBQ_E4M3) RBQ_DEQUANT(RBQ_F32, RBQ_E4M3);
    else RBQ_DEQUANT(RBQ_F32, RBQ_I8);
  }
#undef RBQ_DEQUANT
  return hipGetLastError() == hipSuccess ? RBQ_OK : RBQ_EDEVICE;
}

}  // namespace rbq
