// rbq_prefill_attention: softmax attention of prompts (or chunks of them over rows
// already cached), causal or full, grouped heads, packed sequences.
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(sm_scale (<q_i, k_j> - max_j)),
//   over the j < Lk of the query's sequence, for causal j <= i + Lk - Lq
//
// One pass over the keys with the running maximum and sum of the softmax.
#include <algorithm>

#include "rbq_device.h"
#include "rbq_internal.h"

namespace rbq {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kPWaves = 4;
constexpr int kPThreads = kPWaves * kWave;
constexpr int kPKeys = 64;       // keys per step
constexpr float kLn2 = 0.69314718055994531f;

#define RBQ_LDS __attribute__((address_space(3)))

// A query tile: the rows (token, head of the group) of one sequence and KV head,
// row r = token r / G, head r % G of the group.
struct TileId {
  int b, tile;   // sequence, tile of its rows; b < 0: none
  int q0, nq;    // first token of the sequence on the packed axis, tokens
  int nk;        // keys
  int64_t k0;    // first row of the sequence's keys (packed), 0 otherwise
};

// The tile'th tile of the batch: sequences in order, each with ceil(tokens * G / BM).
__device__ __forceinline__ TileId find_tile(int tile, int batch, int G, int BM, int total_q, int max_k, int kv_rows,
                                            bool packed, const int32_t* __restrict__ cu_q,
                                            const int32_t* __restrict__ cu_k) {
  const int lane = lane_id();
  TileId t{-1, 0, 0, 0, 0, 0};
  int before = 0;
  for (int b0 = 0; b0 < batch; b0 += kWave) {
    const int b = min(b0 + lane, batch - 1);
    const int qa = min(max(cu_q[b], 0), total_q), qb = min(max(cu_q[b + 1], 0), total_q);
    const int ka = cu_k[b], kb = cu_k[b + 1];
    const int nq = max(qb - qa, 0);
    const int tiles = b0 + lane < batch ? int((int64_t(nq) * G + BM - 1) / BM) : 0;
    int inc = tiles;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int v = __shfl_up(inc, o, kWave);
      inc += lane >= o ? v : 0;
    }
    const unsigned long long mine = __ballot(tile >= before + inc - tiles && tile < before + inc);
    if (mine != 0ull) {
      const int l = __builtin_ctzll(mine);
      t.b = b0 + l;
      t.tile = tile - before - __builtin_amdgcn_readlane(inc - tiles, l);
      t.q0 = __builtin_amdgcn_readlane(qa, l);
      t.nq = __builtin_amdgcn_readlane(nq, l);
      // keys inside [0, kv_rows) of the packed axis, or of the sequence's own rows
      const int a = packed ? min(max(__builtin_amdgcn_readlane(ka, l), 0), kv_rows) : 0;
      const int n = max(__builtin_amdgcn_readlane(kb, l) - __builtin_amdgcn_readlane(ka, l), 0);
      t.nk = min(min(n, max_k), kv_rows - a);
      t.k0 = a;
      return t;
    }
    before += __builtin_amdgcn_readlane(inc, kWave - 1);
  }
  return t;
}

// 16 bytes per lane from global memory straight into LDS (lane l's at lds + 16 l)
__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t r, void* lds, int off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (RBQ_LDS void*)lds, 16, off, 0, 0, 0);
}

// A lane's part of a finished row: dimensions 32 d + 8 g + 4 h .. +4. With one split
// the output itself, otherwise the split's state {m, l, acc}.
template <int D, int DT, int NQ>
__device__ __forceinline__ void store_row(const f32x16 (&o)[D / 32][NQ], int i, float m, float sum, int64_t row, int h,
                                          void* __restrict__ out, float* __restrict__ lse, float* __restrict__ part) {
  float* pr = part + (row * gridDim.y + blockIdx.y) * (D + 2);
  const float scale = part ? 1.f : sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      const f32x4 v = f32x4{o[d][i][4 * g], o[d][i][4 * g + 1], o[d][i][4 * g + 2], o[d][i][4 * g + 3]} * scale;
      const int at = 32 * d + 8 * g + 4 * h;
      if (part) {
        f32x2* p = reinterpret_cast<f32x2*>(pr + 2 + at);
        p[0] = f32x2{v.x, v.y};
        p[1] = f32x2{v.z, v.w};
      } else if constexpr (DT == RBQ_BF16) {
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(out) + row * D + at) =
            __builtin_bit_cast(u32x2, __builtin_convertvector(v, bf16x4));
      } else {
        *reinterpret_cast<f32x4*>(static_cast<float*>(out) + row * D + at) = v;
      }
    }
  if (h != 0) return;
  if (part)
    *reinterpret_cast<f32x2*>(pr) = f32x2{sum > 0.f ? m : -INFINITY, sum};
  else if (lse)
    lse[row] = sum > 0.f ? (m + log2f(sum)) * kLn2 : -INFINITY;
}

// D: head dimension; QT: 32-row query tiles per wave
template <int D, int QT>
__global__ __launch_bounds__(kPThreads, QT == 1 ? 2 : 1) void prefill_kernel(
    const uint16_t* __restrict__ q, int64_t q_ld, const uint16_t* __restrict__ K, const uint16_t* __restrict__ V,
    int64_t kv_ld, int64_t kv_head, int64_t kv_seq, int kv_rows, const int32_t* __restrict__ cu_q,
    const int32_t* __restrict__ cu_k, int batch, int total_q, int max_k, int causal, float scale_log2e,
    uint16_t* __restrict__ out, float* __restrict__ lse, float* __restrict__ part, int Hq, int Hkv, int tiles, int kchunk) {
  constexpr int BM = 32 * QT * kPWaves, C = D / 8, KB = D / 16, DT = D / 32, RB = D * 2;   // chunks, k-blocks, dim tiles, row bytes
  constexpr int KT = kPKeys / 32;
  __shared__ __attribute__((aligned(1024))) char ldsK[2][kPKeys * RB], ldsV[2][kPKeys * RB];
  const int G = Hq / Hkv;
  const int hk = blockIdx.x % Hkv;
  const TileId t = find_tile(tiles - 1 - int(blockIdx.x) / Hkv, batch, G, BM, total_q, max_k, kv_rows, kv_seq == 0, cu_q, cu_k);
  if (t.b < 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int x = lane & 31, h = lane >> 5;
  const int rows = t.nq * G;
  const int row0 = t.tile * BM;
  const int shift = t.nk - t.nq;                                   // query token i sees keys <= i + shift
  auto visible = [&](int token) { return causal ? min(max(token + shift + 1, 0), t.nk) : t.nk; };
  const int kend = visible((min(row0 + BM, rows) - 1) / G);         // keys that some row of the block sees
  const int wrow = row0 + wave * (32 * QT);
  const int kbeg = int(blockIdx.y) * kchunk, kstop = min(kend, kbeg + kchunk);   // this block's keys
  const int wend = wrow < rows ? visible((min(wrow + 32 * QT, rows) - 1) / G) : 0;   // of the wave
  const int wmin = visible(min(wrow, rows - 1) / G);                // keys that every row of the wave sees

  // queries: B operand, lane (row x, half h) holds dimensions 16 kb + 8 h .. +8
  bf16x8 qf[QT][KB];
  int token[QT], head[QT], lim[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const int r = min(wrow + 32 * i + x, rows - 1);
    token[i] = r / G;
    head[i] = hk * G + (r - token[i] * G);
    lim[i] = visible(token[i]);
    const uint16_t* p = q + int64_t(t.q0 + token[i]) * q_ld + head[i] * D + 8 * h;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) qf[i][kb] = *reinterpret_cast<const bf16x8*>(p + 16 * kb);
  }

  const int64_t kvoff = (kv_seq == 0 ? t.k0 * kv_ld : int64_t(t.b) * kv_seq) + int64_t(hk) * kv_head;
  const uint16_t *Kb = K + kvoff, *Vb = V + kvoff;
  // staging: one instruction moves 1024 bytes, 1024 / RB rows; chunk position p of row r
  // holds chunk p ^ f(r), so that the reads below touch every bank once
  constexpr int kRowsPer = 1024 / RB, kIssues = kPKeys / kRowsPer / kPWaves;
  const int srow = lane / C, spos = lane % C;
  int koff[kIssues], voff[kIssues];
#pragma unroll
  for (int i = 0; i < kIssues; ++i) {
    const int r = (wave * kIssues + i) * kRowsPer + srow;
    koff[i] = int(r * kv_ld * 2) + ((spos ^ (r & (C - 1))) * 16);
    voff[i] = int(r * kv_ld * 2) + ((spos ^ (2 * (r & 3))) * 16);
  }
  auto stage = [&](int k0, int buf) {
    const int left = min(t.nk - k0, kPKeys);
    const uint32_t bytes = uint32_t((left - 1) * kv_ld * 2 + RB);
    const __amdgpu_buffer_rsrc_t kr = make_rsrc(Kb + k0 * kv_ld, bytes), vr = make_rsrc(Vb + k0 * kv_ld, bytes);
    if (left < kPKeys) {   // the last rows again in place of those behind them
#pragma unroll
      for (int i = 0; i < kIssues; ++i) {
        const int r = (wave * kIssues + i) * kRowsPer + srow, at = int(min(r, left - 1) * kv_ld * 2);
        load_lds16(kr, &ldsK[buf][(wave * kIssues + i) * 1024], at + ((spos ^ (r & (C - 1))) * 16));
        load_lds16(vr, &ldsV[buf][(wave * kIssues + i) * 1024], at + ((spos ^ (2 * (r & 3))) * 16));
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kIssues; ++i) {
      load_lds16(kr, &ldsK[buf][(wave * kIssues + i) * 1024], koff[i]);
      load_lds16(vr, &ldsV[buf][(wave * kIssues + i) * 1024], voff[i]);
    }
  };
  // read addresses: K rows (lane: key x, chunk 2 kb + h), V columns by the transposing
  // read (16 lanes: 4 keys x 16 dimensions; lane i gives key i / 4, dimensions 4 (i % 4) .. +4)
  const int kbase = x * RB + ((h ^ (x & (C - 1))) * 16);
  const int i16 = lane & 15, g16 = (lane >> 4) & 1;
  const int vbase = (4 * h + (i16 >> 2)) * RB + (((2 * g16 + ((i16 & 3) >> 1)) ^ (2 * (i16 >> 2))) * 16) + (i16 & 1) * 8;

  f32x16 o[DT][QT];
  float m[QT], l[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][i][r] = 0.f;
  }

  if (kbeg < kstop) stage(kbeg, 0);
  int buf = 0;
  for (int k0 = kbeg; k0 < kstop; k0 += kPKeys, buf ^= 1) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (k0 + kPKeys < kstop) stage(k0 + kPKeys, buf ^ 1);
    if (k0 >= wend) continue;
    f32x16 s[KT][QT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < QT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kt][i][r] = 0.f;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(&ldsK[buf][kt * 32 * RB + (kbase ^ (kb * 32))]);
#pragma unroll
        for (int i = 0; i < QT; ++i) s[kt][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[i][kb], s[kt][i], 0, 0, 0);
      }
    if (k0 + kPKeys > wmin) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < QT; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            s[kt][i][r] = k0 + 32 * kt + 8 * (r / 4) + 4 * h + r % 4 < lim[i] ? s[kt][i][r] : -INFINITY;
    }
    bf16x8 p[KT][QT][2];
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      float mx = s[0][i][0];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kt][i][r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, kWave)) * scale_log2e;
      const float mn = fmaxf(m[i], mx);
      if (__ballot(mn != m[i])) {
        const float corr = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - mn);
        l[i] *= corr;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][i][r] *= corr;
        m[i] = mn;
      }
      const float mref = m[i] == -INFINITY ? 0.f : m[i];
      float sum = 0.f;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          f32x8 e;
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            e[r] = __builtin_amdgcn_exp2f(fmaf(s[kt][i][8 * g + r], scale_log2e, -mref));
            sum += e[r];
          }
          p[kt][i][g] = __builtin_convertvector(e, bf16x8);
        }
      l[i] += sum;
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const int at = (kt * 32 + g * 16) * RB + (vbase ^ (d * 64));
          const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((RBQ_LDS s16x4*)&ldsV[buf][at]);
          const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((RBQ_LDS s16x4*)&ldsV[buf][at + 8 * RB]);
          const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int i = 0; i < QT; ++i) o[d][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p[kt][i][g], o[d][i], 0, 0, 0);
        }
  }

#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const float sum = l[i] + __shfl_xor(l[i], 32, kWave);
    if (wrow + 32 * i + x < rows)
      store_row<D, RBQ_BF16>(o, i, m[i], sum, int64_t(t.q0 + token[i]) * Hq + head[i], h, out, lse, part);
  }
}

// fp32 rows: the same on v_mfma_f32_32x32x2_f32, products and probabilities in fp32.
// Lane half h of the logits product takes dimensions h D / 2 .. +D / 2 (the order of the
// dimensions is free as long as K and the queries share it), so both read four at once;
// register r of the result is key 8 (r / 4) + 4 h + r % 4, which is row k = h of step r of
// the second product.
constexpr int kFKeys = 32;
template <int D>
__global__ __launch_bounds__(kPThreads, 2) void prefill_f32_kernel(
    const float* __restrict__ q, int64_t q_ld, const float* __restrict__ K, const float* __restrict__ V, int64_t kv_ld,
    int64_t kv_head, int64_t kv_seq, int kv_rows, const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_k,
    int batch, int total_q, int max_k, int causal, float scale_log2e, float* __restrict__ out, float* __restrict__ lse,
    float* __restrict__ part, int Hq, int Hkv, int tiles, int kchunk) {
  constexpr int BM = 32 * kPWaves, DT = D / 32, LD = D + 4;   // (padded rows: four consecutive keys in other banks)
  constexpr int kPieces = kFKeys * D / 4 / kPThreads;        // 16-byte pieces per thread and tensor
  __shared__ __attribute__((aligned(16))) float ldsK[kFKeys][LD], ldsV[kFKeys][LD];
  const int G = Hq / Hkv;
  const int hk = blockIdx.x % Hkv;
  const TileId t = find_tile(tiles - 1 - int(blockIdx.x) / Hkv, batch, G, BM, total_q, max_k, kv_rows, kv_seq == 0, cu_q, cu_k);
  if (t.b < 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int x = lane & 31, h = lane >> 5;
  const int rows = t.nq * G, row0 = t.tile * BM, shift = t.nk - t.nq;
  auto visible = [&](int token) { return causal ? min(max(token + shift + 1, 0), t.nk) : t.nk; };
  const int kend = visible((min(row0 + BM, rows) - 1) / G);
  const int kbeg = int(blockIdx.y) * kchunk, kstop = min(kend, kbeg + kchunk);
  const int wrow = row0 + wave * 32;
  const int wend = wrow < rows ? visible((min(wrow + 32, rows) - 1) / G) : 0;
  const int r0 = min(wrow + x, rows - 1), token = r0 / G, head = hk * G + (r0 - token * G), lim = visible(token);
  f32x4 qf[D / 8];
  {
    const float* p = q + int64_t(t.q0 + token) * q_ld + head * D + h * (D / 2);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) qf[i] = *reinterpret_cast<const f32x4*>(p + 4 * i) * scale_log2e;
  }
  const int64_t kvoff = (kv_seq == 0 ? t.k0 * kv_ld : int64_t(t.b) * kv_seq) + int64_t(hk) * kv_head;
  f32x4 kreg[kPieces], vreg[kPieces];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int e = i * kPThreads + threadIdx.x, r = e / (D / 4), c = e % (D / 4);
      const int64_t at = kvoff + int64_t(min(k0 + r, t.nk - 1)) * kv_ld + 4 * c;
      kreg[i] = *reinterpret_cast<const f32x4*>(K + at);
      vreg[i] = *reinterpret_cast<const f32x4*>(V + at);
    }
  };
  f32x16 o[DT][1];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][0][r] = 0.f;
  float m = -INFINITY, l = 0.f;
  if (kbeg < kstop) fetch(kbeg);
  for (int k0 = kbeg; k0 < kstop; k0 += kFKeys) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int e = i * kPThreads + threadIdx.x, r = e / (D / 4), c = e % (D / 4);
      *reinterpret_cast<f32x4*>(&ldsK[r][4 * c]) = kreg[i];
      *reinterpret_cast<f32x4*>(&ldsV[r][4 * c]) = vreg[i];
    }
    __syncthreads();
    if (k0 + kFKeys < kstop) fetch(k0 + kFKeys);
    if (k0 >= wend) continue;
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(&ldsK[x][h * (D / 2) + 4 * i]);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], qf[i][e], s, 0, 0, 0);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = k0 + 8 * (r / 4) + 4 * h + r % 4 < lim ? s[r] : -INFINITY;
      mx = fmaxf(mx, s[r]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
    const float mn = fmaxf(m, mx);
    if (__ballot(mn != m)) {
      const float corr = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][0][r] *= corr;
      m = mn;
    }
    const float mref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(s[r] - mref);
      l += s[r];
    }
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int d = 0; d < DT; ++d)
        o[d][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(ldsV[8 * (r / 4) + 4 * h + r % 4][32 * d + x], s[r], o[d][0], 0, 0, 0);
  }
  const float sum = l + __shfl_xor(l, 32, kWave);
  if (wrow + x < rows)
    store_row<D, RBQ_F32>(o, 0, m, sum, int64_t(t.q0 + token) * Hq + head, h, out, lse, part);
}

// Joins the splits of the rows of sequences (tokens [cu_q[0], cu_q[batch])), in order: a
// wave per row, each lane D / 64 dimensions.
template <int D, int DT>
__global__ __launch_bounds__(kPThreads) void prefill_combine_kernel(const float* __restrict__ part, int splits, int64_t rows,
                                                                    int Hq, const int32_t* __restrict__ cu_q, int batch,
                                                                    void* __restrict__ out, float* __restrict__ lse) {
  constexpr int E = D / 64;
  const int64_t row = int64_t(blockIdx.x) * kPWaves + threadIdx.x / kWave;
  if (row >= rows || row < int64_t(cu_q[0]) * Hq || row >= int64_t(cu_q[batch]) * Hq) return;
  const int lane = lane_id();
  const float* p = part + row * splits * (D + 2);
  float M = -INFINITY;
  for (int s = 0; s < splits; ++s) M = fmaxf(M, p[s * (D + 2)]);
  float l = 0.f, acc[E] = {};
  if (M != -INFINITY) {
    for (int s = 0; s < splits; ++s) {
      const float* ps = p + s * (D + 2);
      const float c = __builtin_amdgcn_exp2f(ps[0] - M);
      if (ps[0] == -INFINITY) continue;
      l = fmaf(ps[1], c, l);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(ps[2 + E * lane + e], c, acc[e]);
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int64_t at = row * D + E * lane + e;
    if constexpr (DT == RBQ_BF16)
      static_cast<__bf16*>(out)[at] = __bf16(acc[e] * inv);
    else
      static_cast<float*>(out)[at] = acc[e] * inv;
  }
  if (lse && lane == 0) lse[row] = l > 0.f ? (M + log2f(l)) * kLn2 : -INFINITY;
}
}  // namespace

rbq_status launch_prefill(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const PrefillArgs& a,
                          hipStream_t stream) {
  if (a.total_q == 0) return RBQ_OK;
  const PrefillPlan pl = prefill_plan(batch, heads_q, heads_kv, a.max_k, a.total_q, a.dtype);
  const float c = float(double(a.sm_scale) * 1.4426950408889634);
  float* part = pl.splits > 1 ? static_cast<float*>(a.ws) : nullptr;
  const dim3 grid(uint32_t(int64_t(pl.tiles) * heads_kv), pl.splits);
  const int64_t rows = int64_t(a.total_q) * heads_q;
  const dim3 cgrid(uint32_t((rows + kPWaves - 1) / kPWaves));
#define RBQ_PREFILL(KERNEL, T)                                                                                          \
  KERNEL<<<grid, kPThreads, 0, stream>>>(static_cast<const T*>(a.q), a.q_ld, static_cast<const T*>(a.K),                 \
                                         static_cast<const T*>(a.V), a.kv_ld, a.kv_head, a.kv_seq, a.kv_rows, a.cu_q,   \
                                         a.cu_k, batch, a.total_q, a.max_k, a.causal, c, static_cast<T*>(a.out), a.lse, \
                                         part, heads_q, heads_kv, pl.tiles, pl.kchunk)
#define RBQ_PREFILL_JOIN(D, DT)                                                                                    \
  if (part)                                                                                                        \
  prefill_combine_kernel<D, DT><<<cgrid, kPThreads, 0, stream>>>(part, pl.splits, rows, heads_q, a.cu_q, batch, a.out, \
                                                                 a.lse)
  if (a.dtype == RBQ_F32) {
    if (head_dim == 64) {
      RBQ_PREFILL(prefill_f32_kernel<64>, float);
      RBQ_PREFILL_JOIN(64, RBQ_F32);
    } else {
      RBQ_PREFILL(prefill_f32_kernel<128>, float);
      RBQ_PREFILL_JOIN(128, RBQ_F32);
    }
  } else if (head_dim == 64) {
    if (pl.rows > 128) RBQ_PREFILL((prefill_kernel<64, 2>), uint16_t);
    else RBQ_PREFILL((prefill_kernel<64, 1>), uint16_t);
    RBQ_PREFILL_JOIN(64, RBQ_BF16);
  } else {
    if (pl.rows > 128) RBQ_PREFILL((prefill_kernel<128, 2>), uint16_t);
    else RBQ_PREFILL((prefill_kernel<128, 1>), uint16_t);
    RBQ_PREFILL_JOIN(128, RBQ_BF16);
  }
#undef RBQ_PREFILL_JOIN
#undef RBQ_PREFILL
  return hipGetLastError() == hipSuccess ? RBQ_OK : RBQ_EDEVICE;
}

}  // namespace rbq
