// rbq_prefill_attention: softmax attention of prompts (or chunks of them over rows
// already cached), causal or full, grouped heads, packed sequences.
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(sm_scale (<q_i, k_j> - max_j)),
//   over the j < Lk of the query's sequence, for causal j <= i + Lk - Lq
//
// One pass over the keys with the running maximum and sum of the softmax.
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
  int split;     // of its keys
  int q0, nq;    // first token of the sequence on the packed axis, tokens
  int nk;        // keys
  int64_t k0;    // first row of the sequence's keys (packed), 0 otherwise
};

// One sequence's lengths, inside the buffers: keys inside [0, kv_rows) of the packed axis,
// or of the sequence's own rows.
struct Lengths {
  int q0, nq, k0, nk, tiles;
};
__device__ __forceinline__ Lengths lengths_of(int b, int G, int BM, int total_q, int max_k, int kv_rows, bool packed,
                                              const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_k) {
  Lengths s;
  const int ka = cu_k[b], kb = cu_k[b + 1];
  s.q0 = min(max(cu_q[b], 0), total_q);
  s.nq = max(min(max(cu_q[b + 1], 0), total_q) - s.q0, 0);
  s.k0 = packed ? min(max(ka, 0), kv_rows) : 0;
  s.nk = min(min(max(kb - ka, 0), max_k), kv_rows - s.k0);
  s.tiles = int((int64_t(s.nq) * G + BM - 1) / BM);
  return s;
}

// What block `id` of a KV head does. Query tiles (ceil(tokens * G / BM) a sequence) are
// ranked by their steps of kPKeys keys, the longest first: started last they would run on
// alone. The tiles of a causal sequence see more keys one after the other, so a bisection
// over the number of steps, each lane counting one sequence's tiles, finds the p'th. Of
// split keys, split y is taken by the tiles that have keys there, a number L_y that lane y
// counts, so the blocks are split 0 of L_0 tiles, split 1 of the first L_1, ...: those
// without work all come last. (Spread among the others, as a grid of tiles x splits has
// them, they leave whole shader engines idle, which take blocks in turn: 512 blocks of
// 256 fp32 keys with 512 empty ones between them 84 us, in this order 52.)
// More sequences than lanes: in the sequences' order, backwards, every split of a tile.
__device__ __forceinline__ TileId find_tile(int id, int tiles, int splits, int kchunk, int batch, int G, int BM,
                                            int total_q, int max_k, int kv_rows, bool packed, bool causal,
                                            const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_k) {
  const int lane = lane_id();
  TileId t{-1, 0, 0, 0, 0, 0, 0};
  auto found = [&](const Lengths& s, int b0, int l, int tile) {
    t.b = b0 + l;
    t.tile = tile;
    t.q0 = __builtin_amdgcn_readlane(s.q0, l);
    t.nq = __builtin_amdgcn_readlane(s.nq, l);
    t.nk = __builtin_amdgcn_readlane(s.nk, l);
    t.k0 = __builtin_amdgcn_readlane(s.k0, l);
  };
  auto prefix = [&](int v) {   // inclusive sum over the lanes
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int u = __shfl_up(v, o, kWave);
      v += lane >= o ? u : 0;
    }
    return v;
  };
  if (batch == 1 && splits == 1) {
    const Lengths s = lengths_of(0, G, BM, total_q, max_k, kv_rows, packed, cu_q, cu_k);
    if (id < s.tiles) found(s, 0, 0, s.tiles - 1 - id);
    return t;
  }
  if (batch <= kWave) {
    Lengths s = lengths_of(min(lane, batch - 1), G, BM, total_q, max_k, kv_rows, packed, cu_q, cu_k);
    if (lane >= batch) s.nq = s.tiles = 0;
    // this sequence's tiles of at least n steps: a causal tile's keys end at its last token's
    auto of = [&](int nq, int nk, int tiles_b, int n) {
      if (n <= 0) return tiles_b;
      if (!causal) return (nk + kPKeys - 1) / kPKeys >= n ? tiles_b : 0;
      const int64_t first = int64_t(n - 1) * kPKeys - (nk - nq);   // the token that its last token must reach
      return first >= nq ? 0 : tiles_b - (first > 0 ? int(first * G / BM) : 0);
    };
    auto count = [&](int n) { return of(s.nq, s.nk, s.tiles, n); };
    int p = id;
    if (splits > 1) {
      int live = 0;   // L_y of lane y
      for (int b = 0; b < batch; ++b)
        live += of(__builtin_amdgcn_readlane(s.nq, b), __builtin_amdgcn_readlane(s.nk, b),
                   __builtin_amdgcn_readlane(s.tiles, b), lane > 0 ? lane * (kchunk / kPKeys) + 1 : 0);
      if (lane >= splits) live = 0;
      const int inc = prefix(live);
      const unsigned long long at = __ballot(id >= inc - live && id < inc);
      if (at == 0ull) return t;
      t.split = __builtin_ctzll(at);
      p -= __builtin_amdgcn_readlane(inc - live, t.split);
    }
    if (p >= wave_sum_i32(s.tiles)) return t;
    int lo = 0, hi = (max_k + kPKeys - 1) / kPKeys + 1;   // more than p tiles have at least lo steps, no more than p hi
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (wave_sum_i32(count(mid)) > p) lo = mid;
      else hi = mid;
    }
    const int more = count(lo + 1), here = count(lo) - more, inc = prefix(here);
    const int r = p - wave_sum_i32(more);
    const int l = __builtin_ctzll(__ballot(r >= inc - here && r < inc) | (1ull << 63));
    found(s, 0, l, __builtin_amdgcn_readlane(s.tiles - more - here, l) + r - __builtin_amdgcn_readlane(inc - here, l));
    return t;
  }
  const int tile = tiles - 1 - id / splits;
  t.split = id % splits;
  int before = 0;
  for (int b0 = 0; b0 < batch; b0 += kWave) {
    const Lengths s = lengths_of(min(b0 + lane, batch - 1), G, BM, total_q, max_k, kv_rows, packed, cu_q, cu_k);
    const int mine = b0 + lane < batch ? s.tiles : 0, inc = before + prefix(mine);
    const unsigned long long at = __ballot(tile >= inc - mine && tile < inc);
    if (at != 0ull) {
      const int l = __builtin_ctzll(at);
      found(s, b0, l, tile - __builtin_amdgcn_readlane(inc - mine, l));
      return t;
    }
    before = __builtin_amdgcn_readlane(inc, kWave - 1);
  }
  return t;
}

// 16 bytes per lane from global memory straight into LDS (lane l's at lds + 16 l)
__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t r, char* lds, int off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (RBQ_LDS void*)lds, 16, off, 0, 0, 0);
}
// Waits for this wave's loads: before the barrier that publishes them to the block.
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The 16-byte chunk c of row r of a tile lies at chunk c ^ swizzle(r) of the row, so that the
// lanes served together (256 bytes a clock) touch every bank once: 16 rows' same chunk of K,
// 64 bytes of four rows that follow each other of V. Both depend on r mod 16 alone.
template <int D>
__device__ __forceinline__ int k_swizzle(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
template <int D>
__device__ __forceinline__ int v_swizzle(int r) { return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); }

// A lane's part of a finished row: dimensions 32 d + 8 g + 4 h .. +4. With one split
// the output itself, otherwise the split's state {m, l, acc}.
template <int D, int DT, int NQ>
__device__ __forceinline__ void store_row(const f32x16 (&o)[D / 32][NQ], int i, float m, float sum, int64_t row, int h,
                                          void* __restrict__ out, float* __restrict__ lse, float* __restrict__ part,
                                          int split, int splits, int none) {
  float* pr = part + (row * splits + split) * (D + 2);
  const float scale = part ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
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
  if (part) {
    *reinterpret_cast<f32x2*>(pr) = f32x2{sum == 0.f ? -INFINITY : sum == sum ? m : sum, sum};   // (a NaN is kept)
    // split 0 also writes the states of the splits from `none` on, which no block takes
    for (int k = none; split == 0 && k < splits; ++k) pr[int64_t(k) * (D + 2)] = -INFINITY;
  } else if (lse)
    lse[row] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
}

// bf16 rows. A wave holds 32 query rows as the columns of its products, so that a row's
// maximum and sum are over its own lane and the one 32 away:
//   S^T = K Q^T   v_mfma_f32_32x32x16_bf16, A = 32 keys, B = the queries (in registers);
//                 lane (row x, half h), register r: key 8 (r / 4) + 4 h + r % 4
//   O^T = V^T P^T A = 32 dimensions of V by transposing LDS reads, B = the probabilities
//                 straight from those registers (the order of the 16 keys of a product is
//                 free as long as both operands share it)
// A step takes 64 keys, staged by the block's four waves into double buffers in LDS, K a
// tile ahead of V: the products of the next step's logits run on the matrix cores while
// the softmax of this one runs on the vector units, and K's and V's LDS reads are hidden
// behind both. (32 keys at a time, with a maximum and a rescaling for each: 2000 tokens of
// 32 heads 58.9 us, now 55.0; 16001 2056 and 2004; 4000 of D = 64 98 and 91; 8 x 43..650
// 34.5 and 34.9, of D = 64 20.9 and 22.8.) Two blocks share a compute unit: with its 128
// accumulators for 64 rows a wave would read LDS half as often, but alone on its SIMD it
// waits (16001 tokens: 2772 us; 32 rows 2129). A step of a block takes 1.2 us alone on a
// compute unit and 1.5 beside another, chained by the softmax; in long prompts the power
// limit bounds it: 2.10 TFLOP in 2000 to 2150 us is 0.98 to 1.05 PFLOP/s at the clock that
// it leaves (1.8 of 2.4 GHz); the library's 8192^3 product, in the same state, makes 1.23
// PFLOP/s of its 1.70 on zeros.
template <int D>
__global__ __launch_bounds__(kPThreads, 2) void prefill_kernel(
    const uint16_t* __restrict__ q, int64_t q_ld, const uint16_t* __restrict__ K, const uint16_t* __restrict__ V,
    int64_t kv_ld, int64_t kv_head, int64_t kv_seq, int kv_rows, const int32_t* __restrict__ cu_q,
    const int32_t* __restrict__ cu_k, int batch, int total_q, int max_k, int causal, float scale_log2e,
    uint16_t* __restrict__ out, float* __restrict__ lse, float* __restrict__ part, int Hq, int Hkv, int tiles, int splits,
    int kchunk) {
  constexpr int BM = 32 * kPWaves, C = D / 8, KB = D / 16, DT = D / 32, RB = D * 2;   // chunks, k-blocks, dim tiles, bytes of a row
  __shared__ __attribute__((aligned(1024))) char ldsK[2][kPKeys * RB], ldsV[2][kPKeys * RB];
  __shared__ int odd;   // values were replaced (below)
  const int G = Hq / Hkv;
  const int hk = blockIdx.x % Hkv;
  const TileId t = find_tile(int(blockIdx.x) / Hkv, tiles, splits, kchunk, batch, G, BM, total_q, max_k, kv_rows, kv_seq == 0,
                             causal != 0, cu_q, cu_k);
  if (t.b < 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int x = lane & 31, h = lane >> 5;
  const int rows = t.nq * G;
  const int row0 = t.tile * BM;
  const int shift = t.nk - t.nq;                                   // query token i sees keys <= i + shift
  auto visible = [&](int token) { return causal ? min(max(token + shift + 1, 0), t.nk) : t.nk; };
  const int kend = visible((min(row0 + BM, rows) - 1) / G);         // keys that some row of the block sees
  const int wrow = row0 + wave * 32;
  const int kbeg = t.split * kchunk, kstop = min(kend, kbeg + kchunk);   // this block's keys
  const int wend = wrow < rows ? visible((min(wrow + 32, rows) - 1) / G) : 0;   // of the wave
  const int wmin = visible(min(wrow, rows - 1) / G);                // keys that every row of the wave sees

  // queries: B operand, lane (row x, half h) holds dimensions 16 kb + 8 h .. +8
  bf16x8 qf[KB];
  const int qrow = min(wrow + x, rows - 1), token = qrow / G, head = hk * G + (qrow - token * G), lim = visible(token);
  {
    const uint16_t* p = q + int64_t(t.q0 + token) * q_ld + head * D + 8 * h;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) qf[kb] = *reinterpret_cast<const bf16x8*>(p + 16 * kb);
  }

  const int64_t kvoff = (kv_seq == 0 ? t.k0 * kv_ld : int64_t(t.b) * kv_seq) + int64_t(hk) * kv_head;
  const uint16_t *Kb = K + kvoff, *Vb = V + kvoff;
  // staging: one instruction moves 1024 bytes, 1024 / RB rows
  constexpr int kRowsPer = 1024 / RB, kIssues = kPKeys / kRowsPer / kPWaves;
  const int srow = lane / C, spos = lane % C;
  auto stage = [&](const uint16_t* base, char* lds, int k0, bool v) {
    const int left = min(t.nk - k0, kPKeys);   // (the last rows again in place of those behind them)
    const __amdgpu_buffer_rsrc_t r = make_rsrc(base + k0 * kv_ld, uint32_t((left - 1) * kv_ld * 2 + RB));
#pragma unroll
    for (int i = 0; i < kIssues; ++i) {
      const int row = (wave * kIssues + i) * kRowsPer + srow;
      load_lds16(r, lds + (wave * kIssues + i) * 1024,
                 min(row, left - 1) * int(kv_ld * 2) + ((spos ^ (v ? v_swizzle<D>(row) : k_swizzle<D>(row))) * 16));
    }
  };
  // read addresses: K rows (lane: key x, chunk 2 kb + h), V columns by the transposing
  // read (16 lanes: 4 keys x 16 dimensions; lane i gives key i / 4, dimensions 4 (i % 4) .. +4)
  const int kbase = x * RB + ((h ^ k_swizzle<D>(x)) * 16);
  const int i16 = lane & 15, g16 = (lane >> 4) & 1;
  const int vbase = (4 * h + (i16 >> 2)) * RB + (((2 * g16 + ((i16 & 3) >> 1)) ^ v_swizzle<D>(i16 >> 2)) * 16) + (i16 & 1) * 8;

  f32x16 o[DT][1];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][0][r] = 0.f;

  auto logits = [&](f32x16& d, const char* tile) {   // of the 32 keys whose rows start at `tile`
#pragma unroll
    for (int r = 0; r < 16; ++r) d[r] = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const bf16x8 a = *reinterpret_cast<const bf16x8*>(tile + (kbase ^ (kb * 32)));
      d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[kb], d, 0, 0, 0);
    }
  };
  // the softmax of s (64 keys from k0) and its product with V, and the logits nx of the 64 keys after
  auto step = [&](f32x16 (&s)[2], f32x16 (&nx)[2], int k0, const char* next_k, const char* tile_v) {
    if (k0 + kPKeys > wmin) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = k0 + 32 * t + 8 * (r / 4) + 4 * h + r % 4 < lim ? s[t][r] : -INFINITY;
    }
    float mx[4] = {s[0][0], s[0][1], s[1][0], s[1][1]};
#pragma unroll
    for (int r = 2; r < 16; ++r)
#pragma unroll
      for (int t = 0; t < 2; ++t) mx[2 * t + (r & 1)] = fmaxf(mx[2 * t + (r & 1)], s[t][r]);
    float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale_log2e;
    // (Moving the reference only where the maximum passes it by a factor of 2^8 saves 2 %, but
    // the largest probability is then rounded to bf16 instead of being 1: 1.25 times the
    // plain form's error instead of 1.05.)
    if (__ballot(top > m)) {
      const float mn = fmaxf(m, top);
      const float corr = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][0][r] *= corr;
      m = mn;
    }
    const float mref = m == -INFINITY ? 0.f : m;
    bf16x8 p[4];
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      logits(nx[t], next_k + t * 32 * RB);
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        f32x8 e;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          e[r] = __builtin_amdgcn_exp2f(fmaf(s[t][8 * g + r], scale_log2e, -mref));
          sum[2 * t + (r & 1)] += e[r];
        }
        // (The probabilities are rounded to bf16, the sum is not: up to 2^-8 of each, which moves the
        // outputs by 0.0005 to 0.0015 of their norm, 0.0010 for 8 x 43..650 tokens, 0.0009 for 16001;
        // their own rounding to bf16 by 0.0016. In two parts the second product would be twice the work.)
        p[2 * t + g] = __builtin_convertvector(e, bf16x8);
      }
    }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const char* at = tile_v + g * 16 * RB + (vbase ^ (d * 64));
        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((RBQ_LDS s16x4*)at);
        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((RBQ_LDS s16x4*)(at + 8 * RB));
        const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        o[d][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p[g], o[d][0], 0, 0, 0);
      }
  };
  // A masked probability of 0 would carry an infinity or NaN of V to rows that do not see its
  // key: in tiles that some row sees in part they are replaced by 0 and noted; at the end each
  // row adds those of the keys that it sees (from kodd on).
  const int bmin = visible(row0 / G);
  const int kodd = bmin > kbeg ? kbeg + (bmin - kbeg) / kPKeys * kPKeys : kbeg;
  auto finite_tile = [&](char* tile) {   // the pieces that this lane has staged, before they are published
#pragma unroll
    for (int i = 0; i < kIssues; ++i) {
      u32x4* at = reinterpret_cast<u32x4*>(tile + (wave * kIssues + i) * 1024 + lane * 16);
      u32x4 w = *at;
      uint32_t f = 0u;
#pragma unroll
      for (int e = 0; e < 4; ++e) f |= (w[e] & 0x7F807F80u) + 0x00800080u;   // an exponent of ones carries
      if (f & 0x80008000u) {
        odd = 1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if ((w[e] & 0x7F80u) == 0x7F80u) w[e] &= 0xFFFF0000u;
          if ((w[e] & 0x7F800000u) == 0x7F800000u) w[e] &= 0xFFFFu;
        }
        *at = w;
      }
    }
  };

  // Tile i of K and of V holds the keys kbeg + 64 i .. +64, in buffer i % 2; step i reads tile i
  // of V and tile i + 1 of K. Logits of keys behind the last are formed from whatever the tile
  // holds and masked.
  f32x16 sa[2], sb[2];
  if (kbeg < kstop) {
    stage(Kb, ldsK[0], kbeg, false);
    stage(Vb, ldsV[0], kbeg, true);
    if (kbeg + kPKeys < kstop) stage(Kb, ldsK[1], kbeg + kPKeys, false);
    if (threadIdx.x == 0) odd = 0;
    wait_lds();
    __syncthreads();
    logits(sa[0], ldsK[0]);
    logits(sa[1], &ldsK[0][32 * RB]);
  }
  const int wstop = min(wend, kstop);
  auto publish = [&](int k0, int buf) {   // tile i of V and i + 1 of K have arrived; the ones after are requested
    wait_lds();
    if (k0 >= kodd) finite_tile(ldsV[buf]);
    __syncthreads();
    if (k0 + kPKeys < kstop) stage(Vb, ldsV[buf ^ 1], k0 + kPKeys, true);
    if (k0 + 2 * kPKeys < kstop) stage(Kb, ldsK[buf], k0 + 2 * kPKeys, false);
  };
  for (int k0 = kbeg; k0 < kstop; k0 += 2 * kPKeys) {
    publish(k0, 0);
    if (k0 < wstop) step(sa, sb, k0, ldsK[1], ldsV[0]);
    if (k0 + kPKeys >= kstop) break;
    publish(k0 + kPKeys, 1);
    if (k0 + kPKeys < wstop) step(sb, sa, k0 + kPKeys, ldsK[0], ldsV[1]);
  }

  if (kbeg < kstop && odd) {
#pragma unroll 1
    for (int key = kodd; key < min(lim, kstop); ++key) {
#pragma unroll
      for (int c = 0; c < 4 * DT; ++c) {   // the lane's dimensions 8 c + 4 h .. +4
        const u32x2 w = *reinterpret_cast<const u32x2*>(Vb + key * kv_ld + 8 * c + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = __uint_as_float((w[e / 2] >> (16 * (e % 2))) << 16);
          o[c / 4][0][4 * (c % 4) + e] += fabsf(v) < INFINITY ? 0.f : v;
        }
      }
    }
  }
  const float sum = l + __shfl_xor(l, 32, kWave);
  if (wrow + x < rows)
    store_row<D, RBQ_BF16>(o, 0, m, sum, int64_t(t.q0 + token) * Hq + head, h, out, lse, part, t.split, splits,
                           batch <= kWave ? (kend + kchunk - 1) / kchunk + (kend == 0) : splits);
}

// fp32 rows: the same on v_mfma_f32_32x32x2_f32, products and probabilities in fp32.
// Lane half h of the logits product takes dimensions h D / 2 .. +D / 2 (the order of the
// dimensions is free as long as K and the queries share it), so both read four at once;
// register r of the result is key 8 (r / 4) + 4 h + r % 4, which is row k = h of step r of
// the second product. Bound by the matrix cores (500 tokens of 8 heads of 64 over 6000 rows:
// 56 us and 6 of the join, the cores busy for 0.64 of the time that blocks run, the rest
// uneven numbers of blocks per compute unit).
constexpr int kFKeys = 32;
template <int D>
__global__ __launch_bounds__(kPThreads, 2) void prefill_f32_kernel(
    const float* __restrict__ q, int64_t q_ld, const float* __restrict__ K, const float* __restrict__ V, int64_t kv_ld,
    int64_t kv_head, int64_t kv_seq, int kv_rows, const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_k,
    int batch, int total_q, int max_k, int causal, float scale_log2e, float* __restrict__ out, float* __restrict__ lse,
    float* __restrict__ part, int Hq, int Hkv, int tiles, int splits, int kchunk) {
  constexpr int BM = 32 * kPWaves, DT = D / 32, LD = D + 4;   // (padded rows: four consecutive keys in other banks)
  constexpr int kPieces = kFKeys * D / 4 / kPThreads;        // 16-byte pieces per thread and tensor
  __shared__ __attribute__((aligned(16))) float ldsK[kFKeys][LD], ldsV[kFKeys][LD];
  const int G = Hq / Hkv;
  const int hk = blockIdx.x % Hkv;
  const TileId t = find_tile(int(blockIdx.x) / Hkv, tiles, splits, kchunk, batch, G, BM, total_q, max_k, kv_rows, kv_seq == 0,
                             causal != 0, cu_q, cu_k);
  if (t.b < 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int x = lane & 31, h = lane >> 5;
  const int rows = t.nq * G, row0 = t.tile * BM, shift = t.nk - t.nq;
  auto visible = [&](int token) { return causal ? min(max(token + shift + 1, 0), t.nk) : t.nk; };
  const int kend = visible((min(row0 + BM, rows) - 1) / G);
  const int kbeg = t.split * kchunk, kstop = min(kend, kbeg + kchunk);
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
  // (infinities and NaN of V as in the bf16 kernel)
  const int bmin = visible(row0 / G);
  const int kodd = bmin > kbeg ? kbeg + (bmin - kbeg) / kFKeys * kFKeys : kbeg;
  bool odd = false;
  if (kbeg < kstop) fetch(kbeg);
  for (int k0 = kbeg; k0 < kstop; k0 += kFKeys) {
    if (k0 >= kodd) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const bool f = fabsf(vreg[i][c]) < INFINITY;
          odd |= !f;
          vreg[i][c] = f ? vreg[i][c] : 0.f;
        }
    }
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
    // LDS reads in groups of four, each requested before the last one's products (the fences
    // keep them there)
    f32x4 ka[2][4];
    auto read_k = [&](int g) {
#pragma unroll
      for (int i = 0; i < 4; ++i) ka[g & 1][i] = *reinterpret_cast<const f32x4*>(&ldsK[x][h * (D / 2) + 4 * (4 * g + i)]);
    };
    read_k(0);
#pragma unroll
    for (int g = 0; g < D / 32; ++g) {
      if (g + 1 < D / 32) read_k(g + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(ka[g & 1][i][e], qf[4 * g + i][e], s, 0, 0, 0);
    }
    float va[2][4][DT];
    auto read_v = [&](int g) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 0; d < DT; ++d) va[g & 1][i][d] = ldsV[8 * g + 4 * h + i][32 * d + x];
    };
    read_v(0);
    __builtin_amdgcn_sched_barrier(0);
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
    for (int g = 0; g < 4; ++g) {
      if (g < 3) read_v(g + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 0; d < DT; ++d)
          o[d][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(va[g & 1][i][d], s[4 * g + i], o[d][0], 0, 0, 0);
    }
  }
  if (__syncthreads_or(odd)) {
#pragma unroll 1
    for (int key = kodd; key < min(lim, kstop); ++key) {
#pragma unroll
      for (int c = 0; c < 4 * DT; ++c) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(V + kvoff + key * kv_ld + 8 * c + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[c / 4][0][4 * (c % 4) + e] += fabsf(v[e]) < INFINITY ? 0.f : v[e];
      }
    }
  }
  const float sum = l + __shfl_xor(l, 32, kWave);
  if (wrow + x < rows)
    store_row<D, RBQ_F32>(o, 0, m, sum, int64_t(t.q0 + token) * Hq + head, h, out, lse, part, t.split, splits,
                      batch <= kWave ? (kend + kchunk - 1) / kchunk + (kend == 0) : splits);
}

// Joins the splits of the rows of sequences (tokens [cu_q[0], cu_q[batch])): a wave per
// row; lane s weighs split s, then each lane adds up D / 64 dimensions in the splits' order,
// up to the last one with keys, BATCH at once.
template <int D, int DT, int BATCH>
__global__ __launch_bounds__(kPThreads) void prefill_combine_kernel(const float* __restrict__ part, int splits, int64_t rows,
                                                                    int Hq, const int32_t* __restrict__ cu_q, int batch,
                                                                    void* __restrict__ out, float* __restrict__ lse) {
  constexpr int E = D / 64;
  typedef float vec __attribute__((ext_vector_type(E)));
  const int64_t row = int64_t(blockIdx.x) * kPWaves + threadIdx.x / kWave;
  if (row >= rows || row < int64_t(cu_q[0]) * Hq || row >= int64_t(cu_q[batch]) * Hq) return;
  const int lane = lane_id();
  const float* p = part + row * splits * (D + 2);
  const f32x2 ml = *reinterpret_cast<const f32x2*>(p + min(lane, splits - 1) * (D + 2));
  vec v[BATCH];
  auto load = [&](int s0) {
#pragma unroll
    for (int k = 0; k < BATCH; ++k)
      v[k] = *reinterpret_cast<const vec*>(p + min(s0 + k, splits - 1) * (D + 2) + 2 + E * lane);
  };
  load(0);
  const float ms = lane < splits ? ml.x : -INFINITY;
  const float M = wave_max(ms);
  const float c = ms == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms - M);
  const float l = wave_reduce(c == 0.f ? 0.f : ml.y * c, [](float a, float b) { return a + b; });
  const int live = kWave - __builtin_clzll(__ballot(c != 0.f) | 1ull);
  vec acc = {};
  for (int s0 = 0; s0 < live; s0 += BATCH) {
    if (s0 > 0) load(s0);
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const float ck = __uint_as_float(uint32_t(__builtin_amdgcn_readlane(int(__float_as_uint(c)), min(s0 + k, kWave - 1))));
      if (s0 + k < splits && ck != 0.f) {   // (a split without keys has written nothing else)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(v[k][e], ck, acc[e]);
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int64_t at = row * D + E * lane + e;
    if constexpr (DT == RBQ_BF16)
      static_cast<__bf16*>(out)[at] = __bf16(acc[e] * inv);
    else
      static_cast<float*>(out)[at] = acc[e] * inv;
  }
  if (lse && lane == 0) lse[row] = l == 0.f ? -INFINITY : (M + log2f(l)) * kLn2;
}
}  // namespace

rbq_status launch_prefill(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const PrefillArgs& a,
                          hipStream_t stream) {
  if (a.total_q == 0) return RBQ_OK;
  const PrefillPlan pl = prefill_plan(batch, heads_q, heads_kv, head_dim, a.max_k, a.total_q, a.dtype);
  const float c = float(double(a.sm_scale) * 1.4426950408889634);
  float* part = pl.splits > 1 ? static_cast<float*>(a.ws) : nullptr;
  const dim3 grid(uint32_t(int64_t(pl.tiles) * heads_kv * pl.splits));
  const int64_t rows = int64_t(a.total_q) * heads_q;
  const dim3 cgrid(uint32_t((rows + kPWaves - 1) / kPWaves));
#define RBQ_PREFILL(KERNEL, T)                                                                                          \
  KERNEL<<<grid, kPThreads, 0, stream>>>(static_cast<const T*>(a.q), a.q_ld, static_cast<const T*>(a.K),                 \
                                         static_cast<const T*>(a.V), a.kv_ld, a.kv_head, a.kv_seq, a.kv_rows, a.cu_q,   \
                                         a.cu_k, batch, a.total_q, a.max_k, a.causal, c, static_cast<T*>(a.out), a.lse, \
                                         part, heads_q, heads_kv, pl.tiles, pl.splits, pl.kchunk)
#define RBQ_PREFILL_JOIN(D, DT)                                                                                    \
  if (part && pl.splits <= 4)                                                                                      \
    prefill_combine_kernel<D, DT, 4><<<cgrid, kPThreads, 0, stream>>>(part, pl.splits, rows, heads_q, a.cu_q, batch, \
                                                                      a.out, a.lse);                               \
  else if (part)                                                                                                   \
    prefill_combine_kernel<D, DT, 8><<<cgrid, kPThreads, 0, stream>>>(part, pl.splits, rows, heads_q, a.cu_q, batch, \
                                                                      a.out, a.lse)
  if (a.dtype == RBQ_F32) {
    if (head_dim == 64) {
      RBQ_PREFILL(prefill_f32_kernel<64>, float);
      RBQ_PREFILL_JOIN(64, RBQ_F32);
    } else {
      RBQ_PREFILL(prefill_f32_kernel<128>, float);
      RBQ_PREFILL_JOIN(128, RBQ_F32);
    }
  } else if (head_dim == 64) {
    RBQ_PREFILL(prefill_kernel<64>, uint16_t);
    RBQ_PREFILL_JOIN(64, RBQ_BF16);
  } else {
    RBQ_PREFILL(prefill_kernel<128>, uint16_t);
    RBQ_PREFILL_JOIN(128, RBQ_BF16);
  }
#undef RBQ_PREFILL_JOIN
#undef RBQ_PREFILL
  return hipGetLastError() == hipSuccess ? RBQ_OK : RBQ_EDEVICE;
}

}  // namespace rbq
