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
#include <cmath>
#include <type_traits>

#include "decode_dev.h"

namespace rbq {
namespace {

constexpr int kScaleCap = kKv8DenseChunk / kMinKv8Block;   // scale pairs of a split
constexpr float kLn2 = 0.69314718055994531f;
constexpr int kPad8 = 32;                                // a row list ends on a whole group
constexpr float kBf16Over = 0x1.FFp127f;                 // rounded to bf16, an infinity (from here on)

constexpr int elem_bytes(int src) { return src == RBQ_F32 ? 4 : src == RBQ_BF16 ? 2 : 1; }
constexpr int row_tiles(int src) { return elem_bytes(src) == 1 ? 2 : 1; }   // tiles of 16 rows per group
constexpr int row_parts(int src) { return src == RBQ_F32 ? 3 : 1; }         // bf16 parts of a value

// One group's rows as one lane (x, j) sees them, raw: row x of each tile (dimensions
// 64 i + 16 j .. +16) and dimensions (D / 16) x .. +D / 16 of rows 4j .. 4j+3.
template <int SRC, int D>
struct RowRegs {
  static constexpr int kKw = D * elem_bytes(SRC) / 16, kVw = D * elem_bytes(SRC) / 64;
  uint32_t k[row_tiles(SRC)][kKw];
  uint32_t v[row_tiles(SRC)][4][kVw];
};

template <int WORDS, int CP>
__device__ __forceinline__ void load_words(uint32_t* d, __amdgpu_buffer_rsrc_t r, int off) {
  if constexpr (WORDS == 1) {
    d[0] = __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, CP);
  } else if constexpr (WORDS == 2) {
    const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, CP));
    d[0] = v.x;
    d[1] = v.y;
  } else {
#pragma unroll
    for (int w = 0; w < WORDS / 4; ++w) {
      const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off + 16 * w, 0, CP));
#pragma unroll
      for (int i = 0; i < 4; ++i) d[4 * w + i] = v[i];
    }
  }
}

// two codes (bytes 2 HI, 2 HI + 1 of w) as a pair of bf16
template <int SRC, bool HI>
__device__ __forceinline__ uint32_t codes_bf16(uint32_t w) {
  if constexpr (SRC == RBQ_E4M3) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, HI));
  } else {
    typedef float f32x2v __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const f32x2v v = {float(int8_t(w >> (HI ? 16 : 0))), float(int8_t(w >> (HI ? 24 : 8)))};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  }
}

// a lane's 8 dimensions (group kb of the logits product) of a row as an operand, part `part`
template <int SRC>
__device__ __forceinline__ bf16x8 k_operand(const uint32_t* k, int kb, int part) {
  const uint32_t* w = k + (kb / 2) * 4 * elem_bytes(SRC) + (kb % 2) * 2 * elem_bytes(SRC);
  if constexpr (SRC == RBQ_BF16) {
    return __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
  } else if constexpr (SRC == RBQ_F32) {
    f32x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = __uint_as_float(w[i]);
    bf16x8 p = __builtin_convertvector(r, bf16x8);
#pragma unroll
    for (int t = 0; t < part; ++t) {
      r -= __builtin_convertvector(p, f32x8);
      p = __builtin_convertvector(r, bf16x8);
    }
    return p;
  } else {
    return __builtin_bit_cast(bf16x8, u32x4{codes_bf16<SRC, false>(w[0]), codes_bf16<SRC, true>(w[0]),
                                            codes_bf16<SRC, false>(w[1]), codes_bf16<SRC, true>(w[1])});
  }
}

// column c (of the lane's D / 16) of the lane's four rows as two pairs of bf16, part `part`
template <int SRC, int VW>
__device__ __forceinline__ u32x2 v_column(const uint32_t (*v)[VW], int c, int part) {
  if constexpr (SRC == RBQ_BF16) {
    const uint32_t sel = c % 2 ? 0x07060302u : 0x05040100u;
    return u32x2{__builtin_amdgcn_perm(v[1][c / 2], v[0][c / 2], sel),
                 __builtin_amdgcn_perm(v[3][c / 2], v[2][c / 2], sel)};
  } else if constexpr (SRC == RBQ_F32) {
    f32x4 r = {__uint_as_float(v[0][c]), __uint_as_float(v[1][c]), __uint_as_float(v[2][c]), __uint_as_float(v[3][c])};
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 p = __builtin_convertvector(r, bf16x4);
#pragma unroll
    for (int t = 0; t < part; ++t) {
      r -= __builtin_convertvector(p, f32x4);
      p = __builtin_convertvector(r, bf16x4);
    }
    return __builtin_bit_cast(u32x2, p);
  } else if constexpr (SRC == RBQ_E4M3) {
    const uint32_t sel = (c % 4) < 2 ? 0x05010400u : 0x07030602u;   // {r0.c, r1.c, r0.c+1, r1.c+1} of an even c
    const uint32_t a = __builtin_amdgcn_perm(v[1][c / 4], v[0][c / 4], sel);
    const uint32_t b = __builtin_amdgcn_perm(v[3][c / 4], v[2][c / 4], sel);
    return c % 2 ? u32x2{codes_bf16<SRC, true>(a), codes_bf16<SRC, true>(b)}
                 : u32x2{codes_bf16<SRC, false>(a), codes_bf16<SRC, false>(b)};
  } else {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    const int sh = 8 * (c % 4);
    const f32x4 r = {float(int8_t(v[0][c / 4] >> sh)), float(int8_t(v[1][c / 4] >> sh)), float(int8_t(v[2][c / 4] >> sh)),
                     float(int8_t(v[3][c / 4] >> sh))};
    return __builtin_bit_cast(u32x2, __builtin_convertvector(r, bf16x4));
  }
}

// What a block keeps in LDS for its waves.
template <bool SPARSE, int G, int D>
struct Shared {
  static_assert(kScaleCap <= kDThreads, "one scale pair per thread");
  static constexpr bool kPackedQ = kQParts * G <= 16;
  static constexpr int kQOps = kPackedQ ? 1 : kQParts;
  u32x4 qB[D / 32][kQOps][kWave];   // B operands of the logits product
  f32x2 scale[kScaleCap];           // {ks, vs} of the split's token blocks
  uint32_t bm[SPARSE ? G : 1][kBmWords];
  __attribute__((aligned(16))) int32_t lst[SPARSE ? kListCap : 4];
  __attribute__((aligned(16))) uint16_t hmask[SPARSE ? kListCap : 8];
  int rng_lo[G], rng_hi[G];
  float sm[kDWaves][G], sl[kDWaves][G];
  __attribute__((aligned(16))) float sacc[kDWaves][G][D];
};

// One wave's online softmax over its groups of the block's U rows: row c0 + e of the
// buffers, or lst[e]. m: head x's running maximum (log2 domain, uniform over j), lsum:
// this lane's part of its sum; acc[c] lane (x, j), register i: head 4j + i, dimension
// (D / 16) x + c. begin() requests the first group, so that a block whose rows follow
// each other has them on the way while it stages its queries.
template <int SRC, bool LIST, int G, int D, int CP, class S>
struct Rows {
  static constexpr int NT = row_tiles(SRC), kRows = 16 * NT, EB = elem_bytes(SRC), KB = D / 32, NP = row_parts(SRC);
  static constexpr bool kCodes = EB == 1;
  // One group's registers are reused for the next: its K rows are requested as soon
  // as the logits are done, its V rows as soon as the values are. (fp32 rows, four
  // times the registers: each half is requested when its turn comes.)
  static constexpr bool kAhead = SRC != RBQ_F32;
  using Regs = RowRegs<SRC, D>;
  S& sh;
  const __amdgpu_buffer_rsrc_t Kr, Vr;
  const int c0, U, bshift, in_block, wave, x, j, ngroups;   // in_block: place of row c0 in its token block
  Regs cur;
  uint32_t mk;                // bit 4 t + i: row 4j + i of tile t is valid and taken by head x
  f32x2 sc[LIST ? NT : 1][4];   // its scales {ks, vs} (listed 8-bit rows)

  __device__ __forceinline__ Rows(S& s, __amdgpu_buffer_rsrc_t kr, __amdgpu_buffer_rsrc_t vr, int first, int rows, int shift)
      : sh(s), Kr(kr), Vr(vr), c0(first), U(rows), bshift(shift), in_block(first & ((1 << shift) - 1)),
        wave(threadIdx.x / kWave), x(lane_id() & 15), j(lane_id() >> 4), ngroups((rows + kRows - 1) / kRows) {}

  __device__ __forceinline__ int row_of(int grp, int e) const { return c0 + (e < U ? e : grp * kRows); }
  __device__ __forceinline__ void load_k(int grp, bool skip) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int e = grp * kRows + 16 * t + x;
      int row;
      if constexpr (LIST) row = sh.lst[e];
      else row = row_of(grp, e);
      const int off = skip ? kSkipOffset : row * (D * EB) + 16 * EB * j;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) load_words<4 * EB, CP>(&cur.k[t][4 * EB * i], Kr, off + 64 * EB * i);
    }
  }
  __device__ __forceinline__ void load_v(int grp, bool skip) {
    mk = 0u;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int e0 = grp * kRows + 16 * t + 4 * j;   // this lane's four entries
      i32x4 row;
      if constexpr (LIST) {
        row = *reinterpret_cast<const i32x4*>(sh.lst + e0);
        const u32x2 hm = *reinterpret_cast<const u32x2*>(sh.hmask + e0);
        const uint32_t a = (hm.x >> x) & 0x10001u, b = (hm.y >> x) & 0x10001u;
        mk |= ((a | (a >> 15) | (b << 2) | (b >> 13)) & 15u) << (4 * t);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          row[i] = row_of(grp, e0 + i);
          mk |= uint32_t(e0 + i < U && x < G) << (4 * t + i);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int off = skip ? kSkipOffset : row[i] * (D * EB) + (D * EB / 16) * x;
        load_words<Regs::kVw, CP>(cur.v[t][i], Vr, off);
        if constexpr (LIST && kCodes) sc[t][i] = sh.scale[(in_block + row[i] - c0) >> bshift];
      }
    }
  }
  __device__ __forceinline__ void begin() {
    if (kAhead && wave < ngroups) {
      load_k(wave, false);
      load_v(wave, false);
    }
  }

  __device__ __forceinline__ void run(float& m, float& lsum, f32x4 (&acc)[D / 16]) {
    constexpr int kQOps = S::kQOps;
    int grp = wave;
    while (grp < ngroups) {
      const int nxt = grp + kDWaves;
      const bool last = nxt >= ngroups;
      if constexpr (!kAhead) load_k(grp, false);
      // (an opaque offset: the query operands are re-read from LDS every group, in
      // registers they would cost waves per SIMD)
      int qoff = lane_id();
      asm volatile("" : "+v"(qoff));
      const u32x4* qp = &sh.qB[0][0][0] + qoff;
      f32x2 ts[NT];   // scales of rows that follow each other: 16 from a multiple of 16 are in one token block
      if constexpr (kCodes && !LIST) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int e = grp * kRows + 16 * t;
          ts[t] = sh.scale[(in_block + (e < U ? e : 0)) >> bshift];
        }
      }
      f32x4 s[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          // (kept in this order: moved up, the operands of every group would be held at once)
          __builtin_amdgcn_sched_barrier(0);
          bf16x8 a[NT];
#pragma unroll
          for (int t = 0; t < NT; ++t) a[t] = k_operand<SRC>(cur.k[t], kb, p);
#pragma unroll
          for (int op = 0; op < kQOps; ++op) {
            const bf16x8 b = __builtin_bit_cast(bf16x8, qp[(kb * kQOps + op) * kWave]);
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], b, s[t], 0, 0, 0);
          }
        }
      }
      if constexpr (kAhead) load_k(last ? grp : nxt, last);
      else load_v(grp, false);
      // columns h + G and h + 2G hold the mid and lo parts of head h's logits (through
      // opaque copies: hipcc 7.2 reads one element's register for all four otherwise)
      float lg[NT][4];
      float tmax = -INFINITY;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float sv = s[t][i];
          if constexpr (S::kPackedQ) {
            asm volatile("" : "+v"(sv));
            const int v = __builtin_bit_cast(int, sv);
            const float mid = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, v, 0x100 + G, 0xF, 0xF, false));
            const float lo = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, v, 0x100 + 2 * G, 0xF, 0xF, false));
            sv = (sv + mid) + lo;
          }
          if constexpr (kCodes) sv *= LIST ? sc[LIST ? t : 0][i].x : ts[t].x;
          else sv = fmaf(sv, 0.f, sv);   // (an infinite key's, whatever the signs of the query's parts: NaN)
          lg[t][i] = ((mk >> (4 * t + i)) & 1u) ? sv : -INFINITY;
          tmax = fmaxf(tmax, lg[t][i]);
        }
      }
      tmax = fmaxf(tmax, __shfl_xor(tmax, 16, kWave));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32, kWave));
      const float mn = fmaxf(m, tmax);
      const float mref = mn == -INFINITY ? 0.f : mn;   // (no row yet: every exponential below is that of -inf)
      const float corr = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mref);
      float w[NT * 4], sum = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f(lg[t][i] - mref);
          sum += p;
          w[4 * t + i] = kCodes ? p * (LIST ? sc[LIST ? t : 0][i].y : ts[t].y) : p;
        }
      }
      lsum = fmaf(lsum, corr, sum);
      const bool moved = mn != m;
      m = mn;
      if (__ballot(moved)) {
        float cr[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) cr[i] = __shfl(corr, 4 * j + i, kWave);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[c][i] *= cr[i];
        }
      }
      // the weighted probabilities in three parts: A operands (row = head x; k = rows 4j .. 4j+3
      // of both tiles, or, of one tile, the same rows in two parts)
      bf16x8 pa[3];
      if constexpr (NT == 2) {
        f32x8 wv;
#pragma unroll
        for (int i = 0; i < 8; ++i) wv[i] = w[i];
        split3(wv, pa);
      } else {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        f32x4 r = {w[0], w[1], w[2], w[3]};
        bf16x4 p3[3];
#pragma unroll
        for (int t = 0; t < 3; ++t) {
          p3[t] = __builtin_convertvector(r, bf16x4);
          r -= __builtin_convertvector(p3[t], f32x4);
        }
        const bf16x4 zero = __builtin_bit_cast(bf16x4, u32x2{0u, 0u});
        pa[0] = __builtin_shufflevector(p3[0], p3[1], 0, 1, 2, 3, 4, 5, 6, 7);
        pa[1] = __builtin_shufflevector(p3[2], zero, 0, 1, 2, 3, 4, 5, 6, 7);
      }
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        if (c % 2 == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const u32x2 v0 = v_column<SRC>(cur.v[0], c, p);
          const u32x2 v1 = NT == 2 ? v_column<SRC>(cur.v[NT - 1], c, p) : v0;
          const bf16x8 bv = __builtin_bit_cast(bf16x8, u32x4{v0.x, v0.y, v1.x, v1.y});
#pragma unroll
          for (int t = 0; t < (NT == 2 ? 3 : 2); ++t)
            acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa[t], bv, acc[c], 0, 0, 0);
        }
      }
      if constexpr (kAhead) load_v(last ? grp : nxt, last);
      grp = nxt;
    }
  }
};

// An infinity in a value of the window meets the parts of a probability, of either sign, and
// the zeros of the padding: NaN. Where a sum has come out so, it is the sum of the infinities
// and NaN of its dimension, over the window rows [f0, f1) at V that the block has taken.
template <int LOC, int D>
__device__ __forceinline__ void infinite_values(const char* __restrict__ V, int f0, int f1, f32x4 (&acc)[D / 16]) {
  float t = 0.f;
#pragma unroll
  for (int c = 0; c < D / 16; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) t = fmaf(acc[c][i], 0.f, t);
  if (!__ballot(t != t)) return;
  float odd[D / 16];
#pragma unroll
  for (int c = 0; c < D / 16; ++c) odd[c] = 0.f;
  const int first = D / 16 * (lane_id() & 15);   // the lane's dimensions
#pragma unroll 1
  for (int r = f0; r < f1; ++r) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      float v;
      if constexpr (LOC == RBQ_F32) v = reinterpret_cast<const float*>(V)[r * D + first + c];
      else v = __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(V)[r * D + first + c]) << 16);
      odd[c] += fabsf(v) < kBf16Over ? 0.f : v == v ? copysignf(INFINITY, v) : v;
    }
  }
#pragma unroll
  for (int c = 0; c < D / 16; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[c][i] = fabsf(acc[c][i]) < INFINITY || odd[c] == 0.f ? acc[c][i] : odd[c];
}

// A block's sequence, KV head and place s among its group's blocks: idx of them over
// the sequence's nb cached rows, then win over its wb window rows.
struct BlockId {
  int b, hk, s, nb, wb, idx, win;
};

// Block p of a ragged batch: sequence after sequence, each with the blocks that its own
// lengths call for (one where it has no rows), so that the blocks that follow each other
// are those of one sequence as in a uniform call, and the grid's unused rest comes last.
// (One row of blocks per split, in which short sequences leave gaps: 16 sequences of 2K
// to 32K rows, 32 / 8 heads: 117 us; this order 107.) ordered: densest sequences first (see
// sequence_of_rank), batch <= 64. b = -1: none.
template <bool SPARSE>
__device__ __forceinline__ BlockId ragged_block(int p, int ordered, int batch, int n, int w, int chunk, int Hq, int Hkv,
                                                const int32_t* __restrict__ sel_count, const int32_t* __restrict__ seq_n,
                                                const int32_t* __restrict__ seq_w) {
  const int lane = lane_id();
  BlockId id{-1, 0, 0, 0, 0, 0, 0};
  int before = 0;
  for (int b0 = 0; b0 < batch; b0 += kWave) {
    const int b = min(b0 + lane, batch - 1);
    const int nb = seq_n ? min(max(seq_n[b], 0), n) : n, wb = seq_w ? min(max(seq_w[b], 0), w) : w;
    float dens = 0.f;
    if (SPARSE && ordered) dens = selected_share(b, nb, Hq, Hkv, sel_count);
    const int idx = (nb + chunk - 1) / chunk, win = (wb + kDecodeWinChunk - 1) / kDecodeWinChunk;
    const int blocks = b0 + lane < batch ? max(idx + win, 1) * Hkv : 0;
    int first = 0;   // blocks before this lane's sequence
    if (SPARSE && ordered) {
      for (int o = 0; o < batch; ++o) {
        const float d = __uint_as_float(uint32_t(__builtin_amdgcn_readlane(int(__float_as_uint(dens)), o)));
        first += d > dens || (d == dens && o < lane) ? __builtin_amdgcn_readlane(blocks, o) : 0;
      }
    } else {
      int inc = blocks;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int v = __shfl_up(inc, o, kWave);
        inc += lane >= o ? v : 0;
      }
      first = before + inc - blocks;
      before += __builtin_amdgcn_readlane(inc, kWave - 1);
    }
    const unsigned long long mine = __ballot(p >= first && p < first + blocks);
    if (mine != 0ull) {
      const int l = __builtin_ctzll(mine);
      id.b = b0 + l;
      id.nb = __builtin_amdgcn_readlane(nb, l);
      id.wb = __builtin_amdgcn_readlane(wb, l);
      id.idx = __builtin_amdgcn_readlane(idx, l);
      id.win = __builtin_amdgcn_readlane(win, l);
      const int e = p - __builtin_amdgcn_readlane(first, l), per = max(id.idx + id.win, 1);
      id.hk = e / per;
      id.s = e - id.hk * per;
      return id;
    }
  }
  return id;
}

// FMT: the rows' 8-bit format; LOC: the window's type (RBQ_BF16 or RBQ_F32)
template <int FMT, int LOC, bool SPARSE, int G, int D>
__global__ __launch_bounds__(kDThreads, G == 16 ? 2 : 4) void decode_kv8_kernel(
    const float* __restrict__ q, const char* __restrict__ K8, const char* __restrict__ V8,
    const float* __restrict__ k_scale, const float* __restrict__ v_scale, int bshift, int cap, int n,
    const int32_t* __restrict__ sel_idx, const int32_t* __restrict__ sel_count,
    const unsigned long long* __restrict__ sel_mask, int mask_words, const char* __restrict__ K_loc,
    const char* __restrict__ V_loc, int64_t loc_ld, int w, int chunk, int idx_splits, int total_splits, int fold_s0,
    float scale_log2e, float* __restrict__ part, int Hq, int Hkv, const int32_t* __restrict__ seq_n,
    const int32_t* __restrict__ seq_w, int ragged, int ordered) {
  using S = Shared<SPARSE, G, D>;
  __shared__ S sh;

  BlockId id{int(blockIdx.y), 0, int(blockIdx.x), n, w, idx_splits, total_splits - idx_splits};
  if (ragged) {
    id = ragged_block<SPARSE>(blockIdx.x, ordered, ragged, n, w, chunk, Hq, Hkv, sel_count, seq_n, seq_w);
    if (id.b < 0) return;
  } else {
    id.b = int(blockIdx.y) / Hkv;
    id.hk = int(blockIdx.y) - id.b * Hkv;
  }
  const int b = id.b, hk = id.hk, bh = b * Hkv + hk, nb = id.nb, wb = id.wb;
  const bool window = id.s >= id.idx;
  const int split = window ? idx_splits + id.s - id.idx : id.s;   // its place among the group's states
  const int row0 = b * Hq + hk * G;
  const int wave = threadIdx.x / kWave, lane = lane_id();
  const int x = lane & 15, j = lane >> 4;
  // what does not depend on the sequence's lengths is requested first
  static_assert(G * (D / 8) <= kDThreads, "one piece of the queries per thread");
  const bool stages = int(threadIdx.x) < G * (D / 8);
  const int qh = threadIdx.x / (D / 8), qch = threadIdx.x % (D / 8);
  f32x4 qa = {0.f, 0.f, 0.f, 0.f}, qb = qa;
  if (stages) {
    const f32x4* qp = reinterpret_cast<const f32x4*>(q + int64_t(row0 + qh) * D + 8 * qch);
    qa = qp[0];
    qb = qp[1];
  }
  MaskWords<G> mword{};
  if (SPARSE && !window)
    mword = load_mask_words<G>(sel_mask, mask_words, row0, split * chunk, min(n, (split + 1) * chunk));
  HeadCounts<G> hcount{};
  if constexpr (SPARSE) hcount = load_head_counts<G>(sel_count, row0);
  const int lim = window ? wb : nb;
  const int c0 = window ? (split - idx_splits) * kDecodeWinChunk : split * chunk;
  const int c1 = max(c0, min(lim, c0 + (window ? kDecodeWinChunk : chunk)));
  if (ragged && id.s == 0) {   // the group's first block also writes the empty states that follow the sequence's own
    const int none = total_splits - id.idx - id.win;
    for (int e = threadIdx.x; e < G * none; e += kDThreads) {
      const int g = e / none, k = e - g * none;
      const int slot = k < idx_splits - id.idx ? id.idx + k : idx_splits + id.win + k - (idx_splits - id.idx);
      part[(int64_t(row0 + g) * total_splits + slot) * (D + 2)] = -INFINITY;
    }
  }
  if (c1 == c0) {   // block-uniform: no rows (uniform calls: the one empty split; ragged: written above)
    if (!ragged && int(threadIdx.x) < G) part[(int64_t(row0 + threadIdx.x) * total_splits + split) * (D + 2)] = -INFINITY;
    return;
  }
  constexpr int kLocEl = elem_bytes(LOC);
  const int64_t locb = int64_t(bh) * loc_ld * (D * kLocEl);
  const char* Kb = window ? K_loc + locb : K8 + int64_t(bh) * cap * D;
  const char* Vb = window ? V_loc + locb : V8 + int64_t(bh) * cap * D;
  const uint32_t region = uint32_t(lim) * uint32_t(window ? D * kLocEl : D);   // < 2^31
  const __amdgpu_buffer_rsrc_t Kr = make_rsrc(Kb, region), Vr = make_rsrc(Vb, region);
  float m = -INFINITY, lsum = 0.f;
  f32x4 acc[D / 16];
#pragma unroll
  for (int c = 0; c < D / 16; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  // the split's scales
  const bool scales = !window && int(threadIdx.x) <= ((c1 - 1) >> bshift) - (c0 >> bshift);
  f32x2 own_scale = {0.f, 0.f};
  if (scales) {
    const int64_t s0 = int64_t(bh) * ((int64_t(cap) + (1 << bshift) - 1) >> bshift) + (c0 >> bshift) + threadIdx.x;
    own_scale = f32x2{k_scale[s0], v_scale[s0]};
  }

  // query operands, lane (column c, quarter jj) of group kb = dimensions
  // 64 (kb / 2) + 16 jj + 8 (kb % 2) .. +8. G <= 4: one operand per group, column
  // c = part * G + head; otherwise one per (group, part), column c = head.
  // (Columns without a head stay unwritten: masked, and no other column reads them.)
  auto stage = [&] {
    if (scales) sh.scale[threadIdx.x] = own_scale;
    if (!stages) return;
    const f32x8 qv = __builtin_shufflevector(qa, qb, 0, 1, 2, 3, 4, 5, 6, 7) * scale_log2e;
    bf16x8 parts[kQParts];
    split3(qv, parts);
    const int kb = 2 * (qch / 8) + qch % 2, jj = (qch % 8) / 2;
#pragma unroll
    for (int t = 0; t < kQParts; ++t)
      sh.qB[kb][S::kPackedQ ? 0 : t][16 * jj + (S::kPackedQ ? t * G + qh : qh)] = __builtin_bit_cast(u32x4, parts[t]);
  };

  // the rows' cache policy as in decode.hip: streaming where the gather is bound by bandwidth
  if (window) {
    Rows<LOC, false, G, D, 0, S> rows(sh, Kr, Vr, c0, c1 - c0, 0);
    rows.begin();
    stage();
    __syncthreads();
    rows.run(m, lsum, acc);
    infinite_values<LOC, D>(Vb, c0, c1, acc);
  } else if constexpr (SPARSE) {
    stage();
    const int U = build_union_list<G, kDThreads, true, kPad8, true>(sel_idx, sel_mask, mask_words, row0, n, c0, c1, 0, 0, sh.bm,
                                                              sh.lst, sh.hmask, sh.rng_lo, sh.rng_hi, mword, hcount);
    auto attend = [&](auto cp) {
      Rows<FMT, true, G, D, decltype(cp)::value, S> rows(sh, Kr, Vr, c0, U, bshift);
      rows.begin();
      rows.run(m, lsum, acc);
    };
    if (G <= 4 && int64_t(U) * kStreamDenDen >= int64_t(c1 - c0) * kStreamDenNum) attend(std::integral_constant<int, kStream>{});
    else attend(std::integral_constant<int, 0>{});
    if (split >= fold_s0) {   // the window rows that this split takes along (see decode_kv8_splits)
      const int f0 = (split - fold_s0) * kDecodeWinChunk, f1 = min(w, f0 + kDecodeWinChunk);
      const uint32_t size = uint32_t(w) * uint32_t(D * kLocEl);
      Rows<LOC, false, G, D, 0, S> rows(sh, make_rsrc(K_loc + locb, size), make_rsrc(V_loc + locb, size), f0, f1 - f0, 0);
      rows.begin();
      rows.run(m, lsum, acc);
      infinite_values<LOC, D>(V_loc + locb, f0, f1, acc);
    }
  } else {
    Rows<FMT, false, G, D, kStream, S> rows(sh, Kr, Vr, c0, c1 - c0, bshift);
    rows.begin();
    stage();
    __syncthreads();
    rows.run(m, lsum, acc);
  }

  // ---- merge the waves, write this split's partial state per head
  lsum += __shfl_xor(lsum, 16, kWave);
  lsum += __shfl_xor(lsum, 32, kWave);
  if (j == 0 && x < G) {
    sh.sm[wave][x] = lsum == lsum ? m : lsum;   // (a NaN among the logits goes through the joins as the maximum)
    sh.sl[wave][x] = lsum;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int h = 4 * j + i;
    if (h < G) {
#pragma unroll
      for (int c = 0; c < D / 16; c += 4)
        *reinterpret_cast<f32x4*>(&sh.sacc[wave][h][(D / 16) * x + c]) =
            f32x4{acc[c][i], acc[c + 1][i], acc[c + 2][i], acc[c + 3][i]};
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < G * (D / 4); e += kDThreads) {
    const int g = e / (D / 4), d4 = e % (D / 4);
    float M = -INFINITY;
#pragma unroll
    for (int v = 0; v < kDWaves; ++v) M = fmaxf(M, sh.sm[v][g]);
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll
    for (int v = 0; v < kDWaves; ++v) {
      if (sh.sm[v][g] != -INFINITY) {
        const float sc = __builtin_amdgcn_exp2f(sh.sm[v][g] - M);
        const f32x4 a = *reinterpret_cast<const f32x4*>(&sh.sacc[v][g][4 * d4]);
        r = f32x4{fmaf(a.x, sc, r.x), fmaf(a.y, sc, r.y), fmaf(a.z, sc, r.z), fmaf(a.w, sc, r.w)};
        l = fmaf(sh.sl[v][g], sc, l);
      }
    }
    f32x2* o = reinterpret_cast<f32x2*>(part + (int64_t(row0 + g) * total_splits + split) * (D + 2));
    if (d4 == 0) o[0] = f32x2{l == l ? M : l, l};
    o[1 + 2 * d4] = f32x2{r.x, r.y};
    o[2 + 2 * d4] = f32x2{r.z, r.w};
  }
}

// Joins the splits of query head blockIdx.x (states {m in the log2 domain, l, acc[D]}), a quarter
// of its dimensions per block: a thread takes one dimension of every kGroups'th split, BATCH
// at once, their common maximum first so that the weights do not wait for each other; the
// groups are then added in order. (A state without rows holds m = -inf and nothing else.)
template <int D, int BATCH>
__global__ __launch_bounds__(kDThreads) void join_kv8_kernel(const float* __restrict__ part, int splits,
                                                             float* __restrict__ out, float* __restrict__ lse) {
  constexpr int kDims = D / 4, kGroups = kDThreads / kDims;
  __shared__ float gm[kGroups][kDims], gl[kGroups][kDims], go[kGroups][kDims];
  const int row = blockIdx.x, dl = threadIdx.x % kDims, grp = threadIdx.x / kDims, d = blockIdx.y * kDims + dl;
  const float* pr = part + int64_t(row) * splits * (D + 2);
  auto weight = [](float m, float top) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top); };
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int s0 = grp; s0 < splits; s0 += kGroups * BATCH) {
    float ms[BATCH], ls[BATCH], os[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int s = s0 + kGroups * k;
      const float* ps = pr + int64_t(min(s, splits - 1)) * (D + 2);
      ms[k] = ps[0];
      ls[k] = ps[1];
      os[k] = ps[2 + d];
      if (s >= splits) ms[k] = -INFINITY;
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < BATCH; ++k) top = fmaxf(top, ms[k]);
    const float w0 = weight(m, top);
    l *= w0;
    o *= w0;
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const float w = weight(ms[k], top);
      l = fmaf(w, ms[k] == -INFINITY ? 0.f : ls[k], l);
      o = fmaf(w, ms[k] == -INFINITY ? 0.f : os[k], o);
    }
    m = top;
  }
  gm[grp][dl] = l == l ? m : l;
  gl[grp][dl] = l;
  go[grp][dl] = o;
  __syncthreads();
  if (grp != 0) return;
  float top = -INFINITY;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) top = fmaxf(top, gm[g][dl]);
  l = o = 0.f;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    const float w = weight(gm[g][dl], top);
    l = fmaf(w, gl[g][dl], l);
    o = fmaf(w, go[g][dl], o);
  }
  out[int64_t(row) * D + d] = l == 0.f ? 0.f : o / l;
  if (lse && d == 0) lse[row] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
}

// The smallest batch that takes a thread's splits in one round: with 18 throughout, 512 heads
// of 33 splits take 7.8 us instead of 4.8, 32 heads of 19 3.4 instead of 2.8. (The
// full-precision decode's join, whose weights wait for each other, 6.3 and 4.2.)
template <int D>
void launch_join(int rows, int splits, const float* part, float* out, float* lse, hipStream_t stream) {
  constexpr int kGroups = kDThreads / (D / 4);
  const dim3 grid(rows, 4);
  const int own = (splits + kGroups - 1) / kGroups;
  if (own <= 2) join_kv8_kernel<D, 2><<<grid, kDThreads, 0, stream>>>(part, splits, out, lse);
  else if (own <= 5) join_kv8_kernel<D, 5><<<grid, kDThreads, 0, stream>>>(part, splits, out, lse);
  else if (own <= 10) join_kv8_kernel<D, 10><<<grid, kDThreads, 0, stream>>>(part, splits, out, lse);
  else join_kv8_kernel<D, 18><<<grid, kDThreads, 0, stream>>>(part, splits, out, lse);
}

struct Call {
  dim3 grid;
  hipStream_t stream;
  const float* q;
  const Kv8Cache& c;
  int n;
  const int32_t *sel_idx, *sel_count;
  const unsigned long long* sel_mask;
  int mask_words;
  const Kv8Window& win;
  DecodeSplits sp;
  float scale_log2e;
  float* part;
  int Hq, Hkv;
  const int32_t *seq_n, *seq_w;
  int ragged, ordered;
};

template <int FMT, int LOC, bool SPARSE, int G, int D>
void launch(const Call& a) {
  decode_kv8_kernel<FMT, LOC, SPARSE, G, D><<<a.grid, kDThreads, 0, a.stream>>>(
      a.q, static_cast<const char*>(a.c.K8), static_cast<const char*>(a.c.V8), a.c.k_scale, a.c.v_scale,
      __builtin_ctz(unsigned(a.c.block)), a.c.cap, a.n, a.sel_idx, a.sel_count, a.sel_mask, a.mask_words,
      static_cast<const char*>(a.win.K), static_cast<const char*>(a.win.V), a.win.ld, a.win.w, a.sp.chunk,
      a.sp.idx_splits, a.sp.total(), a.sp.fold_wq > 0 ? a.sp.fold_s0 : INT32_MAX, a.scale_log2e, a.part, a.Hq, a.Hkv,
      a.seq_n, a.seq_w, a.ragged, a.ordered);
}
template <int FMT, int LOC, bool SPARSE, int D>
rbq_status launch_g(int G, const Call& a) {
  switch (G) {
    case 1: launch<FMT, LOC, SPARSE, 1, D>(a); break;
    case 2: launch<FMT, LOC, SPARSE, 2, D>(a); break;
    case 4: launch<FMT, LOC, SPARSE, 4, D>(a); break;
    case 8: launch<FMT, LOC, SPARSE, 8, D>(a); break;
    case 16: launch<FMT, LOC, SPARSE, 16, D>(a); break;
    default: return RBQ_EUNSUPPORTED;
  }
  return RBQ_OK;
}
template <int FMT, int LOC, int D>
rbq_status launch_kind(bool sparse, int G, const Call& a) {
  return sparse ? launch_g<FMT, LOC, true, D>(G, a) : launch_g<FMT, LOC, false, D>(G, a);
}
}  // namespace

rbq_status launch_decode_kv8(int32_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const float* q,
                             const Kv8Cache& cache, int32_t n, const int32_t* sel_idx, const int32_t* sel_count,
                             const Kv8Window& win, float sm_scale, float* out, float* lse, void* ws, bool sparse,
                             hipStream_t stream, const unsigned long long* sel_mask, int32_t mask_words,
                             const int32_t* seq_n, const int32_t* seq_w) {
  const int G = heads_q / heads_kv;
  const DecodeSplits sp = decode_kv8_splits(batch, heads_kv, n, win.w, sparse, seq_n != nullptr, seq_w != nullptr);
  const bool ragged = seq_n || seq_w;
  const dim3 grid = ragged ? dim3(uint32_t(batch * heads_kv * int64_t(sp.total()))) : dim3(sp.total(), batch * heads_kv);
  const int64_t blocks = int64_t(batch) * heads_kv * sp.total();
  // (more blocks than the full-precision kernel has at once; this one has 4 or 5 at D = 64 where that has 4 or 6)
  const int ordered = sparse && seq_n && batch > 1 && batch <= kWave && sp.chunk >= kOrderMinChunk &&
                              blocks > resident_blocks(head_dim, G) ? batch : 0;
  const Call a{grid, stream, q, cache, n, sel_idx, sel_count, sel_mask, mask_words, win, sp,
               float(double(sm_scale) * 1.4426950408889634), static_cast<float*>(ws), heads_q, heads_kv, seq_n, seq_w,
               ragged ? batch : 0, ordered};
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
