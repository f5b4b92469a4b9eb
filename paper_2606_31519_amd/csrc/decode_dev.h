// Device code that the decode kernels share: the row list of a sparse split,
// the order of a ragged batch's blocks, and the split of fp32 values into bf16
// parts for the matrix cores.
#pragma once

#include "rbq_device.h"
#include "rbq_internal.h"

namespace rbq {
namespace {

constexpr int kDWaves = 4;
constexpr int kDThreads = kDWaves * kWave;
constexpr int kBmWords = kDecodeChunk / 32;                       // words of the indexed positions
constexpr int kListRounds = (kDecodeChunk + kDecodeFoldMax + kDThreads - 1) / kDThreads;
constexpr int kListCap = kListRounds * kDThreads;                 // list positions (indexed + folded window)
static_assert(kListCap == kDecodeListCap, "the split sizing on the host assumes this list capacity");
constexpr int kListPad = 16;                                      // a list ends on a whole group of rows
static_assert(kListCap % kListPad == 0, "the padding fits");

// K / V buffer loads: an offset past every buffer (the load is dropped), the streaming
// policy's bits, and the share of a sparse block's positions from which on it is used.
constexpr int kSkipOffset = 0x7FFFFF00;
constexpr int kStream = 2;   // cache-policy bits of the K / V buffer loads: nt
constexpr int kStreamDenNum = 1, kStreamDenDen = 3;   // a third of the block's positions

// Lower bounds of x0 and x1 in the ascending a[0, cnt) (first index whose
// value is >= x), found together by one wave: each round probes 64 evenly
// spaced entries per search and keeps the gap where the answer lies, so a list
// of 2^17 entries takes three rounds of loads for both. Every lane returns both.
__device__ __forceinline__ void wave_lower_bounds(const int32_t* __restrict__ a, int cnt, int x0, int x1, int& r0,
                                                  int& r1) {
  const int lane = lane_id();
  int lo0 = 0, hi0 = cnt, lo1 = 0, hi1 = cnt;   // each answer lies in [lo, hi]
  while (hi0 > lo0 || hi1 > lo1) {
    const int st0 = (hi0 - lo0 + kWave - 1) / kWave, st1 = (hi1 - lo1 + kWave - 1) / kWave;
    const int p0 = lo0 + lane * st0, p1 = lo1 + lane * st1;
    // both probes' loads unconditionally, the indices clamped into the list
    // (which holds an entry here: cnt > lo >= 0), so that they are in flight together
    const int v0 = a[min(p0, cnt - 1)], v1 = a[min(p1, cnt - 1)];
    const bool lt0 = p0 < hi0 && v0 < x0;
    const bool lt1 = p1 < hi1 && v1 < x1;
    const int k0 = __popcll(__ballot(lt0)), k1 = __popcll(__ballot(lt1));   // the first k probes are below x
    if (hi0 > lo0) {
      if (k0 == 0) {
        hi0 = lo0;
      } else {
        lo0 += (k0 - 1) * st0 + 1;
        hi0 = min(hi0, lo0 - 1 + st0);
      }
    }
    if (hi1 > lo1) {
      if (k1 == 0) {
        hi1 = lo1;
      } else {
        lo1 += (k1 - 1) * st1 + 1;
        hi1 = min(hi1, lo1 - 1 + st1);
      }
    }
  }
  r0 = lo0;
  r1 = lo1;
}

// Lower bounds of x in H lists a[h][0, cnt[h]) at once: their rounds of loads overlap.
template <int H>
__device__ __forceinline__ void wave_lower_bound_of(const int32_t* const (&a)[H], const int (&cnt)[H], int x,
                                                    int (&lo)[H]) {
  const int lane = lane_id();
  int hi[H];
  bool open = false;
#pragma unroll
  for (int h = 0; h < H; ++h) {
    lo[h] = 0;
    hi[h] = cnt[h];
    open |= cnt[h] > 0;
  }
  while (open) {
    int v[H], st[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      st[h] = (hi[h] - lo[h] + kWave - 1) / kWave;
      v[h] = a[h][max(min(lo[h] + lane * st[h], cnt[h] - 1), 0)];   // (clamped into the row: some list holds an entry)
    }
    open = false;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int k = __popcll(__ballot(lo[h] + lane * st[h] < hi[h] && v[h] < x));   // the first k probes are below x
      if (hi[h] > lo[h]) {
        if (k == 0) {
          hi[h] = lo[h];
        } else {
          lo[h] += (k - 1) * st[h] + 1;
          hi[h] = min(hi[h], lo[h] - 1 + st[h]);
        }
      }
      open |= hi[h] > lo[h];
    }
  }
}

// This lane's words of the split's selection bitmaps: word l % 16 (keys
// c0 + 64 (l % 16) .. + 64) of heads l / 16 + 4k. Every wave of the block reads
// the same words; the matrix-core kernel requests them at its start so that the
// loads overlap the query staging. (Bits past the split's last position are
// cleared where the words are used, so that no wait for the loads is placed here.)
template <int G>
struct MaskWords {
  unsigned long long w[(G + 3) / 4];
};
template <int G>
__device__ __forceinline__ MaskWords<G> load_mask_words(const unsigned long long* __restrict__ sel_mask,
                                                        int mask_words, int row0, int c0, int c1) {
  MaskWords<G> m;
  const int lane = lane_id(), wd = lane & 15;
#pragma unroll
  for (int k = 0; k < (G + 3) / 4; ++k) {
    const int g = lane / 16 + 4 * k;
    m.w[k] = sel_mask != nullptr && g < G && c0 + 64 * wd < c1
                 ? sel_mask[int64_t(row0 + g) * mask_words + c0 / 64 + wd]
                 : 0ull;
  }
  return m;
}

// The selection counts of this wave's heads (wave, wave + kDWaves, ...) for
// the searches of the separate sparse call, requested at the start of the
// kernel so that the load overlaps the query staging.
template <int G>
struct HeadCounts {
  int c[(G + kDWaves - 1) / kDWaves];
};
template <int G>
__device__ __forceinline__ HeadCounts<G> load_head_counts(const int32_t* __restrict__ sel_count, int row0) {
  HeadCounts<G> h;
  const int wave = threadIdx.x / kWave;
#pragma unroll
  for (int i = 0; i < (G + kDWaves - 1) / kDWaves; ++i) {
    const int g = min(wave + kDWaves * i, G - 1);   // (a wave past the heads loads the last one's, unused)
    h.c[i] = sel_count[row0 + g];                    // (clamped where it is used: no wait here)
  }
  return h;
}

// Per-block row list of a sparse split: the union over the G heads of the
// group of the positions in [c0, c1) that each head selected, in ascending
// order, with a bit mask of the heads that selected each entry, followed by
// the nwin window rows folded into the split (every head; list positions
// c1 - c0 + i, rows c1 + wshift + i), and padded to whole groups of kPad
// entries with a listed row that no head takes. Returns the number of entries without
// the padding (block-uniform). All threads of the block must call it.
// The list is ranked from the split's 16 words of 64 positions per head: the
// selection's bitmaps themselves when given (sel_mask != NULL, [rows][mask_words]
// words of 64 keys, c0 a multiple of 64); otherwise each wave finds the part
// [lower bound of c0, lower bound of c1) of its heads' selection lists (their
// counts in hc), and the entries, loaded all at once, are marked in per-head
// LDS bitmaps that then serve as the words.
// ONE (the 8-bit decode): only the lower bound of c0 is searched for, of a wave's heads
// together, and the entries are read on from there until they pass c1. A round of probes
// touches 64 lines per wave, which costs more than entries read in vain: the call over
// 128K rows, a fifth per head 45.0 -> 43.9 us, 8 x 2-32K of 64 heads 37.2 -> 34.3, 64K at
// D = 64 16.3 -> 15.4. (More probes per round, to save one: 51, 38.2 and 17.1.)
template <int G, int kThreads, bool PRE, int kPad = kListPad, bool ONE = false>
__device__ __forceinline__ int build_union_list(const int32_t* __restrict__ sel_idx,
                                const unsigned long long* __restrict__ sel_mask, int mask_words, int row0,
                                int n, int c0, int c1, int nwin, int wshift, uint32_t (*bm)[kBmWords], int32_t* lst,
                                uint16_t* hmask, int* rng_lo, int* rng_hi, MaskWords<G> mw,
                                const HeadCounts<G>& hc) {
  constexpr int kWaves = kThreads / kWave;
  const int t = threadIdx.x, wave = t / kWave, lane = lane_id();
  const int wd = lane & 15;
  if (sel_mask == nullptr) {
    static_assert(kWaves == kDWaves, "the preloaded counts assume the decode block");
    constexpr int kHeads = (G + kWaves - 1) / kWaves;   // of a wave
    if constexpr (ONE) {
      const int32_t* rows[kHeads];
      int cnts[kHeads], at[kHeads];
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        rows[i] = sel_idx + int64_t(row0 + min(wave + kWaves * i, G - 1)) * n;
        cnts[i] = min(max(__builtin_amdgcn_readfirstlane(hc.c[i]), 0), n);
      }
      wave_lower_bound_of<kHeads>(rows, cnts, c0, at);
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        if (lane == 0 && wave + kWaves * i < G) {
          rng_lo[wave + kWaves * i] = at[i];
          rng_hi[wave + kWaves * i] = cnts[i];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        const int g = wave + kWaves * i;
        if (g >= G) break;   // (wave-uniform)
        const int32_t* sel = sel_idx + int64_t(row0 + g) * n;
        const int cnt = min(max(hc.c[i], 0), n);
        int lo, hi;
        wave_lower_bounds(sel, cnt, c0, c1, lo, hi);
        if (lane == 0) {
          rng_lo[g] = lo;
          rng_hi[g] = hi;
        }
      }
    }
    for (int e = t; e < G * kBmWords; e += kThreads) bm[e / kBmWords][e % kBmWords] = 0u;
    __syncthreads();
    // mark the selected positions: every entry's load first, then the LDS bit sets
    constexpr int kPer = kDecodeChunk / kThreads;            // entries per thread per head (a split has <= chunk)
    constexpr int kHB = G < 4 ? G : 4;                      // heads per batch of loads
#pragma unroll
    for (int g0 = 0; g0 < G; g0 += kHB) {
      if constexpr (ONE) {
        // a first round of every head's entries, then on for those whose last one lies in the split
        int v[kHB], from[kHB], end[kHB];
#pragma unroll
        for (int gg = 0; gg < kHB; ++gg) {
          from[gg] = rng_lo[g0 + gg];
          end[gg] = min(rng_hi[g0 + gg], from[gg] + (c1 - c0));
        }
        bool more = true;
        for (int u = 0; more; u += kThreads) {
          int last[kHB];
#pragma unroll
          for (int gg = 0; gg < kHB; ++gg) {
            const int32_t* sel = sel_idx + int64_t(row0 + g0 + gg) * n;
            v[gg] = sel[max(min(from[gg] + u + t, end[gg] - 1), 0)];
            last[gg] = sel[max(min(from[gg] + u + kThreads - 1, end[gg] - 1), 0)];
          }
          more = false;
#pragma unroll
          for (int gg = 0; gg < kHB; ++gg) {
            const int pos = from[gg] + u + t < end[gg] ? v[gg] - c0 : -1;
            if (pos >= 0 && pos < c1 - c0) atomicOr(&bm[g0 + gg][pos >> 5], 1u << (pos & 31));
            more |= from[gg] + u + kThreads < end[gg] && last[gg] < c1;
          }
        }
        continue;
      }
      int pv[kHB][kPer];
#pragma unroll
      for (int gg = 0; gg < kHB; ++gg) {
        const int g = g0 + gg;
        const int32_t* sel = sel_idx + int64_t(row0 + g) * n;
        const int lo = rng_lo[g], hi = rng_hi[g];
#pragma unroll
        for (int u = 0; u < kPer; ++u) {   // (loaded unconditionally, the index clamped into the row, so
          const int e = lo + u * kThreads + t;   // that every load is in flight at once)
          const int v = sel[max(min(e, hi - 1), 0)];
          pv[gg][u] = e < hi ? v - c0 : -1;
        }
      }
#pragma unroll
      for (int gg = 0; gg < kHB; ++gg)
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
          const int pos = pv[gg][u];
          if (pos >= 0 && pos < c1 - c0) atomicOr(&bm[g0 + gg][pos >> 5], 1u << (pos & 31));
        }
    }
    __syncthreads();
    // this lane's words, laid out as load_mask_words gives them
#pragma unroll
    for (int k = 0; k < (G + 3) / 4; ++k) {
      const int g = lane / 16 + 4 * k;
      mw.w[k] = g < G ? (uint64_t(bm[g][2 * wd + 1]) << 32) | bm[g][2 * wd] : 0ull;
    }
  } else if (!PRE) {
    mw = load_mask_words<G>(sel_mask, mask_words, row0, c0, c1);
  }
  // Every wave ranks the split's 16 union words itself: lane l holds word
  // l % 16 of heads l / 16 + 4k, the heads' words are ORed across the rows of
  // 16 lanes, and an exclusive prefix of their popcounts gives each word's
  // first list entry. Wave v then writes the entries of words v, v + kWaves,
  // ... and the last wave the folded window rows; one barrier publishes the list.
  const int lim = c1 - c0 - 64 * wd;   // positions of word wd inside the split
  const unsigned long long keep = lim >= 64 ? ~0ull : lim > 0 ? (1ull << lim) - 1ull : 0ull;
  unsigned long long u = 0ull;
#pragma unroll
  for (int k = 0; k < (G + 3) / 4; ++k) {
    mw.w[k] &= keep;
    u |= mw.w[k];
  }
  u |= swap16_u64(u);   // lanes l and l ^ 16
  u |= (uint64_t(uint32_t(__shfl_xor(int(uint32_t(u >> 32)), 32, kWave))) << 32) |
       uint32_t(__shfl_xor(int(uint32_t(u)), 32, kWave));
  const uint32_t c = uint32_t(__popcll(u));
  uint32_t inc = c;   // inclusive prefix over the 16 words of each row of lanes
  inc += RBQ_DPP_U32(inc, 0x111);   // row_shr:1
  inc += RBQ_DPP_U32(inc, 0x112);   // row_shr:2
  inc += RBQ_DPP_U32(inc, 0x114);   // row_shr:4
  inc += RBQ_DPP_U32(inc, 0x118);   // row_shr:8
  const uint32_t excl = inc - c;
  const int nidx = __builtin_amdgcn_readlane(int(inc), 15);
  for (int v = wave; v < kBmWords / 2; v += kWaves) {   // (wave-uniform)
    const unsigned long long uw = readlane_u64(u, v);
    const int off = __builtin_amdgcn_readlane(int(excl), v);
    uint32_t mk = 0u;   // (a head's word is the lane mask itself: one select per head)
#pragma unroll
    for (int g = 0; g < G; ++g)
      mk |= __builtin_amdgcn_inverse_ballot_w64(readlane_u64(mw.w[g / 4], (g % 4) * 16 + v)) ? 1u << g : 0u;
    if (__builtin_amdgcn_inverse_ballot_w64(uw)) {
      const int o = off + int(__builtin_amdgcn_mbcnt_hi(uint32_t(uw >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(uw), 0u)));
      lst[o] = c0 + 64 * v + lane;
      hmask[o] = uint16_t(mk);
    }
  }
  if (wave == kWaves - 1) {
    for (int i = lane; i < nwin; i += kWave) {   // the folded window rows, every head
      lst[nidx + i] = c1 + wshift + i;
      hmask[nidx + i] = uint16_t((1u << G) - 1u);
    }
    // up to a whole group: a listed row once more, for no head (a row that is not
    // listed may hold anything, and its values would meet probabilities of zero)
    const int v0 = __builtin_ctzll(__ballot(u != 0ull) | (1ull << 63)) & 15;
    const unsigned long long w0 = readlane_u64(u, v0);
    const int o = nidx + nwin + lane;
    if (lane < kPad && o < (nidx + nwin + kPad - 1) / kPad * kPad) {
      lst[o] = nidx > 0 ? c0 + 64 * v0 + __builtin_ctzll(w0 | (1ull << 63)) : c1 + wshift;
      hmask[o] = 0;
    }
  }
  __syncthreads();
  return nidx + nwin;
}

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kQParts = 3;       // the query as hi + mid + lo bf16 parts

// x = hi + mid + lo in bf16 parts, each rounded to nearest even
__device__ __forceinline__ void split3(const f32x8 x, bf16x8* p) {
  f32x8 r = x;
#pragma unroll
  for (int t = 0; t < kQParts; ++t) {
    p[t] = __builtin_convertvector(r, bf16x8);
    if (t + 1 < kQParts) r -= __builtin_convertvector(p[t], f32x8);
  }
}

// The sequence that the blocks of rank r take: sequences by the share of their
// indexed keys that is selected (of one query head each of up to 8 KV heads),
// the densest first. Lane b weighs sequence b (batch <= 64); its n_b in `own`.
// Blocks of dense sequences take several times as long as the others (16 sequences
// of 2K to 32K keys, p 0.5 to 0.95: 37 to 46 us against 7 to 13), and started last
// they run on alone: 72 us for that launch, densest first 58. The order costs a block
// one more round of loads, so launches that are resident at once keep theirs (64
// dimensions, 6 x 28K keys, 1344 blocks: 29.9 us, ordered 34.4), and so do launches
// in the shortest chunks, whose blocks are too short for it (32 / 8 heads of 128, 9 x
// 4K keys, 1152 blocks: 19.5 us, ordered 22.4; 6 x 8K, 1536 blocks: 21.9 and 22.9).
// Longer ones gain: 12 x 8K, chunks of 512: 44.5 -> 33.7; 64 dimensions, 8 x 28K:
// 47.8 -> 36.2; groups of 16, 12 x 32K, 1512 blocks: 73.6 -> 55.6.
constexpr int kOrderMinChunk = 512;
// blocks resident at once (256 CUs; registers, for groups of 16 heads the LDS)
constexpr int64_t resident_blocks(int D, int G) { return 256 * (D == 64 ? (G == 16 ? 4 : 6) : (G == 16 ? 2 : 4)); }
constexpr int kOrderHeads = 8;
// the share of sequence b's `own` indexed keys that up to kOrderHeads of its query heads select
__device__ __forceinline__ float selected_share(int b, int own, int Hq, int Hkv, const int32_t* __restrict__ sel_count) {
  const int G = Hq / Hkv;
  int cnt[kOrderHeads];
#pragma unroll
  for (int k = 0; k < kOrderHeads; ++k) cnt[k] = sel_count[b * Hq + k * Hkv / kOrderHeads * G];
  int sum = 0;
#pragma unroll
  for (int k = 0; k < kOrderHeads; ++k) sum += cnt[k];
  return float(sum) / float(max(own, 1));
}
__device__ __forceinline__ int sequence_of_rank(int r, int batch, int n, int Hq, int Hkv,
                                                const int32_t* __restrict__ sel_count,
                                                const int32_t* __restrict__ seq_n, int& own) {
  const int lane = lane_id(), b = min(lane, batch - 1);
  own = min(max(seq_n[b], 0), n);
  const float dens = selected_share(b, own, Hq, Hkv, sel_count);
  int rank = 0;
  for (int o = 0; o < batch; ++o) {
    const float d = __uint_as_float(uint32_t(__builtin_amdgcn_readlane(int(__float_as_uint(dens)), o)));
    rank += d > dens || (d == dens && o < lane) ? 1 : 0;
  }
  return __builtin_ctzll(__ballot(lane < batch && rank == r) | (1ull << 63));
}

}  // namespace
}  // namespace rbq
