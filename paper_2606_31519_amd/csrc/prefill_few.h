// rbq_prefill_attention_kv4 of few rows: a turn of some tokens, drafted tokens that are
// checked, over long 4-bit rows. Included by prefill.hip.
#pragma once

namespace rbq {
namespace {

template <int DTYPE>
struct Elem {
  typedef uint16_t T;
};
template <>
struct Elem<RBQ_F32> {
  typedef float T;
};
__device__ __forceinline__ float element(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }
__device__ __forceinline__ float element(const float* p) { return *p; }
__device__ __forceinline__ f32x8 load8(const float* p) {
  const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
// N bf16 parts of eight values, each the top 8 bits of what the ones before leave (24 bits in three,
// the largest floats among them)
template <int N>
__device__ __forceinline__ void top_parts(f32x8 v, u32x4* to) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      to[n][i] = __builtin_amdgcn_perm(__float_as_uint(v[2 * i + 1]), __float_as_uint(v[2 * i]), 0x07060302u);
    if (n + 1 < N) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] -= __uint_as_float(__float_as_uint(v[i]) & 0xFFFF0000u);
    }
  }
}

// Block id of a KV head: sequence after sequence, tile after tile, the splits that the sequence's
// keys call for; the grid's rest has none (b < 0).
template <int FMT>
__device__ __forceinline__ TileId find_few(int id, int kchunk, int batch, int G, int BM, int total_q, int& live,
                                           const int32_t* __restrict__ cu_q, const Cached& c4) {
  const int lane = lane_id();
  TileId t{-1, 0, 0, 0, 0, 0, 0, 0};
  int before = 0;
  for (int b0 = 0; b0 < batch; b0 += kWave) {
    const Lengths s = lengths_of<FMT>(min(b0 + lane, batch - 1), G, BM, total_q, 0, 0, true, cu_q, cu_q, c4);
    const int splits = (s.nk + kchunk - 1) / kchunk, mine = b0 + lane < batch ? s.tiles * splits : 0;
    int inc = mine;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int u = __shfl_up(inc, o, kWave);
      inc += lane >= o ? u : 0;
    }
    const int first = before + inc - mine;
    const unsigned long long at = __ballot(id >= first && id < first + mine);
    if (at != 0ull) {
      const int l = __builtin_ctzll(at), e = id - __builtin_amdgcn_readlane(first, l);
      live = __builtin_amdgcn_readlane(splits, l);
      t.b = b0 + l;
      t.tile = e / live;
      t.split = e - t.tile * live;
      t.q0 = __builtin_amdgcn_readlane(s.q0, l);
      t.nq = __builtin_amdgcn_readlane(s.nq, l);
      t.nk = __builtin_amdgcn_readlane(s.nk, l);
      t.k0 = t.q0;
      t.nb = __builtin_amdgcn_readlane(s.nb, l);
      return t;
    }
    before += __builtin_amdgcn_readlane(inc, kWave - 1);
  }
  return t;
}

// A block takes 32 rows (token, head of the group) of a sequence and KV head, as prefill_kernel's
// wave does, and its four waves take groups of 32 keys in turn, each with its own maximum, sum
// and outputs, merged at the end. The codes go from memory into the operands, without LDS:
//   S^T = K Q^T    A = 32 keys: lane (key x, half h) holds dimensions (D / 2) h .. +D / 2, one load
//                  or two; int4's codes as whole numbers, its steps and bases meet the products
//                  (logit = s <q, c> + m sum(q)), so that keys are not rounded
//   O^T = V^T P^T  A = 32 x (D / 32) dimensions: lane (x, h) holds dimensions (D / 32) x .. of the 16
//                  keys whose probabilities it has; int4: weights w = bf16(p s) on the codes, and
//                  w (m / s) beside them, so that both see the same rounding
// fp32: queries and weights in three bf16 parts, 24 bits (4-bit codes and values are exact in
// bf16), the chunk's own rows too: three products for one are a fifth of what the fp32 matrix
// instructions take (2 x 31-500 tokens of 8 / 2 heads of 64 over up to 6000 rows, int4: 38.8 us,
// 72.1 with them in prefill_f32_kernel). int4's rows as c - 7.5 and m + 7.5 s: sums of c itself, which m then cancels, cost
// twice the rounding (rel. error of the outputs 1.6e-6, so 7.8e-7).
// (In prefill_kernel, 128 rows and tiles through LDS, 8 x 7 tokens of 32 / 8 heads over up to
// 8000 rows take 36.2 us in int4 and 30.3 in fp4, here 22.2 and 20.1.)
// At D = 128 fp32 has all 256 registers and 96 (fp4) or 108 bytes (int4) of scratch a lane: 2 x 31-500 tokens of
// 8 / 2 heads over up to 6000 rows, int4, 70 us (in prefill_f32_kernel 130).
template <int D, int FMT, int DTYPE>
__global__ __launch_bounds__(kPThreads, 2) void prefill_few_kernel(
    const typename Elem<DTYPE>::T* __restrict__ q, int64_t q_ld, const typename Elem<DTYPE>::T* __restrict__ K,
    const typename Elem<DTYPE>::T* __restrict__ V, int64_t kv_ld, int64_t kv_head, const int32_t* __restrict__ cu_q,
    int batch, int total_q, int causal,
    float scale_log2e, typename Elem<DTYPE>::T* __restrict__ out, float* __restrict__ lse, float* __restrict__ part,
    int Hq, int Hkv, int splits, int kchunk, Cached c4) {
  constexpr int KB = D / 16, DT = D / 32, kGroup = 32, KW = D / 16;   // k-blocks, dimensions of a lane, words of K
  constexpr bool kBase = FMT == RBQ_I4, kF32 = DTYPE == RBQ_F32;
  constexpr int NP = kF32 ? 3 : 1;   // bf16 parts of a query, a probability, a row of the chunk's own
  using T = typename Elem<DTYPE>::T;
  __shared__ u32x4 qparts[kF32 ? NP : 1][kF32 ? KB : 1][kF32 ? kWave : 1];   // fp32: the queries' operands
  struct Wave {
    // fp4: V's scales of four groups; int4: K's s and m, V's s and m / s (fp32: m + 7.5 s of both)
    __attribute__((aligned(16))) float word[4][kGroup];
  };
  __shared__ Wave per_wave[kPWaves];
  __shared__ __attribute__((aligned(16))) f32x4 held[2][4 * DT][kWave];   // outputs of two waves
  __shared__ float held_m[2][kWave], held_l[2][kWave];
  __shared__ int odd;
  const int G = Hq / Hkv, hk = blockIdx.x % Hkv;
  int live = 0;   // splits of its sequence
  const TileId t = find_few<FMT>(int(blockIdx.x) / Hkv, kchunk, batch, G, kGroup, total_q, live, cu_q, c4);
  if (t.b < 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int x = lane & 31, h = lane >> 5;
  const int rows = t.nq * G, row0 = t.tile * kGroup, shift = t.nk - t.nq, cached = t.nb;
  const int nbp = (cached + kPKeys - 1) / kPKeys * kPKeys;   // first of the chunk's own keys
  auto visible = [&](int token) { return causal ? min(max(token + shift + 1, 0), t.nk) : t.nk; };
  const int kend = visible((min(row0 + kGroup, rows) - 1) / G), kbeg = t.split * kchunk, kstop = min(kend, kbeg + kchunk);
  const int all = visible(row0 / G);                                 // keys that every row sees
  const int qrow = min(row0 + x, rows - 1), token = qrow / G, head = hk * G + (qrow - token * G), lim = visible(token);
  bf16x8 qf[kF32 ? 1 : KB];
  float qsum = 0.f, odd_q = 0.f;   // odd_q (bf16): NaN where the lane's half of the query has an infinity or NaN
  {
    const T* p = q + int64_t(t.q0 + token) * q_ld + head * D + (D / 2) * h;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      if constexpr (kF32) {
        const f32x8 v = load8(p + 8 * kb);
        if constexpr (kBase) qsum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        if (kb % kPWaves == wave) {
          u32x4 part[NP];
          top_parts<NP>(v, part);
#pragma unroll
          for (int n = 0; n < NP; ++n) qparts[n][kb][lane] = part[n];
        }
      } else {
        qf[kb] = *reinterpret_cast<const bf16x8*>(p + 8 * kb);
#pragma unroll
        for (int i = 0; i < 8; ++i) odd_q = fmaf(float(qf[kb][i]), 0.f, odd_q);
        if constexpr (kBase) {
#pragma unroll
          for (int i = 0; i < 8; ++i) qsum += float(qf[kb][i]);
        }
      }
    }
    if constexpr (kBase) qsum += __shfl_xor(qsum, 32, kWave);
  }
  // part n of the queries' dimensions 8 kb .. of the lane's
  auto query = [&](int n, int kb) {
    if constexpr (kF32) return __builtin_bit_cast(bf16x8, qparts[n][kb][lane]);
    else return qf[kb];
  };
  if (threadIdx.x == 0) odd = 0;
  __syncthreads();
  const int64_t first = (int64_t(t.b) * Hkv + hk) * c4.cap;
  const __amdgpu_buffer_rsrc_t rec = make_rsrc(c4.KV4 + first * D, uint32_t(cached) * D);   // < 2^31
  const __amdgpu_buffer_rsrc_t words = make_rsrc(c4.par + 2 * first, uint32_t(cached) * 8u);
  const T *Kb = K + t.k0 * kv_ld + int64_t(hk) * kv_head, *Vb = V + t.k0 * kv_ld + int64_t(hk) * kv_head;
  float(*word)[kGroup] = per_wave[wave].word;

  // a group of 4-bit keys on its way; places behind the last row lie past the buffers' ends: zeros
  uint32_t kw[KW], vw[16];
  u32x2 pw;
  auto key_of = [&](int i) { return 16 * (i / 8) + 8 * (i % 8 / 4) + 4 * h + i % 4; };   // of the lane's 16 probabilities
  auto load_k = [&](int k0) {
    const int row = k0 + x, at = row * D + D / 4 * h;
#pragma unroll
    for (int i = 0; i < KW / 4; ++i) {
      const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rec, at + 16 * i, 0, 0));
#pragma unroll
      for (int e = 0; e < 4; ++e) kw[4 * i + e] = v[e];
    }
    pw = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(words, row * 8, 0, 0));
  };
  // (the word of eight dimensions that holds the lane's 4 or 2)
  auto load_v = [&](int k0) {
    const int at = (k0 + 4 * h) * D + D / 2 + 4 * (x * DT / 8);
#pragma unroll
    for (int i = 0; i < 16; ++i) vw[i] = __builtin_amdgcn_raw_buffer_load_b32(rec, at + (key_of(i) - 4 * h) * D, 0, 0);
  };

  f32x16 o[DT];
  float m = -INFINITY, l = odd_q, base = 0.f;   // (such a query is NaN, also where all its logits are -infinity)
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  // The softmax of a group's logits: masked, the maximum raised, probabilities in p
  auto softmax = [&](f32x16& s, int k0) {
    if (k0 + kGroup > all || (k0 < nbp && k0 + kGroup > cached)) {
      const int end = k0 < nbp ? min(lim, cached) : lim;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = k0 + key_of(r) < end ? s[r] : -INFINITY;
    }
    float top = fmaxf(s[0], s[1]);
#pragma unroll
    for (int r = 2; r < 16; ++r) top = fmaxf(top, s[r]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale_log2e;
    if (__ballot(top > m)) {
      const float mn = fmaxf(m, top);
      const float corr = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
      base *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= corr;
      m = mn;
    }
    const float mref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale_log2e, -mref));
      l += s[r];
    }
  };
  // weights of keys 16 g .. +16 as operands (bf16: rounded, as in prefill_kernel)
  auto weights = [&](const f32x16& p, int g, u32x4 (&to)[NP]) {
    f32x8 e;
#pragma unroll
    for (int r = 0; r < 8; ++r) e[r] = p[8 * g + r];
    if constexpr (kF32) top_parts<NP>(e, to);
    else to[0] = __builtin_bit_cast(u32x4, __builtin_convertvector(e, bf16x8));
  };
  auto product = [](u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  };

  const int c4groups = max(min(kstop, cached) - kbeg + kGroup - 1, 0) / kGroup;   // of 4-bit keys
  // where the loads of a group behind the last go: past the buffers' ends (or, of a buffer of almost 2^31 bytes, onto
  // rows that are not used), a group's rows before an int's end
  constexpr int kNoRow = 0x7FFE0000 / D;
  if (wave < c4groups) {
    load_k(kbeg + wave * kGroup);
    load_v(kbeg + wave * kGroup);
  }
  // the chunk's own keys, few of them, by the waves that have fewer of the others
  const int own0 = max(kbeg, nbp);   // (a multiple of the groups' 32)
  for (int k0 = own0 + ((wave - c4groups) & 3) * kGroup; k0 < kstop; k0 += kPWaves * kGroup) {
    const T* kp = Kb + int64_t(min(k0 - nbp + x, t.nq - 1)) * kv_ld + (D / 2) * h;
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      if constexpr (kF32) {
        u32x4 a[NP];
        top_parts<NP>(load8(kp + 8 * kb), a);
#pragma unroll
        for (int i = 0; i < NP; ++i)   // (the products of 2^-24 and less are left out)
#pragma unroll
          for (int n = 0; i + n < NP; ++n) s = product(a[i], __builtin_bit_cast(u32x4, query(n, kb)), s);
      } else {
        s = product(*reinterpret_cast<const u32x4*>(kp + 8 * kb), __builtin_bit_cast(u32x4, query(0, kb)), s);
      }
    }
    if constexpr (kF32) {
      // An infinity has no parts (those after the first are NaN): logits that came out infinite or NaN are
      // formed again, from the values themselves.
      float odd_logit = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) odd_logit = fmaf(s[r], 0.f, odd_logit);
      if (__ballot(odd_logit != odd_logit)) {
        const T* qp = q + int64_t(t.q0 + token) * q_ld + head * D;
#pragma unroll 1
        for (int r = 0; r < 16; ++r) {   // (one at a time: registers are short)
          const T* k = Kb + int64_t(min(k0 - nbp + key_of(r), t.nq - 1)) * kv_ld;
          float v = 0.f;
#pragma unroll 2
          for (int d = 0; d < D; d += 8) {
            const f32x8 a = load8(k + d), b = load8(qp + d);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              v = fmaf(a[e], b[e], v);
              l = fmaf(b[e], 0.f, l);   // (as with odd_q)
            }
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = i == r && !(fabsf(s[i]) < INFINITY) ? v : s[i];
        }
      }
    }
    softmax(s, k0);
    bool inf = false;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      u32x4 p[NP];
      weights(s, g, p);
      float v[8][DT];
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const T* vp = Vb + int64_t(min(k0 - nbp + key_of(8 * g + r), t.nq - 1)) * kv_ld + DT * x;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          v[r][d] = element(vp + d);
          // (infinities and NaN: replaced here, added where they are seen, at the end)
          if (!(fabsf(v[r][d]) < INFINITY)) v[r][d] = 0.f, inf = true;
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        f32x8 col;
#pragma unroll
        for (int r = 0; r < 8; ++r) col[r] = v[r][d];
        u32x4 a[NP];
        top_parts<NP>(col, a);   // (bf16: itself)
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
          for (int n = 0; i + n < NP; ++n) o[d] = product(a[i], p[n], o[d]);
      }
    }
    if (inf) odd = 1;
  }

  for (int grp = wave; grp < c4groups; grp += kPWaves) {
    const int k0 = kbeg + grp * kGroup, next = grp + kPWaves < c4groups ? k0 + kPWaves * kGroup : kNoRow;
    // the words' values, of each key, for the lanes that hold it
    float kscale[2] = {0.f, 0.f};
    if constexpr (kBase) {
      const float ks = __uint_as_float(pw.x << 16), km = __uint_as_float(pw.x & 0xFFFF0000u);
      float vs = __uint_as_float(pw.y << 16);
      const float vm = __uint_as_float(pw.y & 0xFFFF0000u);
      if (!kF32) vs = vs == 0.f ? 1.f : vs;   // (a row of one value: its codes are 0)
      word[2 * h][x] = h ? vs : ks;
      word[2 * h + 1][x] = h ? (kF32 ? fmaf(7.5f, vs, vm) : vm / vs) : kF32 ? fmaf(7.5f, ks, km) : km;
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        kscale[i] = __uint_as_float((pw.x >> (8 * (2 * h + i)) & 255u) << 23);
        word[2 * h + i][x] = __uint_as_float((pw.y >> (8 * (2 * h + i)) & 255u) << 23);
      }
    }
    __builtin_amdgcn_wave_barrier();
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      u32x4 a;
      if constexpr (kBase) a = word_whole<kF32>(kw[kb]);
      else a = word_bf16<FMT>(kw[kb], f32x2{kscale[kb / (KB / 2)], 0.f});
#pragma unroll
      for (int n = 0; n < NP; ++n) s = product(a, __builtin_bit_cast(u32x4, query(n, kb)), s);
    }
    load_k(next);
    if constexpr (kBase) {
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 ks = *reinterpret_cast<const f32x4*>(&word[0][8 * a + 4 * h]);
        const f32x4 km = *reinterpret_cast<const f32x4*>(&word[1][8 * a + 4 * h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * a + i] = fmaf(ks[i], s[4 * a + i], km[i] * qsum);
      }
    }
    softmax(s, k0);
    float vscale[16];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(&word[kBase ? 2 : x / 8][8 * a + 4 * h]);
#pragma unroll
      for (int i = 0; i < 4; ++i) vscale[4 * a + i] = v[i];
    }
    u32x4 p[2][NP];
    if constexpr (kBase) {
      f32x16 w;
#pragma unroll
      for (int r = 0; r < 16; ++r) w[r] = s[r] * vscale[r];
      weights(w, 0, p[0]);
      weights(w, 1, p[1]);
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 m4 = *reinterpret_cast<const f32x4*>(&word[3][8 * a + 4 * h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * (a % 2) + i;
          float weight = s[4 * a + i];
          if constexpr (!kF32) weight = r % 2 ? bf16_hi(p[a / 2][0][r / 2]) : bf16_lo(p[a / 2][0][r / 2]);
          base = fmaf(weight, m4[i], base);
        }
      }
    } else {
      weights(s, 0, p[0]);
      weights(s, 1, p[1]);
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 16; ++i)   // the lane's dimensions to the low end (int4: of each half)
      vw[i] >>= kBase ? (D == 128 ? 8 * (x % 2) : 4 * (x % 4)) : (D == 128 ? 16 * (x % 2) : 8 * (x % 4));
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      uint32_t a[DT][4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {   // pairs of keys
        const uint32_t w0 = vw[8 * g + 2 * r], w1 = vw[8 * g + 2 * r + 1];
        if constexpr (kBase) {
          const uint32_t y = __builtin_amdgcn_perm(w1, w0, 0x06020400u), lo = y & 0x0F0F0F0Fu, hi = y >> 4 & 0x0F0F0F0Fu;
          if constexpr (kF32) {
            const uint32_t cl = centred_bytes(lo);
            a[0][r] = centred_bf16<false>(cl);
            a[1][r] = centred_bf16<true>(cl);
            if constexpr (DT == 4) {
              const uint32_t ch = centred_bytes(hi);
              a[2][r] = centred_bf16<false>(ch);
              a[3][r] = centred_bf16<true>(ch);
            }
          } else {
            a[0][r] = bytes_bf16<false>(lo);
            a[1][r] = bytes_bf16<true>(lo);
            if constexpr (DT == 4) {
              a[2][r] = bytes_bf16<false>(hi);
              a[3][r] = bytes_bf16<true>(hi);
            }
          }
        } else {
          const float s0 = vscale[8 * g + 2 * r], s1 = vscale[8 * g + 2 * r + 1];
#pragma unroll
          for (int b = 0; b < DT / 2; ++b) {
            const uint32_t u0 = b ? fp4_pair<1>(w0, s0) : fp4_pair<0>(w0, s0);
            const uint32_t u1 = b ? fp4_pair<1>(w1, s1) : fp4_pair<0>(w1, s1);
            a[2 * b][r] = __builtin_amdgcn_perm(u1, u0, 0x05040100u);
            a[2 * b + 1][r] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
          }
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int n = 0; n < NP; ++n) o[d] = product(u32x4{a[d][0], a[d][1], a[d][2], a[d][3]}, p[g][n], o[d]);
    }
    load_v(next);
  }

  l += __shfl_xor(l, 32, kWave);
  if constexpr (kBase) {
    base += __shfl_xor(base, 32, kWave);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] += base;
  }
  // the waves' states: 2 and 3 into 0 and 1, then 1 into 0
  auto put = [&](int at) {
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) held[at][4 * d + g][lane] = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
    held_m[at][lane] = m;
    held_l[at][lane] = l;
  };
  auto merge = [&](int at) {
    const float om = held_m[at][lane], mn = fmaxf(m, om);
    const float c0 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
    const float c1 = om == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(om - mn);
    l = fmaf(held_l[at][lane], c1, l * c0);   // (a NaN stays one)
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 v = held[at][4 * d + g][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[d][4 * g + e] = fmaf(v[e], c1, o[d][4 * g + e] * c0);
      }
    m = mn;
  };
  const int used = c4groups + (max(kstop - own0, 0) + kGroup - 1) / kGroup;   // groups: a wave each, up to four
  if (used > 2) {
    if (wave >= 2) put(wave - 2);
    __syncthreads();
    if (wave < 2) merge(wave);
    __syncthreads();
  }
  if (used > 1) {
    if (wave == 1) put(0);
    __syncthreads();
    if (wave == 0) merge(0);
  } else {
    __syncthreads();   // (odd)
  }
  if (wave != 0) return;
  if (odd) {
#pragma unroll 1
    for (int key = own0; key < min(lim, kstop); ++key) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {   // dimensions DT (8 (r / 4) + 4 h + r % 4) .. +DT
        const T* vp = Vb + int64_t(key - nbp) * kv_ld + DT * (8 * (r / 4) + 4 * h + r % 4);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const float v = element(vp + d);
          o[d][r] += fabsf(v) < INFINITY ? 0.f : v;
        }
      }
    }
  }
  if (row0 + x >= rows) return;
  const int64_t row = int64_t(t.q0 + token) * Hq + head;
  float* pr = part + (row * splits + t.split) * (D + 2);
  const float scale = part ? 1.f : l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    typedef float vec __attribute__((ext_vector_type(DT)));
    typedef __bf16 hvec __attribute__((ext_vector_type(DT)));
    vec v;
#pragma unroll
    for (int d = 0; d < DT; ++d) v[d] = o[d][r] * scale;
    const int at = DT * (8 * (r / 4) + 4 * h + r % 4);
    if (part) {
#pragma unroll
      for (int d = 0; d < DT; d += 2) *reinterpret_cast<f32x2*>(pr + 2 + at + d) = f32x2{v[d], v[d + 1]};
    } else if constexpr (kF32) {
      *reinterpret_cast<vec*>(out + row * D + at) = v;
    } else {
      *reinterpret_cast<hvec*>(out + row * D + at) = __builtin_convertvector(v, hvec);
    }
  }
  if (h != 0) return;
  if (part) {
    *reinterpret_cast<f32x2*>(pr) = f32x2{l == 0.f ? -INFINITY : l == l ? m : l, l};   // (a NaN is kept)
    // split 0 also writes the states of the splits that no block takes
    for (int k = live; t.split == 0 && k < splits; ++k) pr[int64_t(k) * (D + 2)] = -INFINITY;
  } else if (lse) {
    lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  }
}

}  // namespace
}  // namespace rbq
