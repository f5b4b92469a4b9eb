// The host's plans of the decode over a 4-bit cache, one line per call: reads
//   B Hq Hkv D n w form      (form: 0 dense, 1 sparse; +2 with seq_n, +4 with seq_w)
// and prints
//   chunk idx_splits win_splits   of its plan
//   chunk idx_splits win_splits   of the same call over an 8-bit cache
//   the check of its arguments with a workspace of exactly the states of the larger of the two, and of
//   one byte less
//   whether its blocks are taken for one round
// Built by tests/test_kv4_plans.py with g++ from csrc/validate.cpp and this file; no HIP runtime, no GPU.
#include <algorithm>
#include <cstdint>
#include <cstdio>

#include "../../paper_2606_31519_amd/csrc/rbq_internal.h"

using namespace rbq;

int main() {
  // aligned fake device pointers: never dereferenced by the host checks
  const void* const p = reinterpret_cast<const void*>(uintptr_t(1) << 40);
  const float* const f = static_cast<const float*>(p);
  const int32_t* const i = static_cast<const int32_t*>(p);
  int B, Hq, Hkv, D, n, w, form;
  while (std::scanf("%d %d %d %d %d %d %d", &B, &Hq, &Hkv, &D, &n, &w, &form) == 7) {
    const bool sparse = form & 1, rows = form & 2, windows = form & 4;
    const DecodeSplits a = decode_kv4_splits(B, Hq, Hkv, D, n, w, sparse, rows, windows);
    const DecodeSplits b = decode_kv8_splits(B, Hkv, n, w, sparse, rows, windows);
    const size_t bytes = size_t(B) * Hq * std::max(a.total(), b.total()) * (D + 2) * sizeof(float);
    const Kv4Cache c{p, static_cast<const uint32_t*>(p), RBQ_FP4, n};
    const Kv8Window win{p, p, RBQ_BF16, w, w};
    auto check = [&](size_t have) {
      return int(check_decode_kv4(B, Hq, Hkv, D, f, c, n, sparse, i, i, win, 0.1f, f, p, have, rows ? i : nullptr,
                                  windows ? i : nullptr));
    };
    std::printf("%d %d %d %d %d %d %d %d %d\n", a.chunk, a.idx_splits, a.win_splits, b.chunk, b.idx_splits, b.win_splits,
                check(bytes), check(bytes - 1), int(kv4_one_round(B, Hq, Hkv, D, a)));
  }
  return 0;
}
