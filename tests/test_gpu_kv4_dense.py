"""Dense decode over the 4-bit cache at sizes whose blocks are planned for one round of the
GPU, against 64 bits: every head group, both head dimensions, windows in splits of their
own, splits longer than the 8-bit cache's, and calls whose windows leave no such plan."""
import math

import numpy as np
import pytest
import torch

import kv4_util as ku
from kv8_util import EPS, attention

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def R():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2606_31519_amd import rbq
    return rbq


def signed_rows(rng, B, Hkv, n, D, fmt):
    """Codes and words of K (any) and of V, whose values have one sign over every 500 rows or so, another over the next: a
    split that is lost, or weighed otherwise, moves the mean by its share."""
    K = ku.random_cache(rng, (B, Hkv, n), D, fmt)
    codes, word = ku.random_cache(rng, (B, Hkv, n), D, fmt)
    minus = rng.integers(0, 2, (B, Hkv, n // 500 + 1)).repeat(500, axis=2)[:, :, :n].astype(bool)
    if fmt == "fp4":
        codes = (codes & 7) | np.where(minus, 8, 0).astype(np.uint8)[..., None]
    else:
        s, _ = ku.parts(word)
        m = np.where(minus, -16 * s, s).astype(np.float32)          # (s has 8 bits, and so has m)
        word = (word & np.uint32(0xFFFF)) | (m.view(np.uint32) & np.uint32(0xFFFF0000))
    return K, (codes, word)


# B, Hq, Hkv, D, rows, window, its type, splits of the cached rows
CASES = [
    (2, 32, 8, 128, 20011, 300, "bf16", 53),        # 4 heads a group, windows of two splits
    (1, 128, 8, 128, 40000, 256, "f32", 90),        # 16 heads a group: 768 places
    (3, 32, 2, 64, 50001, 0, "bf16", 157),          # 16 at D = 64, no window; places that the groups do not divide
    (5, 8, 8, 128, 9000, 33, "f32", 24),            # one head a group
    (4, 16, 8, 64, 10003, 700, "bf16", 27),         # two; a window of three splits
    (1, 16, 2, 128, 200000, 4096, "bf16", 447),     # eight; the longest window, 16 splits
    (1, 2, 1, 64, 2100001, 300, "f32", 995),        # splits of 2112 rows
    (8, 8, 8, 64, 8000, 4096, "bf16", 16),          # the window's splits take the places: the 8-bit cache's plan
]


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("case", CASES, ids=[f"B{c[0]}-G{c[1] // c[2]}-D{c[3]}-n{c[4]}-w{c[5]}" for c in CASES])
def test_dense_decode_in_one_round(R, case, fmt):
    B, Hq, Hkv, D, n, w, loc, splits = case
    print("dense", case, fmt, flush=True)
    rng = np.random.default_rng(n + w)
    K, V = signed_rows(rng, B, Hkv, n, D, fmt)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    kv = dev(ku.records(K[0], V[0], fmt))
    par = dev(np.stack([K[1], V[1]], axis=-1).astype(np.uint32).view(np.int32))
    q = rng.standard_normal((B, Hq, D)).astype(np.float32)
    win = [torch.from_numpy(rng.standard_normal((B, Hkv, max(w, 1), D))).to(DT[loc]) for _ in range(2)]
    out, lse = torch.full((B, Hq, D), 9.0, device="cuda"), torch.full((B, Hq), 9.0, device="cuda")
    ws = R.workspace(R.RBQ_OP_DECODE_KV4, B, Hq, Hkv, D, n, w)
    ws.fill_(255)
    tau = 1.0 / math.sqrt(D)
    R.rbq_dense_decode_kv4(B, Hq, Hkv, D, dev(q), kv, par, R.KV4_FORMATS[fmt], n, n, *(t.cuda() for t in win), max(w, 1), w, tau,
                           out, lse, ws)
    out, lse = out.cpu().numpy(), lse.cpu().numpy()
    # a sum is a chain over the rows of a split, one over the splits, and a few joins: that many roundings of what it holds
    terms = -(-n // splits) + 64 + splits + -(-w // 256) + 64
    for b, h in {(0, 0), (B - 1, Hq - 1)}:
        val, blk = [], []
        for (c, word), x in zip((K, V), win):
            c, word, x = c[b, h // (Hq // Hkv)], word[b, h // (Hq // Hkv)], x[b, h // (Hq // Hkv), :w].double().numpy()
            val.append(np.concatenate([ku.exact_values(c, word, fmt), x]))
            blk.append(np.concatenate([ku.bulk(c, word, fmt), np.abs(x)]))
        qd = q[b, h].astype(np.float64)
        o, l = attention(qd, *val, tau)
        d = (D + 8) * EPS * float((blk[0] @ np.abs(qd)).max()) * tau      # a logit's error, as in ku.attention_tolerance
        ot = float(np.abs(val[1]).max()) * 4 * d + 2 * terms * EPS * float(blk[1].max())
        lt = d + terms * EPS + 2 * EPS * (float(np.abs(val[0] @ qd * tau).max()) + np.log(n + w))
        assert np.abs(out[b, h] - o).max() <= ot and abs(lse[b, h] - l) <= lt, (b, h, np.abs(out[b, h] - o).max(), ot,
                                                                                abs(lse[b, h] - l), lt)
