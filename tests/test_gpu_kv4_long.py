"""The 4-bit cache at its longest: 2^24 - 1 rows of 128 dimensions (one head's records end 128 bytes before 2^31, the
third head's begin past 2^32), zeros but for a few rows at both ends and between."""
import math

import numpy as np
import pytest
import torch

from paper_2606_31519_amd import pipeline, rbq as R

pytestmark = pytest.mark.gpu
H, D, N = 3, 128, (1 << 24) - 1
BLOCK = 40
STARTS = [0, (1 << 23) - 20, (1 << 24) - 1 - BLOCK]
TAU = 1.0 / math.sqrt(D)
# A lane's sum of the rows' weights has a rounding of 2^-24 per addition: one per 16 rows of a split of the decode
# (four waves, four lanes each; 341 splits), one per 8 of the chunk call's (four waves of two lanes; 64 splits). The
# weights, of logits of up to 40, are good to 40 * 2^-21.
DECODE_TOL = N / 341 / 16 * 2.0 ** -24 + 40 * 2.0 ** -21
CHUNK_TOL = N / 64 / 8 * 2.0 ** -24 + 40 * 2.0 ** -21


@pytest.fixture(scope="module", params=["fp4", "int4"])
def held(request):
    g = torch.Generator(device="cuda").manual_seed(3)
    cache = pipeline.Kv4Cache(1, H, D, N + 1, request.param)
    q = torch.randn(1, H, D, device="cuda", generator=g)
    K, V, rows = [], [], []
    for start in STARTS:
        k = q[:, :, None] * (1.2 + 0.5 * torch.rand(1, H, BLOCK, 1, device="cuda", generator=g))
        k = k + 0.1 * torch.randn(1, H, BLOCK, D, device="cuda", generator=g)
        v = torch.randn(1, H, BLOCK, D, device="cuda", generator=g)
        cache.append(k, v, BLOCK, BLOCK, start)
        small = pipeline.Kv4Cache(1, H, D, BLOCK, request.param)
        small.append(k, v, BLOCK, BLOCK, 0)
        at = slice(start, start + BLOCK)
        assert torch.equal(cache.kv4[:, :, at], small.kv4) and torch.equal(cache.par[:, :, at], small.par)
        want, got = ([torch.empty(1, H, BLOCK, D, device="cuda") for _ in "KV"] for _ in range(2))
        small.read(*want, BLOCK, BLOCK)
        cache.read(*got, BLOCK, BLOCK, start)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        K.append(want[0]), V.append(want[1]), rows.append(torch.arange(start, start + BLOCK, device="cuda"))
    yield cache, q, torch.cat(K, 2)[0].double(), torch.cat(V, 2)[0].double(), torch.cat(rows)
    del cache
    torch.cuda.empty_cache()


def answer(q, K, V, zeros):
    """Attention of queries q [n][D] over rows K, V and `zeros` rows of zeros: out, its scale (the weighted mean of |V|), lse."""
    s = q.double() @ K.T * TAU
    top = torch.clamp(s.amax(1), min=0.0)
    p = torch.exp(s - top[:, None])
    tot = p.sum(1) + zeros * torch.exp(-top)
    return p @ V / tot[:, None], p @ V.abs() / tot[:, None], top + torch.log(tot)


def check(out, lse, want, tol, rounding=0.0):
    o, scale, l = want
    assert torch.all((out.double() - o).abs() <= (2 * tol + rounding) * scale), ((out.double() - o).abs() / scale).max()
    assert torch.all((lse.double() - l).abs() <= tol), (lse.double() - l).abs().max()


def decode(cache, q, n, w, sel=None, seqs=(None, None)):
    out, lse = torch.empty(1, H, D, device="cuda"), torch.empty(1, H, device="cuda")
    ws = R.workspace(R.RBQ_OP_DECODE_KV4, 1, H, H, D, n, w)
    ws.fill_(255)
    loc = (None, None, 0, w, TAU)
    if sel is None:
        R.rbq_dense_decode_kv4(1, H, H, D, q, cache.kv4, cache.par, cache.code, cache.cap, n, *loc, out, lse, ws, *seqs)
    else:
        R.rbq_sparse_decode_kv4(1, H, H, D, q, cache.kv4, cache.par, cache.code, cache.cap, n, *sel, *loc, out, lse, ws, *seqs)
    return out[0], lse[0]


def by_head(q, K, V, zeros):
    parts = [answer(q[:, h], K[h], V[h], zeros) for h in range(H)]
    return tuple(torch.cat([p[i] for p in parts]) for i in range(3))


@pytest.mark.parametrize("ragged", [False, True])
def test_every_row(held, ragged):
    cache, q, K, V, rows = held
    seqs = tuple(torch.tensor([v], dtype=torch.int32, device="cuda") for v in (N, 0)) if ragged else (None, None)
    check(*decode(cache, q, N, 0, seqs=seqs), by_head(q, K, V, N - len(rows)), DECODE_TOL)


def test_a_selection(held):
    cache, q, K, V, rows = held
    step = 16001
    idx = torch.unique(torch.cat([rows, torch.arange(0, N, step, device="cuda")])).int()
    sel = torch.zeros(1, H, N, dtype=torch.int32, device="cuda")
    sel[:, :, :len(idx)] = idx
    cnt = torch.full((1, H), len(idx), dtype=torch.int32, device="cuda")
    check(*decode(cache, q, N, 0, (sel, cnt)), by_head(q, K, V, len(idx) - len(rows)), DECODE_TOL)


@pytest.mark.parametrize("tokens,dt", [(3, torch.float32), (600, torch.float32), (5, torch.bfloat16), (600, torch.bfloat16)])
def test_a_chunk(held, tokens, dt):
    cache, q, K, V, rows = held
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(3, tokens, H, D, device="cuda", generator=g)
    x[0] = q * (0.9 + 0.2 * torch.rand(tokens, 1, 1, device="cuda", generator=g))
    x[1] = 0.3 * x[1] + q
    x = x.to(dt)
    # bf16: each probability, int4's cached values and the result are off by up to half a step
    rounding = 3 * 2.0 ** -8 if dt == torch.bfloat16 else 0.0
    lse = torch.empty(tokens, H, device="cuda")
    out = pipeline.ChunkAttention(H, cache, [tokens], [N])(x[0], x[1], x[2], lse=lse)
    for i in (0, 1, tokens - 1):
        for h in range(H):
            Kh, Vh = (torch.cat([a[h], b[:i + 1, h].double()]) for a, b in ((K, x[1]), (V, x[2])))
            check(out[i:i + 1, h], lse[i:i + 1, h], answer(x[0][i:i + 1, h], Kh, Vh, N - len(rows)), CHUNK_TOL, rounding)
