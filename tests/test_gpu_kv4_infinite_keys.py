"""Infinities among a chunk's own keys and queries (rbq_prefill_attention_kv4): a key with
one has the logits that IEEE arithmetic gives it, so that a logit of -infinity is a weight
of 0 and one of +infinity, or the product of an infinity with 0, is NaN in its head; a
query with one is NaN. Alike in the kernels of few rows and of tiles, for either type."""
import numpy as np
import pytest
import torch

import kv4_util as ku
from test_gpu_kv4_chunk import Inputs, R  # noqa: F401

pytestmark = pytest.mark.gpu

# dtype, D, tokens, cached rows: few rows over long keys (split), few over short ones, whole tiles (fp32: mostly own keys)
CASES = [("f32", 64, [6], [2000]), ("f32", 128, [40, 6], [70, 33]), ("f32", 64, [1200], [70]), ("f32", 128, [1100], [40]),
         ("bf16", 128, [6], [2000]), ("bf16", 64, [600], [70])]
IDS = [f"{c[0]}-D{c[1]}-q{max(c[2])}-n{max(c[3])}" for c in CASES]


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_an_infinite_key_has_the_logits_of_its_sign(R, case, fmt):  # noqa: F811
    dt, D, qs, ns = case
    print("key", case, fmt, flush=True)
    inp = Inputs(41, fmt, dt, 4, 2, D, qs, ns)
    at, end = inp.cu[-1] - 5, inp.cu[-1]                   # the fifth last token's key, seen by five
    col = 7
    for t in range(at, end):                                # signs of the queries' places for it, one of them 0
        mag = inp.q[t, :, col].abs().clamp(min=0.25)
        inp.q[t, 0, col], inp.q[t, 1, col] = mag[0] * (-1) ** t, -mag[1]
    inp.q[end - 1, 0, col] = 0.0
    inp.q[at + 2] = inp.q[at + 2].to(torch.bfloat16).to(inp.q.dtype)      # (of 8 bits: their further parts are zeros)
    clean = [t.clone() for t in inp.run(R, True)]
    for value in (float("inf"), float("-inf")):
        inp.K[at, 0, col] = value
        out, lse = (t.double().cpu().numpy() for t in inp.run(R, True))
        seen = np.zeros(lse.shape, bool)
        seen[at:end, :2] = True
        assert np.array_equal(out[~seen], clean[0].double().cpu().numpy()[~seen])
        assert np.array_equal(lse[~seen], clean[1].double().cpu().numpy()[~seen])
        b, nb = len(ns) - 1, ns[-1]
        first = inp.cu[b]
        own = [t[first:end, 0].double().cpu().numpy() for t in (inp.K, inp.V)]
        val, blk = [], []
        for k, x in zip("KV", own):
            c, w = (t[b, 0][:nb] for t in inp.code[k])
            val.append(np.concatenate([ku.exact_values(c, w, fmt), x]))
            blk.append(np.concatenate([ku.bulk(c, w, fmt), np.abs(x)]))
        for t in range(at, end):
            for h in (0, 1):
                q = inp.q[t, h].double().cpu().numpy()
                if not q[col] * np.sign(value) < 0:
                    assert np.isnan(out[t, h]).all() and np.isnan(lse[t, h]), (t, h, q[col])
                    continue
                keys = [i for i in range(nb + t - first + 1) if i != nb + at - first]
                S = val[0][keys] @ q * inp.tau
                p = np.exp(S - S.max())
                want, wl = p @ val[1][keys] / p.sum(), S.max() + np.log(p.sum())
                ot, lt = ku.attention_tolerance(q, val[0][keys], val[1][keys], blk[0][keys], blk[1][keys], inp.tau)
                if dt == "bf16":      # half a step of each probability, cached value and output
                    ot = ot + 2.0 ** -8 * ((2 if fmt == "int4" else 1) * (p @ np.abs(val[1][keys])) / p.sum() + np.abs(want))
                assert np.all(np.abs(out[t, h] - want) <= ot) and abs(lse[t, h] - wl) <= lt, (t, h, q[col])


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_an_infinite_query_is_nan_whatever_its_logits(R, case, fmt):  # noqa: F811
    """Also where the only key that it sees has a logit of -infinity."""
    dt, D, qs, ns = case
    print("query", case, fmt, flush=True)
    for rows in (ns, [0] * len(ns)):
        inp = Inputs(43, fmt, dt, 4, 2, D, qs, rows, cap=max(ns) + 3)
        inp.K[0, 0, 3] = -1.0
        clean = [t.clone() for t in inp.run(R, True)]
        inp.q[0, 1, 3] = float("inf")
        out, lse = inp.run(R, True)
        assert out[0, 1].isnan().all() and lse[0, 1].isnan()
        out[0, 1], lse[0, 1] = clean[0][0, 1], clean[1][0, 1]
        assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])
