"""rbq_prefill_attention: a query with an infinity is NaN, also where every logit of it is
-infinity, and 0 as any other where it sees no key; no other token is touched."""
import pytest
import torch

from test_gpu_prefill import Inputs, R  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D,qs,ks", [(4, 2, 128, [300], [300]), (4, 2, 64, [40, 9], [40, 9]),
                                            (2, 1, 128, [3], [3000]), (2, 2, 64, [20], [12])])
def test_an_infinite_query_is_nan_whatever_its_logits(R, dt, Hq, Hkv, D, qs, ks):  # noqa: F811
    print("query", dt, Hq, D, qs, ks, flush=True)
    inp = Inputs(51, dt, Hq, Hkv, D, qs, ks, "packed")
    first = max(qs[0] - ks[0], 0)                          # the first token that sees a key
    inp.K[:max(ks[0] - qs[0], 0) + 1, 0, 3] = -1.0         # its keys
    clean = [t.clone() for t in inp.run(R, True)]
    inp.q[0, 0, 3] = inp.q[first, 0, 3] = float("inf")
    out, lse = inp.run(R, True)
    assert out[first, 0].isnan().all() and lse[first, 0].isnan()
    if first > 0:
        assert torch.all(out[0, 0] == 0) and lse[0, 0] == -float("inf")
    out[first, 0], lse[first, 0] = clean[0][first, 0], clean[1][first, 0]
    assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])
