"""pipeline.ChunkAttention takes K and V whose strides differ only where they have one entry, as
pipeline.PromptAttention does: a single token, or a single head, cut from larger tensors."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hkv,q_lens", [(2, [1]), (1, [5, 3]), (1, [1]), (2, [0, 1])])
def test_strides_of_single_tokens_and_heads(Hkv, q_lens):
    from paper_2606_31519_amd import pipeline
    Hq, D, B, T = 4, 64, len(q_lens), sum(q_lens)
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    cache = pipeline.Kv4Cache(B, Hkv, D, 40, "int4")
    cache.append(rnd(B, Hkv, 40, D), rnd(B, Hkv, 40, D), 40, 40, 0)
    plan = pipeline.ChunkAttention(Hq, cache, q_lens, [40] * B)
    x = rnd(T, Hq + 2 * Hkv, D)
    own = lambda t: torch.empty(t.shape, dtype=t.dtype, device="cuda").copy_(t)  # noqa: E731
    q, K, V = x[:, :Hq], x[:, Hq:Hq + Hkv], own(x[:, Hq + Hkv:])
    want = plan(own(q), own(K), V)
    if T == 1:                       # a token of a fused projection beside one of its own
        assert K.stride() != V.stride() and torch.equal(plan(q, K, V), want)
    if Hkv == 1:                     # a head that is one of several, its rows as far apart as the other's
        rows = torch.zeros(T, 3, D, device="cuda", dtype=x.dtype)
        rows[:, 1:2] = K
        other = torch.zeros(T, 3 * D, device="cuda", dtype=x.dtype)
        other[:, D:2 * D] = V[:, 0]
        one = other[:, None, D:2 * D]           # (strides 3 D, 3 D, 1, the other's 3 D, D, 1)
        assert rows[:, 1:2].stride() != one.stride() and torch.equal(plan(own(q), rows[:, 1:2], one), want)
    if T > 1:
        with pytest.raises(ValueError, match="strides"):
            plan(own(q), K, V)
