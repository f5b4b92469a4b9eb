"""rbq_prefill_attention without a GPU: argument checks, workspace sizes and the
binding's refusals."""
import pytest
import torch

FAKE = 1 << 40   # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def R():
    from paper_2606_31519_amd import rbq
    return rbq


def _call(R, **k):
    g = k.get
    return R.lib.rbq_prefill_attention(g("B", 2), g("Hq", 8), g("Hkv", 4), g("D", 128), g("q", FAKE), g("q_ld", 1024),
                                       g("K", FAKE), g("V", FAKE), g("dt", 1), g("kv_ld", 512), g("kv_head", 128),
                                       g("kv_seq", 0), g("kv_rows", 100), g("cu_q", FAKE), g("cu_k", FAKE), g("T", 100),
                                       g("max_k", 60), 1, g("tau", 0.1), g("out", FAKE), None, g("ws", None), g("wsb", 0), 0)


def test_invalid_arguments_are_rejected_on_the_host(R):
    E, U = R.RBQ_EINVAL, R.RBQ_EUNSUPPORTED
    for kw, want in [(dict(B=0), E), (dict(Hq=6), E), (dict(Hq=128), U), (dict(D=96), U), (dict(D=100), E), (dict(dt=2), U),
                     (dict(dt=16), U), (dict(T=-1), E), (dict(max_k=-1), E), (dict(kv_rows=-1), E), (dict(q_ld=1016), E),
                     (dict(q_ld=1028), E), (dict(q_ld=1 << 23), U), (dict(kv_ld=120), E), (dict(kv_ld=516), E),
                     (dict(kv_ld=1 << 23), U), (dict(kv_head=-8), E), (dict(kv_head=4), E), (dict(kv_seq=-8), E),
                     (dict(kv_seq=12), E), (dict(tau=0.0), E), (dict(tau=float("nan")), E), (dict(q=None), E),
                     (dict(q=FAKE + 8), E), (dict(K=None), E), (dict(V=FAKE + 2), E), (dict(out=None), E),
                     (dict(cu_q=None), E), (dict(cu_k=None), E), (dict(cu_q=FAKE + 4), E), (dict(T=1 << 30), U)]:
        assert _call(R, **kw) == want, kw
    assert _call(R, T=0, q=None, K=None, V=None, out=None, cu_q=None, cu_k=None) == R.RBQ_OK   # nothing to do


def test_few_rows_over_long_keys_need_a_workspace(R):
    assert R.rbq_workspace_bytes(R.RBQ_OP_PREFILL, 1, 32, 8, 128, 16000, 16000) == 0
    need = R.rbq_workspace_bytes(R.RBQ_OP_PREFILL, 1, 32, 8, 128, 131072, 5)
    assert need >= 5 * 32 * 130 * 4 * 2
    kw = dict(B=1, Hq=32, Hkv=8, q_ld=4096, kv_ld=1024, kv_rows=131072, max_k=131072, T=5)
    assert _call(R, **kw) == R.RBQ_EINVAL
    assert _call(R, **kw, ws=FAKE, wsb=need - 256) == R.RBQ_EINVAL
    assert _call(R, **kw, ws=FAKE + 8, wsb=need) == R.RBQ_EINVAL
    for a in [(0, 32, 8, 128, 100, 5), (1, 32, 0, 128, 100, 5), (1, 6, 4, 128, 100, 5), (1, 32, 8, 128, -1, 5),
              (1, 32, 8, 128, 100, 0)]:
        assert R.rbq_workspace_bytes(R.RBQ_OP_PREFILL, *a) == 0


def test_binding_refuses_short_or_mixed_buffers(R):
    T, H, D = 4, 2, 64
    x, cu = torch.zeros(T, H, D), torch.tensor([0, T], dtype=torch.int32)
    args = lambda **k: (1, H, H, D, k.get("q", x), H * D, k.get("K", x), x, H * D, D, 0, T, k.get("cu_q", cu),  # noqa: E731
                        k.get("cu_k", cu), T, T, True, 0.1, k.get("out", torch.zeros(T, H, D)),
                        k.get("lse", torch.zeros(T, H)))
    for kw in (dict(q=x.bfloat16()), dict(K=x.bfloat16()), dict(out=torch.zeros(T, H, D).bfloat16()),
               dict(out=torch.zeros(T - 1, H, D)), dict(lse=torch.zeros(T, H - 1)), dict(cu_q=cu[:1]), dict(cu_k=cu[:1])):
        with pytest.raises(ValueError):
            R.rbq_prefill_attention(*args(**kw))
    half = x.half()
    with pytest.raises(ValueError):
        R.rbq_prefill_attention(*args(q=half, K=half, out=half)[:7], half, *args(out=half)[8:])


def test_many_empty_sequences_do_not_split_the_keys_or_fill_the_grid(R):
    """One token in each of many sequences has a tile of its own: no keys are split for them; sequences without tokens
    count for nothing."""
    assert R.rbq_workspace_bytes(R.RBQ_OP_PREFILL, 1000, 4, 1, 128, 5000, 1000) == 0
    assert R.rbq_workspace_bytes(R.RBQ_OP_PREFILL, 65535, 4, 1, 128, 5000, 3) == \
        R.rbq_workspace_bytes(R.RBQ_OP_PREFILL, 3, 4, 1, 128, 5000, 3) > 0


def test_a_plan_without_tokens_enqueues_nothing(R):
    from paper_2606_31519_amd import pipeline
    plan = pipeline.PromptAttention(4, 2, 64, [0, 0], [3, 0], device="cpu")
    k = torch.zeros(3, 2, 64)
    assert plan(torch.zeros(0, 4, 64), k, k, stream=0).shape == (0, 4, 64)
    with pytest.raises(ValueError):
        pipeline.PromptAttention(4, 2, 64, [1, -1], device="cpu")
    with pytest.raises(ValueError):
        pipeline.PromptAttention(4, 2, 64, [], device="cpu")


def test_workspaces_of_every_size_are_bounded(R):
    """At most 64 splits, none without keys for them, and the same size for the same call."""
    for T in (1, 7, 40, 300, 2000):
        for k in (0, 1, 64, 65, 1000, 9001, 131072, (1 << 31) - 1):
            for Hq, Hkv, D in ((8, 8, 64), (32, 8, 128), (6, 2, 128)):
                a = R.rbq_workspace_bytes(R.RBQ_OP_PREFILL, 1, Hq, Hkv, D, k, T)
                assert a == R.rbq_workspace_bytes(R.RBQ_OP_PREFILL, 1, Hq, Hkv, D, k, T)
                assert a <= T * Hq * min(64, (k + 63) // 64) * (D + 2) * 4 + 256, (T, k, Hq)
                if k <= 64:
                    assert a == 0


def test_binding_refuses_rows_that_end_early(R):
    """q, K and V by the rows and strides that the call is given: buffers and views that end before the last row."""
    T, H, D = 4, 2, 64
    cu, out = torch.tensor([0, T], dtype=torch.int32), torch.zeros(T, H, D)
    fused, cache = torch.zeros(T, 3 * H, D), torch.zeros(2, H, T, D)

    def call(q, K, V, lay, rows=T, q_ld=H * D, B=1, tau=-1.0):
        R.rbq_prefill_attention(B, H, H, D, q, q_ld, K, V, *lay, rows, torch.zeros(B + 1, dtype=torch.int32) if B > 1 else cu,
                                cu if B == 1 else torch.zeros(B + 1, dtype=torch.int32), T, T, True, tau, out, None, stream=0)

    x, packed, held, fl = torch.zeros(T, H, D), (H * D, D, 0), (D, T * D, H * T * D), (3 * H * D, D, 0)
    views = [fused[:, i * H:(i + 1) * H] for i in range(3)]
    for kw in (dict(q=x, K=x, V=x, lay=packed), dict(q=views[0], K=views[1], V=views[2], lay=fl, q_ld=3 * H * D),
               dict(q=x, K=cache, V=cache, lay=held, B=2), dict(q=x, K=None, V=None, lay=packed, rows=0)):
        if kw["K"] is None:
            kw["K"] = kw["V"] = torch.zeros(0, H, D)
        with pytest.raises(R.RbqError) as e:      # (large enough: to the library's refusal of a negative scale)
            call(**kw)
        assert e.value.status == R.RBQ_EINVAL
    for kw in (dict(q=x[1:], K=x, V=x, lay=packed), dict(q=x, K=x[1:], V=x, lay=packed), dict(q=x, K=x, V=x[:3], lay=packed),
               dict(q=x, K=x, V=x, lay=packed, rows=T + 1), dict(q=x, K=x, V=x, lay=packed, q_ld=H * D + 8),
               dict(q=views[0][1:], K=views[1], V=views[2], lay=fl, q_ld=3 * H * D),
               dict(q=x, K=cache[:1], V=cache, lay=held, B=2), dict(q=x, K=cache, V=cache[:1].expand(2, -1, -1, -1), lay=held, B=2),
               dict(q=x, K=cache, V=cache, lay=held, B=2, rows=T + 1)):
        with pytest.raises(ValueError):
            call(**kw)


def test_a_dimension_of_one_entry_may_have_any_stride(R, monkeypatch):
    """One token, one key row, one KV head or one sequence, cut from larger tensors: their strides say nothing, and the
    call is given those of contiguous rows."""
    from paper_2606_31519_amd import pipeline
    seen = {}
    monkeypatch.setattr(R, "rbq_prefill_attention", lambda *a: seen.update(q_ld=a[5], lay=a[8:12], rows=a[11]))
    H, D = 2, 64

    def strides(q, K, V, q_lens, k_lens, Hq=4, Hkv=H):
        pipeline.PromptAttention(Hq, Hkv, D, q_lens, k_lens, device="cpu")(q, K, V, stream=0)
        return seen["q_ld"], seen["lay"]

    q1 = torch.zeros(4, 1, D).transpose(0, 1)                                # [1][4][D], strides (D, D, 1)
    far = torch.zeros(1, 1 << 16, 4, D)[:, 7]                                # [1][4][D], a row stride of 2^24
    k1 = torch.zeros(H, 1, D).transpose(0, 1)                                # [1][2][D]
    assert strides(q1, k1, k1, [1], [1]) == (4 * D, (H * D, D, 0, 1))
    assert strides(far, k1, k1.contiguous(), [1], [1]) == (4 * D, (H * D, D, 0, 1))
    c = torch.zeros(1, H, 5, D).as_strided((1, H, 5, D), (3, 5 * D, D, 1))   # one sequence
    assert strides(q1, c, torch.zeros(1, H, 5, D), [1], [5]) == (4 * D, (D, 5 * D, 0, 5))
    m = torch.zeros(5, 1, D).as_strided((5, 1, D), (D, 1, 1))                # one KV head
    assert strides(q1, m, m, [1], [5], Hkv=1) == (4 * D, (D, D, 0, 5))
    with pytest.raises(ValueError):                                          # (two heads a key apart are no such case)
        strides(q1, c, torch.zeros(1, 5, H, D).transpose(1, 2), [1], [5])


def test_a_plan_of_more_tokens_than_the_call_counts_is_refused():
    from paper_2606_31519_amd import pipeline
    for q, k in (([1 << 31], None), ([1 << 30, 1 << 30], None), ([1, 1], [1 << 30, 1 << 30])):
        with pytest.raises(ValueError, match="2\\^31"):
            pipeline.PromptAttention(4, 2, 64, q, k, device="cpu")
