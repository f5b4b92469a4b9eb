"""The 4-bit cache's calls without a GPU: argument checks on the host, workspace
sizes, the Python binding's refusals, and the tests' own model of the formats."""
import numpy as np
import pytest
import torch

import kv4_util as ku

FAKE = 1 << 40   # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def R():
    from paper_2606_31519_amd import rbq
    return rbq


def _rows(R, back=False, **k):
    g = k.get
    if back:
        return R.lib.rbq_dequantize_kv4(g("B", 1), g("H", 2), g("D", 128), g("kv", FAKE), g("par", FAKE), g("fmt", 32),
                                        g("cap", 100), g("n", 10), g("off", 0), g("K", FAKE), FAKE, g("dt", 1), g("ld", 10),
                                        g("so", None), g("sn", None), 0)
    return R.lib.rbq_quantize_kv4(g("B", 1), g("H", 2), g("D", 128), g("K", FAKE), FAKE, g("dt", 1), g("ld", 10), g("n", 10),
                                  g("off", 0), g("cap", 100), g("fmt", 32), g("kv", FAKE), g("par", FAKE), g("so", None),
                                  g("sn", None), 0)


@pytest.mark.parametrize("back", [False, True])
def test_cache_writes_and_reads_reject_invalid_arguments(R, back):
    E, U = R.RBQ_EINVAL, R.RBQ_EUNSUPPORTED
    for kw, want in [(dict(B=0), E), (dict(H=0), E), (dict(D=96), U), (dict(D=100), E), (dict(dt=2), U), (dict(dt=32), U),
                     (dict(fmt=16), U), (dict(fmt=34), U), (dict(n=-1), E), (dict(off=-1), E), (dict(off=91), E),
                     (dict(ld=9), E), (dict(ld=1 << 31), E), (dict(cap=9), E), (dict(K=None), E), (dict(K=FAKE + 8), E),
                     (dict(kv=None), E), (dict(kv=FAKE + 4), E), (dict(par=None), E), (dict(par=FAKE + 8), E),
                     (dict(so=FAKE + 4), E), (dict(sn=FAKE + 8), E), (dict(cap=(1 << 31) - 1, off=1 << 24), E),
                     (dict(B=65536), E)]:
        assert _rows(R, back, **kw) == want, kw
    assert _rows(R, back, n=0, K=None, kv=None, par=None) == R.RBQ_OK   # no rows: nothing read, nothing enqueued


def _decode(R, sparse, **k):
    g = k.get
    sel = (g("sel", FAKE), g("cnt", FAKE)) if sparse else ()
    fn = R.lib.rbq_sparse_decode_kv4 if sparse else R.lib.rbq_dense_decode_kv4
    return fn(g("B", 1), g("Hq", 8), g("Hkv", 4), g("D", 128), g("q", FAKE), g("kv", FAKE), g("par", FAKE), g("fmt", 33),
              g("cap", 100), g("n", 100), *sel, g("kl", FAKE), FAKE, g("ldt", 1), g("ld", 20), g("w", 10), g("tau", 0.1),
              g("out", FAKE), None, g("ws", FAKE), g("wsb", 1 << 30), g("sn", None), g("sw", None), 0)


@pytest.mark.parametrize("sparse", [False, True])
def test_attention_rejects_invalid_arguments(R, sparse):
    E, U = R.RBQ_EINVAL, R.RBQ_EUNSUPPORTED
    cases = [(dict(B=0), E), (dict(Hq=6), E), (dict(Hq=12), U), (dict(Hq=128), U), (dict(D=96), U), (dict(fmt=17), U),
             (dict(fmt=0), U), (dict(n=101), E), (dict(n=-1), E), (dict(cap=99), E), (dict(w=5000, ld=5000), E),
             (dict(w=21), E), (dict(w=-1), E), (dict(kl=None), E), (dict(kl=FAKE + 2), E), (dict(ldt=32), U),
             (dict(tau=0.0), E), (dict(tau=float("nan")), E), (dict(tau=float("inf")), E), (dict(q=None), E),
             (dict(kv=None), E), (dict(par=None), E), (dict(par=FAKE + 4), E), (dict(out=None), E), (dict(ws=None), E),
             (dict(wsb=64), E), (dict(sn=FAKE + 4), E), (dict(sw=FAKE + 4), E), (dict(n=1 << 24, cap=1 << 24), E),
             (dict(B=60000, Hq=4, Hkv=1, n=400000, cap=400000, sn=FAKE, wsb=1 << 62), U)]   # 2^24 blocks and more
    if sparse:
        cases += [(dict(sel=None), E), (dict(cnt=None), E), (dict(sel=FAKE + 4), E)]
    for kw, want in cases:
        assert _decode(R, sparse, **kw) == want, kw


def test_the_fused_step_rejects_invalid_arguments(R):
    E, U = R.RBQ_EINVAL, R.RBQ_EUNSUPPORTED

    def step(**k):
        g = k.get
        return R.lib.rbq_decode_step_kv4(
            1, g("Hq", 8), 4, g("D", 128), FAKE, g("P", FAKE), g("c_q", None), FAKE, g("kv", FAKE), g("par", FAKE),
            g("fmt", 32), g("cap", 200), g("n", 100), g("kl", FAKE), FAKE, g("ldt", 1), g("ld", 16), g("w", 10), FAKE,
            g("kf", FAKE), g("kf16", None), g("flush", 1), g("p", 0.9), 0.1, FAKE, FAKE, FAKE, g("sel", FAKE), FAKE, FAKE, None,
            FAKE, g("wsb", 1 << 30), 0)

    for kw, want in [(dict(kf=None), E), (dict(kf16=FAKE), E), (dict(kf=None, kf16=FAKE, c_q=FAKE), E),
                     (dict(kf=None, kf16=FAKE + 2), E), (dict(cap=105), E), (dict(n=-1), E), (dict(n=201), E), (dict(w=-1), E),
                     (dict(w=17), E), (dict(kl=None), E), (dict(ldt=7), U), (dict(fmt=16), U), (dict(D=96), U),
                     (dict(Hq=12), U), (dict(p=0.0), E), (dict(P=None), E), (dict(kv=None), E), (dict(par=None), E),
                     (dict(sel=None), E), (dict(wsb=64), E)]:
        assert step(**kw) == want, kw
    assert R.rbq_workspace_bytes(R.RBQ_OP_DECODE_STEP_KV4, 1, 6, 4, 128, 4000, 64) == 0


def test_chunks_reject_invalid_arguments(R):
    E, U = R.RBQ_EINVAL, R.RBQ_EUNSUPPORTED

    def chunk(**k):
        g = k.get
        return R.lib.rbq_prefill_attention_kv4(
            g("B", 2), g("Hq", 6), g("Hkv", 2), g("D", 128), g("q", FAKE), g("qld", 768), g("K", FAKE), FAKE, g("dt", 1),
            g("ld", 256), g("head", 128), g("cu", FAKE), g("T", 9), g("kv", FAKE), g("par", FAKE), g("fmt", 32), g("cap", 500),
            g("n", 400), g("sn", None), 1, g("tau", 0.1), g("out", FAKE), None, g("ws", FAKE), g("wsb", 1 << 40), 0)

    for kw, want in [(dict(B=0), E), (dict(Hq=5), E), (dict(Hq=34), U), (dict(D=96), U), (dict(dt=2), U), (dict(fmt=16), U),
                     (dict(T=-1), E), (dict(n=-1), E), (dict(n=501), E), (dict(cap=-1), E), (dict(qld=760), E),
                     (dict(qld=769), E), (dict(qld=1 << 23), U), (dict(ld=120), E), (dict(ld=257), E), (dict(ld=1 << 23), U),
                     (dict(head=-128), E), (dict(head=100), E), (dict(tau=0.0), E), (dict(tau=float("nan")), E),
                     (dict(q=None), E), (dict(K=None), E), (dict(cu=None), E), (dict(kv=None), E), (dict(par=None), E),
                     (dict(par=FAKE + 8), E), (dict(sn=FAKE + 4), E), (dict(out=None), E), (dict(out=FAKE + 8), E),
                     (dict(n=1 << 24, cap=1 << 24), E), (dict(T=(1 << 31) - 200), U), (dict(T=1, B=1, n=400000, cap=400000, ws=None), E),
                     (dict(T=1, B=1, n=400000, cap=400000, wsb=64), E)]:
        assert chunk(**kw) == want, kw
    assert chunk(T=0, q=None, K=None, cu=None, out=None, ws=None) == R.RBQ_OK   # no tokens: nothing enqueued


def test_workspaces_cover_every_form_and_every_shorter_window(R):
    rng = np.random.default_rng(4)
    cases = [(1, 8, 128, 0, 0), (1, 8, 128, 130816, 256), (16, 8, 128, 32512, 256), (64, 8, 64, 200, 4096)]
    cases += [(int(2 ** rng.uniform(0, 6)), int(2 ** rng.integers(0, 4)), int(rng.choice([64, 128])),
               int(np.exp(rng.uniform(0, np.log(900000)))), int(rng.integers(0, 4097))) for _ in range(300)]
    for B, Hkv, D, n, w in cases:
        size = lambda op, m: R.rbq_workspace_bytes(op, B, 4 * Hkv, Hkv, D, n, m)  # noqa: E731
        assert size(R.RBQ_OP_DECODE_KV4, w) >= size(R.RBQ_OP_DENSE_DECODE, w) > 0
        for op in (R.RBQ_OP_DECODE_KV4, R.RBQ_OP_DECODE_STEP_KV4):
            need = [size(op, m) for m in sorted({0, min(1, w), *range(256, w, 256), w})]
            assert need == sorted(need)
        # the calls' own checks pass with it, whatever the form (sm_scale refuses them afterwards): dense, ragged, sparse
        ws = size(R.RBQ_OP_DECODE_KV4, w)
        for sparse in (False, True):
            for sn, sw in ((None, None), (FAKE, None), (None, FAKE), (FAKE, FAKE)):
                kw = dict(B=B, Hq=4 * Hkv, Hkv=Hkv, D=D, n=n, cap=max(n, 1), w=w, ld=w + 1, sn=sn, sw=sw)
                if n * D < 1 << 31:
                    assert _decode(R, sparse, wsb=ws // 8, **kw) == R.RBQ_EINVAL
    assert R.rbq_workspace_bytes(R.RBQ_OP_DECODE_KV4, 1, 32, 8, 128, -1, 0) == 0
    assert R.rbq_workspace_bytes(R.RBQ_OP_PREFILL_KV4, 1, 32, 8, 128, 100, 0) == 0
    assert R.rbq_workspace_bytes(R.RBQ_OP_PREFILL_KV4, 1, 32, 8, 128, (1 << 31) - 1, 100) == 0
    assert R.rbq_workspace_bytes(R.RBQ_OP_PREFILL_KV4, 1, 32, 8, 128, 100000, 3) > 0


def test_binding_refuses_short_or_mixed_buffers(R):
    B, H, D, cap = 1, 2, 64, 64
    kv, par = torch.zeros(B, H, cap, D, dtype=torch.uint8), torch.zeros(B, H, cap, 2, dtype=torch.int32)
    x, F = torch.zeros(B, H, 4, D), R.RBQ_FP4
    bad = [lambda: R.rbq_quantize_kv4(B, H, D, x, x, 4, 4, 0, cap, F, kv.view(torch.int8), par),      # other types
           lambda: R.rbq_quantize_kv4(B, H, D, x, x, 4, 4, 0, cap, F, kv, par.float()),
           lambda: R.rbq_quantize_kv4(B, H, D, x, x.bfloat16(), 4, 4, 0, cap, F, kv, par),
           lambda: R.rbq_quantize_kv4(B, H, D, x.half(), x.half(), 4, 4, 0, cap, F, kv, par),
           lambda: R.rbq_quantize_kv4(B, H, D, x, x, 5, 5, 0, cap, F, kv, par),                       # fewer rows
           lambda: R.rbq_quantize_kv4(B, H, D, x, x, 4, 4, 0, cap, F, kv[..., :32], par),
           lambda: R.rbq_quantize_kv4(B, H, D, x, x, 4, 4, 0, cap, F, kv, par[..., :1]),
           lambda: R.rbq_quantize_kv4(2, H, D, x, x, 4, 4, 0, cap, F, kv, par),
           lambda: R.rbq_dequantize_kv4(B, H, D, kv, par, F, cap, 8, 0, x, x, 8),
           lambda: R.rbq_dequantize_kv4(B, H, D, kv, par, F, cap, 4, 0, x, x, 4, par.view(-1)[:0])]
    q, out, lse, ws = torch.zeros(B, 4, D), torch.zeros(B, 4, D), torch.zeros(B, 4), torch.zeros(1 << 16, dtype=torch.uint8)
    sel = torch.zeros(B, 4, cap - 1, dtype=torch.int32)
    bad += [lambda: R.rbq_dense_decode_kv4(B, 4, H, D, q, kv, par, F, cap, cap, x, x, 5, 5, 0.1, out, lse, ws),
            lambda: R.rbq_dense_decode_kv4(B, 4, H, D, q, kv, par, F, cap, cap, x, x.bfloat16(), 4, 4, 0.1, out, lse, ws),
            lambda: R.rbq_dense_decode_kv4(B, 4, H, D, q[:, :3], kv, par, F, cap, cap, x, x, 4, 4, 0.1, out, lse, ws),
            lambda: R.rbq_dense_decode_kv4(B, 4, H, D, q, kv, par, F, cap + 1, cap, x, x, 4, 4, 0.1, out, lse, ws),
            lambda: R.rbq_sparse_decode_kv4(B, 4, H, D, q, kv, par, F, cap, cap, sel, sel[:, :, 0].contiguous(), None, None, 0,
                                            0, 0.1, out, lse, ws)]
    t, cu = torch.zeros(6, 4, D), torch.zeros(2, dtype=torch.int32)
    y = torch.zeros(6, H, D)
    chunk = lambda q=t, K=y, V=y, c=kv, p=par, cu=cu, o=t, T=6: R.rbq_prefill_attention_kv4(  # noqa: E731
        B, 4, H, D, q, 4 * D, K, V, H * D, D, cu, T, c, p, F, cap, cap, None, True, 0.1, o, None)
    bad += [lambda: chunk(q=t[:5]), lambda: chunk(K=y[:5]), lambda: chunk(V=y.bfloat16()), lambda: chunk(q=t.bfloat16()),
            lambda: chunk(o=t[:5]), lambda: chunk(cu=cu[:1]), lambda: chunk(c=kv[:, :, :60]), lambda: chunk(p=par.long())]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print(i)


def test_pipeline_objects_refuse_what_they_cannot_hold():
    from paper_2606_31519_amd import pipeline
    with pytest.raises(ValueError):
        pipeline.Kv4Cache(1, 2, 64, 32, fmt="e4m3", device="cpu")
    c = pipeline.Kv4Cache(2, 2, 64, 32, device="cpu")
    for q, n in (([1], [2]), ([1, 2], [3]), ([1, -1], [2, 2]), ([1, 1], [2, 33]), ([1 << 30, 1 << 30], [1, 1])):
        with pytest.raises(ValueError):
            pipeline.ChunkAttention(4, c, q, n)
    att = pipeline.ChunkAttention(4, c, [3, 5], [32, 0])
    q, K = torch.zeros(8, 4, 64), torch.zeros(8, 2, 64)
    for bad in ((q[:7], K, K), (q[:, :2], K, K), (q, K[:7], K[:7]), (q, K, K[:, :, :32]), (q, torch.zeros(8, 4, 64), K),
                (q, K, torch.zeros(8, 4, 64)[:, :2]), (q.transpose(1, 2).contiguous().transpose(1, 2), K, K)):
        with pytest.raises(ValueError):
            att(*bad)
    K = torch.zeros(1, 2, 40, 64)
    for kw in (dict(kv4="fp4"), dict(kv4="int4")):      # fewer rows than the prefill
        with pytest.raises(ValueError):
            pipeline.DecodeSession(1, 4, 2, 64, 100, 50, 16, K, K, torch.eye(64), device="cpu", **kw)
    with pytest.raises(ValueError, match="not both"):
        pipeline.DecodeSession(1, 4, 2, 64, 100, 30, 16, K, K, torch.eye(64), device="cpu", kv8="int8", kv4="fp4")


def test_the_models_fp4_and_int4():
    """The element-by-element model against the formats' own properties: every value in range within half a step, codes of
    representable values exact, ties to even."""
    rng = np.random.default_rng(6)
    for D in (64, 128):
        for _ in range(50):
            x = (rng.standard_normal(D) * np.exp(rng.uniform(-20, 20))).astype(np.float32).astype(np.float64)
            c, w = ku.encode_row(x, "fp4")
            v = ku.row_values(c, np.array(w), "fp4")
            s = 2.0 ** (np.array([(w >> 8 * g) & 255 for g in range(4)]) - 127.0).repeat(D // 4)
            assert np.all(np.abs(v - x) <= np.maximum(s * np.where(np.abs(x) > 4 * s, 1.0, 0.5), 0))
            c, w = ku.encode_row(x, "int4")
            step, base = (float(t) for t in ku.parts(np.array(w)))
            assert base <= x.min() and base + 15 * step >= x.max() * (1 - 2.0 ** -23)
            assert np.all(np.abs(ku.exact_values(c, np.array(w), "int4") - x) <= step * (0.5 + 2.0 ** -18) + 2.0 ** -23 * np.abs(x).max())
        assert np.array_equal(ku.unpack(ku.pack(c[None], "int4"), "int4")[0], c)
    ties = np.resize([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], 64)
    assert np.array_equal(ku.row_values(*[np.asarray(t) for t in ku.encode_row(ties, "fp4")], "fp4"),
                          np.resize([0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0], 64))
