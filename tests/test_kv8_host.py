"""The 8-bit cache's calls without a GPU: argument checks on the host, workspace
sizes, the Python binding's refusals, and the tests' own model of the formats."""
import numpy as np
import pytest
import torch

import kv8_util as ku

FAKE = 1 << 40   # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def R():
    from paper_2606_31519_amd import rbq
    return rbq


def _quant(R, back=False, **k):
    g = k.get
    if back:
        return R.lib.rbq_dequantize_kv(g("B", 1), g("H", 2), g("D", 128), g("K8", FAKE), FAKE, g("fmt", 16), g("block", 64),
                                       g("ks", FAKE), FAKE, g("cap", 100), g("n", 10), g("off", 0), g("K", FAKE), FAKE,
                                       g("dt", 1), g("ld", 10), g("so", None), g("sn", None), 0)
    return R.lib.rbq_quantize_kv(g("B", 1), g("H", 2), g("D", 128), g("K", FAKE), FAKE, g("dt", 1), g("ld", 10),
                                 g("n", 10), g("off", 0), g("cap", 100), g("block", 64), g("fmt", 16), g("K8", FAKE), FAKE,
                                 g("ks", FAKE), FAKE, g("so", None), g("sn", None), 0)


@pytest.mark.parametrize("back", [False, True])
def test_cache_writes_and_reads_reject_invalid_arguments(R, back):
    E, U = R.RBQ_EINVAL, R.RBQ_EUNSUPPORTED
    for kw, want in [(dict(B=0), E), (dict(H=0), E), (dict(D=96), U), (dict(D=100), E), (dict(dt=2), U), (dict(dt=16), U),
                     (dict(fmt=1), U), (dict(fmt=18), U), (dict(block=0), E), (dict(block=-16), E), (dict(block=48), E),
                     (dict(block=8), U), (dict(block=512), U), (dict(n=-1), E), (dict(off=-1), E), (dict(off=91), E),
                     (dict(ld=9), E), (dict(ld=1 << 31), E), (dict(cap=9), E), (dict(K=None), E), (dict(K=FAKE + 8), E),
                     (dict(K8=None), E), (dict(K8=FAKE + 4), E), (dict(ks=None), E), (dict(so=FAKE + 4), E),
                     (dict(sn=FAKE + 8), E), (dict(cap=(1 << 31) - 1, off=1 << 24), E), (dict(B=65536), E)]:
        assert _quant(R, back, **kw) == want, kw
    assert _quant(R, back, n=0, K=None, K8=None, ks=None) == R.RBQ_OK   # no rows: nothing read, nothing enqueued


def _decode(R, sparse, **k):
    g = k.get
    sel = (g("sel", FAKE), g("cnt", FAKE)) if sparse else ()
    fn = R.lib.rbq_sparse_decode_kv8 if sparse else R.lib.rbq_dense_decode_kv8
    return fn(g("B", 1), g("Hq", 8), g("Hkv", 4), g("D", 128), g("q", FAKE), g("K8", FAKE), FAKE, g("fmt", 17),
              g("block", 32), g("ks", FAKE), FAKE, g("cap", 100), g("n", 100), *sel, g("kl", FAKE), FAKE, g("ldt", 1),
              g("ld", 20), g("w", 10), g("tau", 0.1), g("out", FAKE), None, g("ws", FAKE), g("wsb", 1 << 30),
              g("sn", None), g("sw", None), 0)


@pytest.mark.parametrize("sparse", [False, True])
def test_attention_rejects_invalid_arguments(R, sparse):
    E, U = R.RBQ_EINVAL, R.RBQ_EUNSUPPORTED
    cases = [(dict(B=0), E), (dict(Hq=6), E), (dict(Hq=12), U), (dict(Hq=128), U), (dict(D=96), U), (dict(fmt=0), U),
             (dict(block=24), E), (dict(block=1024), U), (dict(n=101), E), (dict(n=-1), E), (dict(cap=99), E),
             (dict(w=5000, ld=5000), E), (dict(w=21), E), (dict(w=-1), E), (dict(kl=None), E), (dict(kl=FAKE + 2), E),
             (dict(ldt=16), U), (dict(tau=0.0), E), (dict(tau=float("nan")), E), (dict(tau=float("inf")), E),
             (dict(q=None), E), (dict(K8=None), E), (dict(ks=None), E), (dict(ks=FAKE + 4), E), (dict(out=None), E),
             (dict(ws=None), E), (dict(wsb=64), E), (dict(sn=FAKE + 4), E), (dict(sw=FAKE + 4), E),
             (dict(n=1 << 24, cap=1 << 24), E)]
    if sparse:
        cases += [(dict(sel=None), E), (dict(cnt=None), E), (dict(sel=FAKE + 4), E)]
    for kw, want in cases:
        assert _decode(R, sparse, **kw) == want, kw


def test_other_calls_do_not_take_the_8_bit_formats(R):
    st = R.lib.rbq_dense_decode(1, 8, 4, 128, FAKE, FAKE, FAKE, R.RBQ_E4M3, 100, 100, None, None, 0, 0, 0.1, FAKE, None,
                                FAKE, 1 << 30, 0)
    assert st == R.RBQ_EUNSUPPORTED


def test_workspace_covers_every_form_of_the_call(R):
    """One size serves dense, sparse and ragged calls: at least that of the full-precision call's splits."""
    for B, n, w in [(1, 0, 0), (1, 1, 0), (1, 0, 5), (1, 4000, 129), (1, 130816, 256), (16, 32512, 256), (64, 200, 4096)]:
        a = R.rbq_workspace_bytes(R.RBQ_OP_DECODE_KV8, B, 32, 8, 128, n, w)
        assert a >= R.rbq_workspace_bytes(R.RBQ_OP_DENSE_DECODE, B, 32, 8, 128, n, w) > 0
    assert R.rbq_workspace_bytes(R.RBQ_OP_DECODE_KV8, 1, 32, 8, 128, -1, 0) == 0


def test_binding_refuses_short_or_mixed_buffers(R):
    B, H, D, cap, block = 1, 2, 64, 64, 16
    i8 = torch.zeros(B, H, cap, D, dtype=torch.int8)
    e4 = torch.zeros(B, H, cap, D, dtype=torch.float8_e4m3fn)
    s = torch.zeros(B, H, cap // block)
    x = torch.zeros(B, H, 4, D)
    with pytest.raises(ValueError):    # two formats
        R.rbq_quantize_kv(B, H, D, x, x, 4, 4, 0, cap, block, i8, e4, s, s)
    with pytest.raises(ValueError):    # scales for fewer blocks
        R.rbq_quantize_kv(B, H, D, x, x, 4, 4, 0, cap, block, i8, i8, s[:, :, :3], s)
    with pytest.raises(ValueError):    # fewer source rows
        R.rbq_quantize_kv(B, H, D, x, x, 5, 5, 0, cap, block, i8, i8, s, s)
    with pytest.raises(ValueError):    # two source types
        R.rbq_quantize_kv(B, H, D, x, x.bfloat16(), 4, 4, 0, cap, block, i8, i8, s, s)
    with pytest.raises(ValueError):    # no 8-bit type
        R.rbq_quantize_kv(B, H, D, x, x, 4, 4, 0, cap, block, x, x, s, s)
    with pytest.raises(ValueError):    # outputs of fewer rows
        R.rbq_dequantize_kv(B, H, D, i8, i8, block, s, s, cap, 8, 0, x, x, 8)
    q, out, lse, ws = torch.zeros(B, 4, D), torch.zeros(B, 4, D), torch.zeros(B, 4), torch.zeros(1 << 16, dtype=torch.uint8)
    with pytest.raises(ValueError):    # a window of fewer rows
        R.rbq_dense_decode_kv8(B, 4, H, D, q, i8, i8, block, s, s, cap, cap, x, x, 5, 5, 0.1, out, lse, ws)
    with pytest.raises(ValueError):    # a selection of fewer entries
        R.rbq_sparse_decode_kv8(B, 4, H, D, q, i8, i8, block, s, s, cap, cap, torch.zeros(B, 4, cap - 1, dtype=torch.int32),
                                torch.zeros(B, 4, dtype=torch.int32), None, None, 0, 0, 0.1, out, lse, ws)


def test_the_models_e4m3_is_the_ocp_format():
    v = np.concatenate([ku.E4M3, -ku.E4M3])
    t = torch.from_numpy(v).float().to(torch.float8_e4m3fn)
    assert np.array_equal(t.double().numpy(), v)
    assert np.array_equal(t.view(torch.uint8).numpy(), ku.encode_values(v, "e4m3"))
    x = np.random.default_rng(1).standard_normal(20000) * np.exp(np.random.default_rng(2).uniform(-9, 5, 20000))
    x = np.clip(x.astype(np.float32), -448, 448)
    mid = ((ku.E4M3[:-1] + ku.E4M3[1:]) / 2).astype(np.float32)   # ties
    for y in (x, mid, -mid):
        t = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        assert np.array_equal(t, ku.encode_values(y.astype(np.float64), "e4m3"))


def test_the_fused_step_rejects_invalid_arguments(R):
    E, U = R.RBQ_EINVAL, R.RBQ_EUNSUPPORTED

    def step(**k):
        g = k.get
        return R.lib.rbq_decode_step_kv8(
            1, g("Hq", 8), 4, g("D", 128), FAKE, g("P", FAKE), g("c_q", None), FAKE, g("K8", FAKE), FAKE, g("fmt", 16),
            g("block", 64), FAKE, FAKE, g("cap", 200), g("n", 100), g("kl", FAKE), FAKE, g("ldt", 1), g("ld", 16), g("w", 10),
            FAKE, g("kf", FAKE), g("kf16", None), g("flush", 1), g("p", 0.9), 0.1, FAKE, FAKE, FAKE, g("sel", FAKE), FAKE,
            FAKE, None, FAKE, g("wsb", 1 << 30), 0)

    for kw, want in [(dict(kf=None), E), (dict(kf16=FAKE), E), (dict(kf=None, kf16=FAKE, c_q=FAKE), E),
                     (dict(kf=None, kf16=FAKE + 2), E), (dict(cap=105), E), (dict(n=-1), E), (dict(n=201), E), (dict(w=-1), E),
                     (dict(w=17), E), (dict(kl=None), E), (dict(ldt=7), U), (dict(block=20), E), (dict(fmt=2), U),
                     (dict(D=96), U), (dict(Hq=12), U), (dict(p=0.0), E), (dict(P=None), E), (dict(K8=None), E),
                     (dict(sel=None), E), (dict(wsb=64), E)]:
        assert step(**kw) == want, kw
    need = R.rbq_workspace_bytes(R.RBQ_OP_DECODE_STEP_KV8, 1, 32, 8, 128, 4000, 64)
    assert need >= R.rbq_workspace_bytes(R.RBQ_OP_DECODE_KV8, 1, 32, 8, 128, 4000, 64) > 0
    assert R.rbq_workspace_bytes(R.RBQ_OP_DECODE_STEP_KV8, 1, 6, 4, 128, 4000, 64) == 0


def test_pipeline_objects_refuse_what_they_cannot_hold():
    from paper_2606_31519_amd import pipeline
    with pytest.raises(ValueError):
        pipeline.Kv8Cache(1, 2, 64, 32, fmt="e5m2", device="cpu")
    for q, k in (([], None), ([3], [3, 4]), ([-1], None), ([3], [-2])):
        with pytest.raises(ValueError):
            pipeline.PromptAttention(4, 2, 64, q, k, device="cpu")
    att = pipeline.PromptAttention(4, 2, 64, [3, 5], [3, 9], device="cpu")
    q, K, C = torch.zeros(8, 4, 64), torch.zeros(12, 2, 64), torch.zeros(2, 2, 9, 64)
    for bad in ((q[:7], K, K), (torch.zeros(8, 4, 32), K, K), (torch.zeros(8, 2, 64), K, K), (q, K[:11], K[:11]),
                (q, K, K.double()[:, :, :32]), (q, C[:, :, :8], C[:, :, :8]), (q, C[:1], C[:1]), (q, K[0], K[0]),
                (q, C, C.transpose(1, 2).contiguous().transpose(1, 2)), (q.transpose(1, 2).contiguous().transpose(1, 2), K, K)):
        with pytest.raises(ValueError):
            att(*bad)
    K = torch.zeros(1, 2, 40, 64)
    with pytest.raises(ValueError):    # fewer rows than the prefill
        pipeline.DecodeSession(1, 4, 2, 64, 100, 50, 16, K, K, torch.eye(64), device="cpu", kv8="int8")
    with pytest.raises(ValueError):    # rows that are not contiguous
        pipeline.DecodeSession(1, 4, 2, 64, 100, 30, 16, K[:, :, :35], K[:, :, :35], torch.eye(64), device="cpu", kv8="int8")


@pytest.mark.parametrize("sparse", [False, True])
def test_a_ragged_batch_of_too_many_blocks_is_refused(R, sparse):
    kw = dict(B=16383, Hq=4, Hkv=4, D=64, n=(1 << 25) - 1, cap=(1 << 25) - 1, wsb=(1 << 63) - 1)
    assert _decode(R, sparse, sn=FAKE, **kw) == R.RBQ_EUNSUPPORTED


def test_workspace_of_every_length_covers_shorter_windows(R):
    """The splits' number goes by rules on the sizes: the workspace of a call is that of its own sizes, and every size of a
    growing cache has one."""
    for Hkv, D in [(8, 128), (4, 64), (1, 128)]:
        for n in list(range(0, 3000, 97)) + list(range(3000, 200000, 7919)):
            for w in (0, 1, 256, 700):
                a = R.rbq_workspace_bytes(R.RBQ_OP_DECODE_KV8, 1, 4 * Hkv, Hkv, D, n, w)
                # a split has at least 128 rows, a window's 256, and a call without rows one: so many states of D + 2 floats
                most = (n + 127) // 128 + (w + 255) // 256 + 1
                assert a > 0 and a % 256 == 0 and a <= (4 * Hkv) * (D + 2) * 4 * most + 256, (n, w)


def test_windows_of_their_own_take_splits_of_their_own(R):
    """seq_w without seq_n: the window's length is the device's, so its rows are no part of the last splits (as they are
    where w is every sequence's). The call needs the states of the windows' splits, and the workspace has them."""
    for kw, idx, win in [(dict(B=1, Hq=32, Hkv=8, D=128, n=130816, cap=130816, w=256, ld=256), 128, 1),
                         (dict(B=8, Hq=64, Hkv=8, D=64, n=15700, cap=15700, w=300, ld=300), 16, 2),
                         (dict(B=4, Hq=8, Hkv=8, D=128, n=32768, cap=32768, w=200, ld=200), 32, 1)]:
        state = kw["B"] * kw["Hq"] * (kw["D"] + 2) * 4
        assert _decode(R, True, **kw, wsb=idx * state - 1) == R.RBQ_EINVAL          # (the windows are taken along)
        assert _decode(R, True, **kw, sw=FAKE, wsb=(idx + win) * state - 1) == R.RBQ_EINVAL, kw
        assert R.rbq_workspace_bytes(R.RBQ_OP_DECODE_KV8, *(kw[k] for k in ("B", "Hq", "Hkv", "D", "n", "w"))) >= \
            (idx + win) * state


def test_prompt_attention_refuses_one_cache_for_several_sequences():
    """A cache expanded over the sequences has no stride from one to the next, which the call takes for packed rows."""
    from paper_2606_31519_amd import pipeline
    att = pipeline.PromptAttention(4, 2, 64, [3, 5], [7, 9], device="cpu")
    q, C = torch.zeros(8, 4, 64), torch.zeros(1, 2, 9, 64).expand(2, -1, -1, -1)
    with pytest.raises(ValueError, match="rows of its own"):
        att(q, C, C, stream=0)


@pytest.mark.parametrize("op", ["DECODE_KV8", "DECODE_STEP_KV8"])
def test_a_workspace_serves_every_shorter_window(R, op):
    """A decode loop holds one workspace for each index length, sized with the full window, and passes every window from
    none to it: the size must not shrink as the window grows."""
    op = getattr(R, "RBQ_OP_" + op)
    rng = np.random.default_rng(2)
    # B, Hkv, D, n, window: first lengths at which the splits of a shorter window are more
    cases = [(2, 8, 128, 56490, 512), (2, 8, 128, 103519, 1024), (1, 8, 128, 96953, 1024), (1, 8, 128, 195923, 128)]
    cases += [(int(2 ** rng.uniform(0, 5)), int(2 ** rng.integers(0, 4)), int(rng.choice([64, 128])),
               int(np.exp(rng.uniform(0, np.log(400000)))), int(rng.integers(1, 4097))) for _ in range(3000)]
    for B, Hkv, D, n, window in cases:
        need = [R.rbq_workspace_bytes(op, B, 4 * Hkv, Hkv, D, n, w) for w in sorted({0, 1, *range(256, window, 256),
                                                                                     *range(257, window, 256), window})]
        assert need == sorted(need), (B, Hkv, D, n, window)


def test_a_session_in_8_bits_is_never_refused_a_step(R):
    """The call's own check, with the workspace that DecodeSession would hold, at every index length and window of it."""
    for B, n0, window, cap in [(2, 54954, 512, 57002), (2, 103519, 1024, 107615), (1, 92857, 1024, 96953),
                               (1, 195923, 128, 196435)]:
        size = lambda n, w: R.rbq_workspace_bytes(R.RBQ_OP_DECODE_STEP_KV8, B, 32, 8, 128, n, w)  # noqa: E731
        sizes = list(range(n0, cap + 1, window))
        held = max([size(n, window) for n in sizes] +
                   [R.rbq_workspace_bytes(R.RBQ_OP_DECODE_STEP, B, 32, 8, 128, sizes[-1], window)])
        for n in sizes:
            for w in [0, 1, *range(256, window + 1, 256), *range(257, window + 1, 256)]:
                assert size(n, w) <= held, (B, n, w)


def test_rows_may_be_the_tail_of_a_longer_buffer(R):
    """K + n * D with ld = cap, as the calls allow: the view has gaps between the heads and holds fewer elements than it
    reaches over. The binding lets it through (to the library's own refusal here); views that end too early it refuses."""
    B, H, D, cap, block, n, w = 2, 2, 64, 64, 16, 48, 16
    i8, s = torch.zeros(B, H, cap, D, dtype=torch.int8), torch.zeros(B, H, cap // block)
    x = torch.zeros(B, H, cap, D)
    tail = x[:, :, n:]
    q, out, lse, ws = torch.zeros(B, 4, D), torch.zeros(B, 4, D), torch.zeros(B, 4), torch.zeros(1 << 16, dtype=torch.uint8)
    calls = {
        "write": lambda t, m: R.rbq_quantize_kv(B, H, D, t, t, cap, m, cap, cap, block, i8, i8, s, s, stream=0),
        "read": lambda t, m: R.rbq_dequantize_kv(B, H, D, i8, i8, block, s, s, cap, m, cap, t, t, cap, stream=0),
        "window": lambda t, m: R.rbq_dense_decode_kv8(B, 4, H, D, q, i8, i8, block, s, s, cap, cap, t, t, cap, m, -1.0, out,
                                                      lse, ws, stream=0),
    }
    for name, call in calls.items():
        with pytest.raises(R.RbqError) as e:      # (rows past the cache's capacity, a negative scale)
            call(tail, w)
        assert e.value.status == R.RBQ_EINVAL, name
        for short in (x[:, :, n + 1:], x[:1, :, n:], tail.contiguous(), x[:1].expand(B, -1, -1, -1)):
            with pytest.raises(ValueError):
                call(short, w)


def test_without_its_call_module_the_binding_has_the_other_calls():
    """The library's calls through ctypes do not need the call module: it is asked for where a call goes through it."""
    import subprocess
    import sys
    code = """if True:
        import sys
        sys.modules["paper_2606_31519_amd._rbqcall"] = None      # (an import of it fails)
        import torch
        from paper_2606_31519_amd import pipeline, rbq
        assert rbq.rbq_version() > 0 and rbq.rbq_workspace_bytes(rbq.RBQ_OP_TOPP, 1, 8, 2, 128, 100) > 0
        x, c, s = torch.zeros(1, 1, 4, 64), torch.zeros(1, 1, 16, 64, dtype=torch.int8), torch.zeros(1, 1, 1)
        try:
            rbq.rbq_quantize_kv(1, 1, 64, x, x, 4, 4, 0, 16, 16, c, c, s, s)
        except ImportError as e:
            assert "_rbqcall" in str(e)
            print("refused")
    """
    from conftest import ROOT
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "refused", r.stderr
