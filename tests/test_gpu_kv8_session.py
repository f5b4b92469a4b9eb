"""The 8-bit cache in use: the fused step against its separate calls, and a whole run,
prompt attention, index and 8-bit cache of the prompt, a session whose window is flushed
into both, a second chunk of the prompt behind the rows read back, each stage checked."""
import math

import numpy as np
import pytest
import torch

import kv8_util as ku
import parity_util as pu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2606_31519_amd import pipeline, rbq
    return rbq, pipeline


def rotation(D):
    return torch.linalg.qr(torch.randn(D, D, dtype=torch.float64, generator=torch.Generator().manual_seed(1)))[0].float().cuda()


class Setup:
    def __init__(self, mods, B, Hq, Hkv, D, n, w, fmt, block, loc, compact, seed=3):
        R, pl = mods
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        self.dims, self.n, self.w, self.compact = (B, Hq, Hkv, D), n, w, compact
        self.cap = n + w + 5
        K, V = (rnd(B, Hkv, n, D).to(torch.bfloat16) for _ in range(2))
        self.cache = pl.Kv8Cache(B, Hkv, D, self.cap, fmt, block)
        self.cache.append(K, V, n, n, 0)
        self.Kw, self.Vw = (rnd(B, Hkv, max(w, 1), D).to(loc) for _ in range(2))
        c_q = None if compact else 0.3 * rnd(B, Hkv, D)
        self.st = pl.DecodeState(B, Hq, Hkv, D, self.cap, n, w, self.Kw, self.Vw, 3.0 * rnd(B, Hq, D), rotation(D), c_q,
                                 "cuda", compact)
        st = self.st
        if compact:
            R.rbq_encode_keys_f16(B, Hkv, D, K, n, n, 0, self.cap, st.P, st.c_k, st.codes, st.kfac16, 1, st.ws_encode)
        else:
            R.rbq_encode_keys(B, Hkv, D, K, n, n, 0, self.cap, st.P, c_q, st.c_k, st.codes, st.kfac, 1, None, st.ws_encode)
        self.ws = R.workspace(R.RBQ_OP_DECODE_STEP_KV8, B, Hq, Hkv, D, n, w)
        self.ws.fill_(255)

    def outputs(self):
        torch.cuda.synchronize()
        st, c = self.st, self.cache
        cnt = st.sel_count.cpu()
        o = dict(qplanes=st.qplanes, qscal=st.qscal, scores=st.scores, cnt=cnt, out=st.out, lse=st.lse, codes=st.codes,
                 K8=c.K8.view(torch.int8), V8=c.V8.view(torch.int8), ks=c.k_scale, vs=c.v_scale,
                 fac=st.kfac16 if self.compact else st.kfac)
        o = {k: v.cpu().clone() for k, v in o.items()}
        B, Hq = self.dims[:2]
        o["sel"] = torch.cat([st.sel_idx[b, h, :int(cnt[b, h])].cpu() for b in range(B) for h in range(Hq)])
        return o


@pytest.mark.parametrize("flush", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,D,n,w,fmt,block,loc,compact", [
    (1, 32, 8, 128, 3967, 129, "e4m3", 64, torch.bfloat16, False),
    (2, 8, 2, 64, 1234, 40, "int8", 16, torch.float32, False),
    (1, 8, 2, 128, 40000, 64, "int8", 128, torch.bfloat16, True),
    (1, 16, 1, 64, 2000, 0, "e4m3", 256, torch.bfloat16, True),
    (2, 4, 4, 128, 1, 7, "e4m3", 32, torch.float32, False),
    (8, 16, 8, 64, 15700, 300, "int8", 64, torch.bfloat16, False),     # windows taken along by the last splits
])
def test_fused_step_is_its_separate_calls(mods, B, Hq, Hkv, D, n, w, fmt, block, loc, compact, flush):
    R, _ = mods
    print("step", B, Hq, Hkv, D, n, w, fmt, block, loc, compact, flush, flush=True)
    args = (mods, B, Hq, Hkv, D, n, w, fmt, block, loc, compact)
    a, b = Setup(*args), Setup(*args)
    st, c = a.st, a.cache
    head = (B, Hq, Hkv, D)
    st.quantize()
    if compact:
        R.rbq_score_f16(*head, n, a.cap, st.codes, st.kfac16, st.qplanes, st.qscal, st.scores)
    else:
        R.rbq_score(*head, n, a.cap, st.codes, st.kfac, st.qplanes, st.qscal, st.scores)
    st.select(0.9)
    ws = R.workspace(R.RBQ_OP_DECODE_KV8, *head, n, w)
    R.rbq_sparse_decode_kv8(*head, st.q, c.K8, c.V8, block, c.k_scale, c.v_scale, a.cap, n, st.sel_idx, st.sel_count, a.Kw,
                            a.Vw, max(w, 1), w, st.sm_scale, st.out, st.lse, ws)
    if flush and w:
        if compact:
            R.rbq_encode_keys_f16(B, Hkv, D, a.Kw, w, w, n, a.cap, st.P, st.c_k, st.codes, st.kfac16, 0)
        else:
            R.rbq_encode_keys(B, Hkv, D, a.Kw, w, w, n, a.cap, st.P, st.c_q, st.c_k, st.codes, st.kfac, 0)
        c.append(a.Kw, a.Vw, w, w, n)
    want = a.outputs()
    st, c = b.st, b.cache
    R.rbq_decode_step_kv8(*head, st.q, st.P, st.c_q, st.c_k, c.K8, c.V8, block, c.k_scale, c.v_scale, b.cap, n, b.Kw, b.Vw,
                          max(w, 1), w, st.codes, st.kfac, st.kfac16, flush, 0.9, st.sm_scale, st.qplanes, st.qscal,
                          st.scores, st.sel_idx, st.sel_count, st.out, st.lse, b.ws)
    got = b.outputs()
    for k in want:
        assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("fmt,block,D,compact,dt", [("e4m3", 64, 128, False, torch.bfloat16), ("int8", 16, 64, True, torch.float32)])
def test_prompt_cache_session_and_next_chunk(mods, fmt, block, D, compact, dt):
    R, pl = mods
    print("run", fmt, block, D, compact, dt, flush=True)
    B, Hq, Hkv, n0, window, steps = 2, 8, 2, 700, 24, 60          # two flushes, then a window of 12
    G, tau = Hq // Hkv, 1.0 / math.sqrt(D)
    g = torch.Generator(device="cuda").manual_seed(11)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, K, V = rnd(B * n0, Hq, D).to(dt), rnd(B, Hkv, n0, D).to(dt), rnd(B, Hkv, n0, D).to(dt)
    # the prompt's attention, from the rows as they will be cached, and the same from packed ones
    att = pl.PromptAttention(Hq, Hkv, D, [n0] * B)
    lse = torch.empty(B * n0, Hq, device="cuda")
    out = att(q, K, V, lse=lse)
    pack = lambda t: t.transpose(1, 2).reshape(B * n0, Hkv, D).contiguous()  # noqa: E731
    assert torch.equal(out, att(q, pack(K), pack(V)))
    for b, i, h in ((0, 0, 0), (1, 350, 3), (1, n0 - 1, Hq - 1)):
        Kd, Vd = (t[b, h // G, :i + 1].double().cpu().numpy() for t in (K, V))
        qd = q[b * n0 + i, h].double().cpu().numpy()
        o, l = ku.attention(qd, Kd, Vd, tau)
        ot, lt = ku.attention_tolerance(qd, Kd, Vd, tau)
        if dt == torch.bfloat16:
            p = np.exp(Kd @ qd * tau - l)
            ot = ot + 2.0 ** -8 * (p @ np.abs(Vd) + np.abs(o))
        assert np.all(np.abs(out[b * n0 + i, h].double().cpu().numpy() - o) <= ot)
        assert abs(float(lse[b * n0 + i, h]) - l) <= lt
    # the session over the 8-bit cache
    cap = n0 + 3 * window
    ses = pl.DecodeSession(B, Hq, Hkv, D, cap, n0, window, K, V, rotation(D), compact=compact, kv8=fmt, kv8_block=block)
    K.fill_(float("nan"))                     # (the session does not read them again)
    rows = {k: [[v[b, hk].double().cpu().numpy() for hk in range(Hkv)] for b in range(B)] for k, v in (("V", V),)}
    model = {k: [[(np.zeros((cap, D), np.uint8), np.zeros((cap + block - 1) // block)) for _ in range(Hkv)] for _ in range(B)]
             for k in "KV"}
    Kp = ses.kv8.K8.view(torch.int8)          # the prompt's K codes are taken as they are (tested on their own)
    for b in range(B):
        for hk in range(Hkv):
            model["K"][b][hk][0][:n0] = Kp[b, hk, :n0].cpu().numpy().view(np.uint8)
            model["K"][b][hk][1][:] = ses.kv8.k_scale[b, hk].cpu().numpy()
            ku.append(*model["V"][b][hk], rows["V"][b][hk], 0, block, fmt)
    win = {"K": [], "V": []}
    flushes = 0
    for t in range(steps):
        k1, v1 = rnd(B, Hkv, D).to(dt), rnd(B, Hkv, D).to(dt)
        ses.append(k1, v1)
        win["K"].append(k1.double().cpu().numpy())
        win["V"].append(v1.double().cpu().numpy())
        qs = 4.0 * rnd(B, Hq, D)
        n, w = ses.n, ses.w
        flushed = ses.step(qs, 0.9)
        if flushed or t in (0, 30, steps - 1):
            torch.cuda.synchronize()
            st = ses.state
            S = st.scores.reshape(-1)[:B * Hq * n].reshape(B, Hq, n).cpu().numpy()
            sel = st.sel_idx.reshape(-1)[:B * Hq * n].reshape(B, Hq, n).cpu().numpy()
            cnt, o, l = st.sel_count.cpu().numpy(), st.out.cpu().numpy(), st.lse.cpu().numpy()
            for b, h in ((0, 0), (B - 1, Hq - 1)):
                hk, got = h // G, sel[b, h, :cnt[b, h]]
                pu.check_topp(S[b, h], 0.9, tau, got)
                Kd, Vd = (np.concatenate([ku.values(model[k][b][hk][0], model[k][b][hk][1], block, fmt)[got],
                                          np.stack([r[b, hk] for r in win[k]])]) for k in "KV")
                qd = qs[b, h].double().cpu().numpy()
                wo, wl = ku.attention(qd, Kd, Vd, tau)
                ot, lt = ku.attention_tolerance(qd, Kd, Vd, tau)
                assert np.abs(o[b, h] - wo).max() <= ot and abs(l[b, h] - wl) <= lt, (t, b, h)
        if flushed:
            flushes += 1
            for k in "KV":
                for b in range(B):
                    for hk in range(Hkv):
                        ku.append(*model[k][b][hk], np.stack([r[b, hk] for r in win[k]]), n, block, fmt)
            win = {"K": [], "V": []}
            got = {k: (t8.view(torch.int8).cpu().numpy().view(np.uint8), s.cpu().numpy()) for k, t8, s in
                   (("K", ses.kv8.K8, ses.kv8.k_scale), ("V", ses.kv8.V8, ses.kv8.v_scale))}
            for k in "KV":
                for b in range(B):
                    for hk in range(Hkv):
                        assert np.array_equal(got[k][1][b, hk], model[k][b][hk][1].astype(np.float32))
                        assert np.array_equal(ku.decode_codes(got[k][0][b, hk, :ses.n], fmt),
                                              ku.decode_codes(model[k][b][hk][0][:ses.n], fmt))
    assert flushes == 2 and ses.n == n0 + 2 * window and ses.w == steps - 2 * window
    # a further chunk of the conversation: its attention over the rows read back and its own
    chunk = 33
    total = ses.n + chunk
    Kc, Vc = (torch.zeros(B, Hkv, total, D, dtype=dt, device="cuda") for _ in range(2))
    ses.kv8.read(Kc, Vc, total, ses.n)
    Kc[:, :, ses.n:], Vc[:, :, ses.n:] = rnd(B, Hkv, chunk, D).to(dt), rnd(B, Hkv, chunk, D).to(dt)
    qc = rnd(B * chunk, Hq, D).to(dt)
    out = pl.PromptAttention(Hq, Hkv, D, [chunk] * B, [total] * B)(qc, Kc, Vc)
    b, i, h = 1, 5, Hq - 1
    Kd = np.concatenate([ku.values(model["K"][b][h // G][0], model["K"][b][h // G][1], block, fmt)[:ses.n],
                         Kc[b, h // G, ses.n:ses.n + i + 1].double().cpu().numpy()])
    Vd = Vc[b, h // G, :ses.n + i + 1].double().cpu().numpy()
    qd = qc[b * chunk + i, h].double().cpu().numpy()
    if dt == torch.bfloat16:                  # rows read back are rounded to bf16 (e4m3 values are exact in it)
        assert fmt == "e4m3"
    o, _ = ku.attention(qd, Kd, Vd, tau)
    ot, _ = ku.attention_tolerance(qd, Kd, Vd, tau)
    if dt == torch.bfloat16:
        p = np.exp(Kd @ qd * tau)
        ot = ot + 2.0 ** -8 * (p @ np.abs(Vd) / p.sum() + np.abs(o))
    else:                                     # (int8 values are rounded to fp32: half a step of each)
        ot = ot + 2 * 2.0 ** -24 * np.abs(Vd).max() + 2 * 2.0 ** -24 * np.abs(Kd).max() * np.abs(qd).sum() * tau * np.abs(Vd).max()
    assert np.all(np.abs(out[b * chunk + i, h].double().cpu().numpy() - o) <= ot)


def test_rows_in_mapped_host_memory(mods):
    """K and V in pinned host memory, read over PCIe: written into the cache, as a window, and as a prompt's keys, bitwise
    as from device memory; buffers that are too small are refused."""
    R = mods[0]
    B, Hq, Hkv, D, n, w, cap, block = 1, 4, 2, 64, 200, 24, 256, 32
    g = torch.Generator().manual_seed(3)
    host = [torch.randn(B, Hkv, n, D, generator=g).to(torch.bfloat16).pin_memory() for _ in range(2)]
    q = torch.randn(B, Hq, D, generator=g).cuda()
    prompt = torch.randn(5, Hq, D, generator=g).to(torch.bfloat16).cuda()
    res = []
    for rows in ([t.cuda() for t in host], [R.MappedHost(t) for t in host]):
        c = [torch.zeros(B, Hkv, cap, D, dtype=torch.int8, device="cuda") for _ in range(2)]
        s = [torch.zeros(B, Hkv, cap // block, device="cuda") for _ in range(2)]
        R.rbq_quantize_kv(B, Hkv, D, *rows, n, n, 0, cap, block, *c, *s)
        out, lse = torch.empty(B, Hq, D, device="cuda"), torch.empty(B, Hq, device="cuda")
        ws = R.workspace(R.RBQ_OP_DECODE_KV8, B, Hq, Hkv, D, n, w)
        R.rbq_dense_decode_kv8(B, Hq, Hkv, D, q, *c, block, *s, cap, n, *rows, n, w, 0.1, out, lse, ws)
        po = torch.empty_like(prompt)
        cu_q, cu_k = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 5], [0, n]))
        pw = R.workspace(R.RBQ_OP_PREFILL, B, Hq, Hkv, D, n, 5)
        R.rbq_prefill_attention(B, Hq, Hkv, D, prompt, Hq * D, *rows, D, n * D, Hkv * n * D, n, cu_q, cu_k, 5, n, True, 0.1, po,
                                None, pw)
        torch.cuda.synchronize()
        res.append((*c, *s, out, lse, po))
        with pytest.raises(ValueError, match="rbq_quantize_kv"):
            R.rbq_quantize_kv(B, Hkv, D, *rows, n + 1, n, 0, cap, block, *c, *s)
    for a, b in zip(*res):
        assert torch.equal(a, b)
