"""The 4-bit cache in use: the fused step against its separate calls, and a whole run,
the first turn's attention, index and 4-bit cache of it, a session whose window is
flushed into both, a further turn over the 4-bit rows, each stage checked."""
import math

import numpy as np
import pytest
import torch

import kv4_util as ku
import parity_util as pu
from kv8_util import attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2606_31519_amd import pipeline, rbq
    return rbq, pipeline


def rotation(D):
    return torch.linalg.qr(torch.randn(D, D, dtype=torch.float64, generator=torch.Generator().manual_seed(1)))[0].float().cuda()


class Setup:
    def __init__(self, mods, B, Hq, Hkv, D, n, w, fmt, loc, compact, seed=3):
        R, pl = mods
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        self.dims, self.n, self.w, self.compact = (B, Hq, Hkv, D), n, w, compact
        self.cap = n + w + 5
        K, V = (rnd(B, Hkv, n, D).to(torch.bfloat16) for _ in range(2))
        self.cache = pl.Kv4Cache(B, Hkv, D, self.cap, fmt)
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
        self.ws = R.workspace(R.RBQ_OP_DECODE_STEP_KV4, B, Hq, Hkv, D, n, w)
        self.ws.fill_(255)

    def outputs(self):
        torch.cuda.synchronize()
        st, c = self.st, self.cache
        cnt = st.sel_count.cpu()
        o = dict(qplanes=st.qplanes, qscal=st.qscal, scores=st.scores, cnt=cnt, out=st.out, lse=st.lse, codes=st.codes,
                 kv=c.kv4, par=c.par, fac=st.kfac16 if self.compact else st.kfac)
        o = {k: v.cpu().clone() for k, v in o.items()}
        B, Hq = self.dims[:2]
        o["sel"] = torch.cat([st.sel_idx[b, h, :int(cnt[b, h])].cpu() for b in range(B) for h in range(Hq)])
        return o


@pytest.mark.parametrize("flush", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,D,n,w,fmt,loc,compact", [
    (1, 32, 8, 128, 3967, 129, "fp4", torch.bfloat16, False),
    (2, 8, 2, 64, 1234, 40, "int4", torch.float32, False),
    (1, 8, 2, 128, 40000, 64, "int4", torch.bfloat16, True),
    (1, 16, 1, 64, 2000, 0, "fp4", torch.bfloat16, True),
    (2, 4, 4, 128, 1, 7, "fp4", torch.float32, False),
    (8, 16, 8, 64, 15700, 300, "int4", torch.bfloat16, False),     # windows taken along by the last splits
    (8, 32, 8, 128, 15700, 300, "fp4", torch.float32, False),
])
def test_fused_step_is_its_separate_calls(mods, B, Hq, Hkv, D, n, w, fmt, loc, compact, flush):
    R, _ = mods
    print("step", B, Hq, Hkv, D, n, w, fmt, loc, compact, flush, flush=True)
    args = (mods, B, Hq, Hkv, D, n, w, fmt, loc, compact)
    a, b = Setup(*args), Setup(*args)
    st, c = a.st, a.cache
    head = (B, Hq, Hkv, D)
    st.quantize()
    if compact:
        R.rbq_score_f16(*head, n, a.cap, st.codes, st.kfac16, st.qplanes, st.qscal, st.scores)
    else:
        R.rbq_score(*head, n, a.cap, st.codes, st.kfac, st.qplanes, st.qscal, st.scores)
    st.select(0.9)
    ws = R.workspace(R.RBQ_OP_DECODE_KV4, *head, n, w)
    R.rbq_sparse_decode_kv4(*head, st.q, c.kv4, c.par, c.code, a.cap, n, st.sel_idx, st.sel_count, a.Kw, a.Vw, max(w, 1), w,
                            st.sm_scale, st.out, st.lse, ws)
    if flush and w:
        if compact:
            R.rbq_encode_keys_f16(B, Hkv, D, a.Kw, w, w, n, a.cap, st.P, st.c_k, st.codes, st.kfac16, 0)
        else:
            R.rbq_encode_keys(B, Hkv, D, a.Kw, w, w, n, a.cap, st.P, st.c_q, st.c_k, st.codes, st.kfac, 0)
        c.append(a.Kw, a.Vw, w, w, n)
    want = a.outputs()
    st, c = b.st, b.cache
    R.rbq_decode_step_kv4(*head, st.q, st.P, st.c_q, st.c_k, c.kv4, c.par, c.code, b.cap, n, b.Kw, b.Vw, max(w, 1), w, st.codes,
                          st.kfac, st.kfac16, flush, 0.9, st.sm_scale, st.qplanes, st.qscal, st.scores, st.sel_idx,
                          st.sel_count, st.out, st.lse, b.ws)
    got = b.outputs()
    for k in want:
        assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("fmt,D,compact,dt", [("fp4", 128, False, torch.bfloat16), ("int4", 64, True, torch.float32),
                                              ("int4", 128, False, torch.bfloat16)])
def test_turns_of_a_chat_over_the_4_bit_cache(mods, fmt, D, compact, dt):
    R, pl = mods
    print("run", fmt, D, compact, dt, flush=True)
    B, Hq, Hkv, n0, window, steps = 2, 8, 2, 700, 24, 60          # two flushes, then a window of 12
    G, tau, T = Hq // Hkv, 1.0 / math.sqrt(D), torch.float32
    g = torch.Generator(device="cuda").manual_seed(11)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, K, V = rnd(B * n0, Hq, D).to(dt), rnd(B, Hkv, n0, D).to(dt), rnd(B, Hkv, n0, D).to(dt)
    # the first turn over an empty cache is the prompt's attention
    pack = lambda t: t.transpose(1, 2).reshape(-1, Hkv, D).contiguous()  # noqa: E731
    first = pl.ChunkAttention(Hq, pl.Kv4Cache(B, Hkv, D, 8, fmt), [n0] * B, [0] * B)(q, pack(K), pack(V))
    want = pl.PromptAttention(Hq, Hkv, D, [n0] * B)(q, K, V)
    near = 2.0 ** -7 if dt == torch.bfloat16 else 2.0 ** -18     # (the plans may cut the keys otherwise)
    assert (first.to(T) - want.to(T)).abs().max() <= near * want.to(T).abs().max()
    # the session over the 4-bit cache
    cap = n0 + 3 * window
    ses = pl.DecodeSession(B, Hq, Hkv, D, cap, n0, window, K, V, rotation(D), compact=compact, kv4=fmt)
    c = ses.kv4
    rows = {k: [[list(t[b, h].double().cpu().numpy()) for h in range(Hkv)] for b in range(B)] for k, t in (("K", K), ("V", V))}
    K.fill_(float("nan"))                     # (the session does not read them again)

    def stored(k, b, h, n):
        """The codes and words of the model's rows, checked against the cache's."""
        enc = [ku.encode_row(r, fmt) for r in rows[k][b][h][:n]]
        codes, word = np.stack([e[0] for e in enc]), np.array([e[1] for e in enc], np.uint32)
        i = "KV".index(k)
        got = ku.unpack(c.kv4[b, h, :n, i * D // 2:(i + 1) * D // 2].cpu().numpy(), fmt)
        assert np.array_equal(c.par[b, h, :n, i].cpu().numpy().view(np.uint32), word)
        assert np.array_equal(ku.row_values(got, word, fmt), ku.row_values(codes, word, fmt))
        return codes, word

    win = {"K": [], "V": []}
    flushes = 0
    for t in range(steps):
        k1, v1 = rnd(B, Hkv, D).to(dt), rnd(B, Hkv, D).to(dt)
        ses.append(k1, v1)
        win["K"].append(k1.double().cpu().numpy())
        win["V"].append(v1.double().cpu().numpy())
        qs = 4.0 * rnd(B, Hq, D)
        n = ses.n
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
                val, blk = [], []
                for k in "KV":
                    codes, word = (x[got] for x in stored(k, b, hk, n))
                    x = np.stack([r[b, hk] for r in win[k]])
                    val.append(np.concatenate([ku.exact_values(codes, word, fmt), x]))
                    blk.append(np.concatenate([ku.bulk(codes, word, fmt), np.abs(x)]))
                qd = qs[b, h].double().cpu().numpy()
                wo, wl = attention(qd, *val, tau)
                ot, lt = ku.attention_tolerance(qd, *val, *blk, tau)
                assert np.abs(o[b, h] - wo).max() <= ot and abs(l[b, h] - wl) <= lt, (t, b, h)
        if flushed:
            flushes += 1
            for k in "KV":
                for b in range(B):
                    for hk in range(Hkv):
                        rows[k][b][hk] += [r[b, hk] for r in win[k]]
                        stored(k, b, hk, ses.n)
            win = {"K": [], "V": []}
    assert flushes == 2 and ses.n == n0 + 2 * window and ses.w == steps - 2 * window
    # a further turn: its attention over the 4-bit rows and its own, which then enter the cache
    lens = [33, 5]
    att = pl.ChunkAttention(Hq, c, lens, [ses.n, ses.n - 100])
    qc, Kc, Vc = rnd(38, Hq, D).to(dt), rnd(38, Hkv, D).to(dt), rnd(38, Hkv, D).to(dt)
    out = att(qc, Kc, Vc).double().cpu().numpy()
    for b, i, h in ((0, 20, 0), (1, 4, Hq - 1)):
        nb, at = ses.n - 100 * b, 33 * b
        val, blk = [], []
        for k, own in (("K", Kc), ("V", Vc)):
            codes, word = stored(k, b, h // G, nb)
            x = own[at:at + i + 1, h // G].double().cpu().numpy()
            v = ku.exact_values(codes, word, fmt)
            val.append(np.concatenate([v, x]))
            blk.append(np.concatenate([np.abs(v) + ku.bulk(codes, word, fmt), np.abs(x)]))
        qd = qc[at + i, h].double().cpu().numpy()
        wo, _ = attention(qd, *val, tau)
        ot, _ = ku.attention_tolerance(qd, *val, *blk, tau)
        if dt == torch.bfloat16:   # half a step of bf16 of each probability, cached value and output
            p = np.exp(val[0] @ qd * tau)
            ot = ot + 2.0 ** -8 * (2 * p @ np.abs(val[1]) / p.sum() + np.abs(wo))
        assert np.all(np.abs(out[at + i, h] - wo) <= ot), (b, i, h)


def test_rows_in_mapped_host_memory(mods):
    """K and V in pinned host memory, read over PCIe: written into the cache, as a window, and as a chunk's own rows,
    bitwise as from device memory; buffers that are too small are refused."""
    R = mods[0]
    B, Hq, Hkv, D, n, w, cap = 1, 4, 2, 64, 200, 24, 256
    g = torch.Generator().manual_seed(3)
    host = [torch.randn(B, Hkv, n, D, generator=g).to(torch.bfloat16).pin_memory() for _ in range(2)]
    q = torch.randn(B, Hq, D, generator=g).cuda()
    turn = torch.randn(5, Hq, D, generator=g).to(torch.bfloat16).cuda()
    res = []
    for rows in ([t.cuda() for t in host], [R.MappedHost(t) for t in host]):
        kv, par = (torch.zeros(B, Hkv, cap, D, dtype=torch.uint8, device="cuda"),
                   torch.zeros(B, Hkv, cap, 2, dtype=torch.int32, device="cuda"))
        R.rbq_quantize_kv4(B, Hkv, D, *rows, n, n, 0, cap, R.RBQ_I4, kv, par)
        out, lse = torch.empty(B, Hq, D, device="cuda"), torch.empty(B, Hq, device="cuda")
        ws = R.workspace(R.RBQ_OP_DECODE_KV4, B, Hq, Hkv, D, n, w)
        R.rbq_dense_decode_kv4(B, Hq, Hkv, D, q, kv, par, R.RBQ_I4, cap, n, *rows, n, w, 0.1, out, lse, ws)
        po = torch.empty_like(turn)
        cu = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
        pw = R.workspace(R.RBQ_OP_PREFILL_KV4, B, Hq, Hkv, D, n, 5)
        R.rbq_prefill_attention_kv4(B, Hq, Hkv, D, turn, Hq * D, *rows, D, n * D, cu, 5, kv, par, R.RBQ_I4, cap, n, None, True,
                                    0.1, po, None, pw)
        torch.cuda.synchronize()
        res.append((kv, par, out, lse, po))
        with pytest.raises(ValueError, match="rbq_quantize_kv4"):
            R.rbq_quantize_kv4(B, Hkv, D, *rows, n + 1, n, 0, cap, R.RBQ_I4, kv, par)
    for a, b in zip(*res):
        assert torch.equal(a, b)
