"""rbq_prefill_attention_kv4 against 64 bits: chunks over 4-bit rows and their own
rows, sequences without either, group sizes that are no powers of two, cached rows
that end inside a step, keys split over blocks, strided and packed rows."""
import math

import numpy as np
import pytest
import torch

import kv4_util as ku

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def R():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2606_31519_amd import rbq
    return rbq


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Inputs:
    """Chunks of qs tokens behind ns cached rows; q, K and V of one fused projection ([tokens][Hq + 2 Hkv][D]) or packed."""

    def __init__(self, seed, fmt, dt, Hq, Hkv, D, qs, ns, fused=False, lead=0, tail=0, cap=None):
        self.fmt, self.dt, self.Hq, self.Hkv, self.D, self.qs, self.ns, B = fmt, dt, Hq, Hkv, D, qs, ns, len(qs)
        self.B, self.n, self.cap, self.tau = B, max(ns), max(ns) + 3 if cap is None else cap, 1.0 / math.sqrt(D)
        rng = np.random.default_rng(seed)
        self.code = {k: ku.random_cache(rng, (B, Hkv, self.cap), D, fmt) for k in "KV"}
        rec = ku.records(self.code["K"][0], self.code["V"][0], fmt)
        par = np.stack([self.code["K"][1], self.code["V"][1]], axis=-1)
        for b in range(B):          # rows that no sequence has
            rec[b, :, ns[b]:] = 0xFF
            par[b, :, ns[b]:] = 0xFFFFFFFF
        self.kv, self.par = dev(rec), dev(par.astype(np.uint32).view(np.int32))
        self.cu = np.cumsum([lead] + list(qs)).tolist()
        self.T = self.cu[-1] + tail
        g = torch.Generator(device="cuda").manual_seed(seed)
        x = torch.randn(max(self.T, 1), Hq + 2 * Hkv, D, device="cuda", generator=g).to(DT[dt])
        self.q, self.K, self.V = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        if not fused:
            self.q, self.K, self.V = (t.contiguous() for t in (self.q, self.K, self.V))
        self.cu_q, self.seq_n = i32(self.cu), i32(ns)

    def buffers(self, R):
        out = torch.full((max(self.T, 1), self.Hq, self.D), 5.0, dtype=DT[self.dt], device="cuda")
        lse = torch.full((max(self.T, 1), self.Hq), 5.0, device="cuda")
        ws = R.workspace(R.RBQ_OP_PREFILL_KV4, self.B, self.Hq, self.Hkv, self.D, self.n, self.T)
        ws.fill_(255)               # NaN patterns: nothing is read before it is written
        return out, lse, ws

    def run(self, R, causal, out=None, lse=None, ws=None, stream=None):
        if out is None:
            out, lse, ws = self.buffers(R)
        R.rbq_prefill_attention_kv4(self.B, self.Hq, self.Hkv, self.D, self.q, self.q.stride(0), self.K, self.V,
                                    self.K.stride(0), self.K.stride(1), self.cu_q, self.T, self.kv, self.par,
                                    R.KV4_FORMATS[self.fmt], self.cap, self.n, self.seq_n, causal, self.tau, out, lse, ws,
                                    stream=stream)
        return out, lse


def check(inp, out, lse, causal, heads=None):
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    q, Ko, Vo = (t.double().cpu().numpy() for t in (inp.q, inp.K, inp.V))
    G = inp.Hq // inp.Hkv
    for b in range(inp.B):
        nq, nb, at = inp.qs[b], inp.ns[b], slice(inp.cu[b], inp.cu[b + 1])
        if nq == 0:
            continue
        for h in (range(inp.Hq) if heads is None else heads):
            K, V, Kb, Vb = [], [], [], []
            for k, own, val, blk in (("K", Ko, K, Kb), ("V", Vo, V, Vb)):
                c, w = (t[b, h // G][:nb] for t in inp.code[k])
                val += [ku.exact_values(c, w, inp.fmt), own[at, h // G]]
                blk += [ku.bulk(c, w, inp.fmt), np.abs(own[at, h // G])]
            K, V, Kb, Vb = (np.concatenate(t) for t in (K, V, Kb, Vb))
            Q = q[at, h]
            S = Q @ K.T * inp.tau
            if causal:
                S = np.where(np.arange(nb + nq)[None] <= np.arange(nq)[:, None] + nb, S, -np.inf)
            m = S.max(axis=1)
            p = np.exp(S - m[:, None])
            tot = p.sum(axis=1)
            want = p @ V / tot[:, None]
            big = Q[np.argmax((np.abs(Q) @ Kb.T).max(axis=1))]
            ot, lt = ku.attention_tolerance(big, K, V, Kb, Vb, inp.tau)
            if inp.dt == "bf16":   # each probability, cached value and the result are off by up to half a step of bf16
                mean = p @ np.abs(V) / tot[:, None]
                ot = ot + 2.0 ** -8 * ((2 if inp.fmt == "int4" else 1) * mean + np.abs(want))
            o, l = out[at, h], lse[at, h]
            assert np.all(np.abs(o - want) <= ot), (b, h, np.abs(o - want).max())
            wl = m + np.log(tot)
            assert np.all(np.abs(l - wl) <= lt), (b, h, np.abs(l - wl).max(), lt)


# dtype, Hq, Hkv, D, tokens, cached rows, fused, causal
CASES = [
    ("bf16", 8, 2, 128, [1], [0], False, True),
    ("bf16", 8, 2, 128, [1], [1], False, True),
    ("bf16", 8, 2, 128, [257], [300], True, True),
    ("bf16", 4, 4, 64, [63, 1, 0, 130, 64], [64, 63, 5, 0, 129], True, True),
    ("bf16", 6, 2, 128, [100, 31, 7], [64, 128, 1], False, True),              # three heads a group
    ("bf16", 16, 1, 64, [9, 40], [700, 65], False, True),
    ("bf16", 8, 2, 128, [33, 65], [190, 66], False, False),
    ("bf16", 32, 8, 128, [300, 17, 460], [0, 1000, 255], False, True),
    ("bf16", 8, 2, 128, [1, 3], [4097, 5000], False, True),                    # keys split over blocks
    ("bf16", 8, 1, 64, [2], [9001], False, False),
    ("bf16", 8, 1, 64, [150, 3], [300, 70], False, True),                      # whole tiles of 128 rows at D = 64
    ("bf16", 12, 1, 128, [100, 1, 0], [0, 129, 64], True, False),               # twelve heads a group
    ("bf16", 3, 1, 64, [40, 41], [31, 32], True, True),
    ("f32", 8, 2, 128, [1, 40], [1, 40], False, True),
    ("f32", 4, 4, 64, [33, 0, 129], [65, 5, 0], True, True),
    ("f32", 6, 2, 128, [20, 5], [90, 3], False, True),
    ("f32", 2, 1, 64, [31], [64], False, False),
    ("f32", 4, 1, 128, [3], [3001], False, True),
    ("f32", 12, 1, 64, [150, 3], [300, 70], False, True),
    ("f32", 2, 1, 128, [1200], [70], False, True),                              # mostly keys of its own
    ("f32", 1, 1, 64, [1100], [100], True, False),
]


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}-Hq{c[1]}-Hkv{c[2]}-D{c[3]}-q{max(c[4])}-n{max(c[5])}" for c in CASES])
def test_chunks_over_cached_rows(R, case, fmt):
    dt, Hq, Hkv, D, qs, ns, fused, causal = case
    print("chunk", case, fmt, flush=True)
    inp = Inputs(sum(ns) + Hq, fmt, dt, Hq, Hkv, D, qs, ns, fused)
    out, lse = inp.run(R, causal)
    torch.cuda.synchronize()
    check(inp, out, lse, causal, None if Hq <= 8 else (0, Hq - 1))


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("dt,D", [("bf16", 128), ("f32", 64)])
def test_many_sequences_and_rows_outside_them(R, dt, D, fmt):
    """More sequences than lanes, empty ones among them; rows before and behind every sequence are left as they were."""
    rng = np.random.default_rng(5)
    qs, ns = rng.integers(0, 6, 70).tolist(), rng.integers(0, 150, 70).tolist()
    inp = Inputs(9, fmt, dt, 4, 2, D, qs, ns, lead=3, tail=4)
    out, lse = inp.run(R, True)
    check(inp, out, lse, True)
    for t in (out, lse):
        assert torch.all(t[:3] == 5.0) and torch.all(t[-4:] == 5.0)


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("dt,D", [("bf16", 64), ("f32", 128)])
def test_lengths_beyond_the_buffers_are_clamped(R, dt, D, fmt):
    inp = Inputs(3, fmt, dt, 4, 2, D, [20, 10], [70, 33], cap=70)
    want = inp.run(R, True)
    inp.seq_n = i32([1 << 30, 33])
    got = inp.run(R, True)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    inp.seq_n, inp.ns = i32([-5, 33]), [0, 33]
    check(inp, *inp.run(R, True), True)
    inp.seq_n, inp.ns, inp.n = None, [33, 33], 33    # without lengths: n rows each
    check(inp, *inp.run(R, True), True)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("qs,ns", [([5], [2000]), ([40, 3], [70, 128])])
def test_infinities_and_nan_of_a_chunk_reach_the_tokens_that_see_them_only(R, dt, qs, ns):
    inp = Inputs(11, "fp4", dt, 4, 2, 128, qs, ns)
    clean = [t.clone() for t in inp.run(R, True)]
    at = inp.cu[1] - 2                                 # the first sequence's last but one token
    inp.V[at, 0, 3], inp.V[at, 0, 5] = float("inf"), float("nan")
    out, lse = inp.run(R, True)
    assert torch.equal(lse, clean[1])
    seen = torch.zeros_like(out, dtype=torch.bool)
    seen[at:inp.cu[1], :2, 3] = True
    seen[at:inp.cu[1], :2, 5] = True
    assert torch.equal(out[~seen], clean[0][~seen])
    assert torch.all(out[at:inp.cu[1], :2, 3] == float("inf")) and torch.all(out[at:inp.cu[1], :2, 5].isnan())
    inp.K[at, 1, 7] = float("nan")                     # a key: the heads that see it
    out, lse = inp.run(R, True)
    assert torch.all(out[at:inp.cu[1], 2:].isnan()) and torch.all(lse[at:inp.cu[1], 2:].isnan())
    assert torch.equal(lse[:at], clean[1][:at]) and torch.equal(lse[:, :2], clean[1][:, :2])


@pytest.mark.parametrize("qs,ns", [([7, 7, 3], [900, 0, 64]), ([130], [65])])
def test_graph_replays_and_two_streams(R, qs, ns):
    """A captured call, replayed with eager calls between the replays, and two calls at once with workspaces of their own."""
    inp = Inputs(21, "int4", "bf16", 8, 2, 128, qs, ns)
    want = [t.clone() for t in inp.run(R, True)]
    out, lse, ws = inp.buffers(R)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        inp.run(R, True, out, lse, ws)
    other = inp.buffers(R)
    side = torch.cuda.Stream()
    for _ in range(3):
        out.fill_(5.0), lse.fill_(5.0), ws.fill_(255)
        side.wait_stream(torch.cuda.current_stream())
        g.replay()
        inp.run(R, True, *other, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        assert torch.equal(other[0], want[0]) and torch.equal(other[1], want[1])


def test_the_chunk_after_rows_in_full_precision(R):
    """Against rbq_prefill_attention over the rows that the cache stands for, read back: the same keys, in bf16."""
    inp = Inputs(31, "fp4", "bf16", 8, 2, 64, [50], [200])
    out, lse = inp.run(R, True)
    K, V = (torch.empty(1, 2, 250, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    R.rbq_dequantize_kv4(1, 2, 64, inp.kv, inp.par, R.RBQ_FP4, inp.cap, 200, 0, K, V, 250)
    K[0, :, 200:], V[0, :, 200:] = inp.K.transpose(0, 1), inp.V.transpose(0, 1)
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    ws = R.workspace(R.RBQ_OP_PREFILL, 1, 8, 2, 64, 250, 50)
    R.rbq_prefill_attention(1, 8, 2, 64, inp.q, 8 * 64, K, V, 64, 250 * 64, 2 * 250 * 64, 250, i32([0, 50]), i32([0, 250]), 50,
                            250, True, inp.tau, o2, l2, ws)
    assert (l2 - lse).abs().max() < 1e-5 and (o2.float() - out.float()).abs().max() <= 2.0 ** -6 * o2.float().abs().max()
