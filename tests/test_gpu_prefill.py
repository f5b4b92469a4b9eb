"""rbq_prefill_attention against 64 bits: whole prompts and chunks over cached rows,
packed and strided layouts, sequences of any length (none, one, many), group sizes
that are no powers of two, rows that see nothing, keys split over blocks."""
import math

import numpy as np
import pytest
import torch

from kv8_util import attention_tolerance

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def R():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2606_31519_amd import rbq
    return rbq


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Inputs:
    """Packed q / k / v of one fused projection ([tokens][Hq + 2 Hkv][D], layout "fused"), packed buffers of their own
    ("packed"), or K and V in a cache [B][Hkv][cap][D] ("cache")."""

    def __init__(self, seed, dt, Hq, Hkv, D, qs, ks, layout, lead=0, tail=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).to(DT[dt])  # noqa: E731
        self.dt, self.Hq, self.Hkv, self.D, self.qs, self.ks, self.layout = dt, Hq, Hkv, D, qs, ks, layout
        B = self.B = len(qs)
        cu_q, cu_k = (np.cumsum([s0] + list(v)).tolist() for s0, v in ((lead, qs), (lead if layout == "fused" else 0, ks)))
        self.cu_q, self.cu_k, self.T = cu_q, cu_k, cu_q[-1] + tail
        self.max_k = max(ks)
        rows = max(cu_k[-1], 1)
        if layout == "fused":
            self.qkv = rnd(max(self.T, rows), Hq + 2 * Hkv, D)
            self.q, self.K, self.V = self.qkv[:, :Hq], self.qkv[:, Hq:Hq + Hkv], self.qkv[:, Hq + Hkv:]
            ld = (Hq + 2 * Hkv) * D
            self.q_ld, self.lay = ld, (ld, D, 0, rows)
        else:
            self.q, self.q_ld = rnd(max(self.T, 1), Hq, D), Hq * D
            if layout == "packed":
                self.K, self.V = rnd(rows, Hkv, D), rnd(rows, Hkv, D)
                self.lay = (Hkv * D, D, 0, rows)
            else:
                cap = self.max_k + 3
                self.K, self.V = rnd(B, Hkv, cap, D), rnd(B, Hkv, cap, D)
                for b in range(B):      # rows that no sequence has
                    self.K[b, :, ks[b]:] = float("nan")
                    self.V[b, :, ks[b]:] = float("nan")
                self.lay = (D, cap * D, Hkv * cap * D, cap)
        self.tau = 1.0 / math.sqrt(D)

    def run(self, R, causal, ws=None, stream=None, out=None, lse=None):
        out = torch.full((max(self.T, 1), self.Hq, self.D), 5.0, dtype=DT[self.dt], device="cuda") if out is None else out
        lse = torch.full((max(self.T, 1), self.Hq), 5.0, device="cuda") if lse is None else lse
        if ws is None:
            ws = R.workspace(R.RBQ_OP_PREFILL, self.B, self.Hq, self.Hkv, self.D, self.max_k, self.T)
            ws.fill_(255)               # NaN patterns: nothing is read before it is written
        if not hasattr(self, "cu"):
            self.cu = i32(self.cu_q), i32(self.cu_k)
        R.rbq_prefill_attention(self.B, self.Hq, self.Hkv, self.D, self.q, self.q_ld, self.K, self.V, *self.lay, *self.cu,
                                self.T, self.max_k, causal, self.tau, out, lse, ws, stream=stream)
        return out, lse

    def sequence(self, b):
        q = self.q[self.cu_q[b]:self.cu_q[b + 1]].double().cpu().numpy()
        if self.layout == "cache":
            k, v = (t[b, :, :self.ks[b]].double().cpu().numpy() for t in (self.K, self.V))
        else:
            k, v = (t[self.cu_k[b]:self.cu_k[b + 1]].double().cpu().numpy().transpose(1, 0, 2) for t in (self.K, self.V))
        return q, k, v


def check(inp, out, lse, causal, heads=None):
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in range(inp.B):
        q, k, v = inp.sequence(b)
        nq, nk = inp.qs[b], inp.ks[b]
        if nq == 0:
            continue
        for h in (range(inp.Hq) if heads is None else heads):
            K, V = k[h // (inp.Hq // inp.Hkv)], v[h // (inp.Hq // inp.Hkv)]
            o, l = out[inp.cu_q[b]:inp.cu_q[b + 1], h], lse[inp.cu_q[b]:inp.cu_q[b + 1], h]
            S = q[:, h] @ K.T * inp.tau
            if causal:
                S = np.where(np.arange(nk)[None] <= np.arange(nq)[:, None] + nk - nq, S, -np.inf)
            m = S.max(axis=1, initial=-np.inf)
            some = m > -np.inf
            p = np.exp(S - np.where(some, m, 0.0)[:, None])
            tot = np.where(some, p.sum(axis=1), 1.0)
            want = p @ V / tot[:, None]
            assert np.all(o[~some] == 0) and np.all(l[~some] == -np.inf)
            if not some.any():
                continue
            # (the fp32 bound of the longest row, for the sequence's largest query)
            big = q[np.argmax((np.abs(q[:, h]) @ np.abs(K).T).max(axis=1)), h]
            ot, lt = attention_tolerance(big, K, V, inp.tau)
            if inp.dt == "bf16":   # each probability and the result are off by up to half a step of bf16
                ot = ot + 2.0 ** -8 * (p @ np.abs(V) / tot[:, None] + np.abs(want))
            assert np.all(np.abs(o - want) <= ot), (b, h, np.abs(o - want).max())
            wl = m + np.log(tot)
            assert np.all(np.abs(l - wl)[some] <= lt), (b, h, np.abs(l - wl)[some].max(), lt)


# dtype, Hq, Hkv, D, tokens, keys, layout, causal
CASES = [
    ("bf16", 8, 2, 128, [1], [1], "packed", True),
    ("bf16", 8, 2, 128, [257], [257], "fused", True),
    ("bf16", 4, 4, 64, [63, 1, 0, 130, 64], [63, 1, 0, 130, 64], "fused", True),
    ("bf16", 6, 2, 128, [100, 31, 7], [164, 31, 300], "packed", True),          # three heads a group; chunks
    ("bf16", 16, 1, 64, [9, 40], [700, 65], "cache", True),
    ("bf16", 5, 1, 128, [50, 3, 20], [20, 0, 20], "packed", True),              # more tokens than keys: rows that see nothing
    ("bf16", 8, 2, 128, [33, 65], [190, 64], "cache", False),
    ("bf16", 32, 8, 128, [300, 17, 460], [300, 17, 460], "packed", True),        # 256-row tiles
    ("bf16", 16, 2, 64, [1100], [1100], "fused", True),
    ("bf16", 8, 2, 128, [1, 3], [4097, 5000], "cache", True),                   # keys split over blocks
    ("bf16", 8, 1, 64, [2], [9001], "packed", False),
    ("f32", 8, 2, 128, [1, 40], [1, 40], "packed", True),
    ("f32", 4, 4, 64, [33, 0, 129], [65, 5, 129], "fused", True),
    ("f32", 6, 2, 128, [20, 5], [90, 3], "cache", True),
    ("f32", 2, 1, 64, [31], [64], "packed", False),
    ("f32", 4, 1, 128, [3], [3001], "cache", True),
]


@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}-Hq{c[1]}-Hkv{c[2]}-D{c[3]}-{c[6]}-q{max(c[4])}-k{max(c[5])}" for c in CASES])
def test_attention_of_prompts(R, case):
    dt, Hq, Hkv, D, qs, ks, layout, causal = case
    if layout == "fused":
        ks = qs                       # one token axis
    print("case", case, flush=True)
    inp = Inputs(17, dt, Hq, Hkv, D, qs, ks, layout)
    out, lse = inp.run(R, causal)
    torch.cuda.synchronize()
    check(inp, out, lse, causal)


@pytest.mark.parametrize("dt,D", [("bf16", 128), ("f32", 64)])
def test_many_sequences_and_rows_outside_them(R, dt, D):
    """More sequences than a wave has lanes, empty ones among them; tokens before the first and behind the last."""
    rng = np.random.default_rng(8)
    qs = [int(v) for v in rng.integers(0, 40, 150)]
    ks = [v + int(e) for v, e in zip(qs, rng.integers(0, 30, 150))]
    inp = Inputs(5, dt, 4, 2, D, qs, ks, "packed", lead=3, tail=11)
    out, lse = inp.run(R, True)
    torch.cuda.synchronize()
    assert torch.all(out[:3] == 5.0) and torch.all(out[-11:] == 5.0) and torch.all(lse[:3] == 5.0) and torch.all(lse[-11:] == 5.0)
    check(inp, out, lse, True, heads=(0, 3))


def test_rows_outside_the_sequences_with_split_keys(R):
    inp = Inputs(6, "bf16", 8, 2, 128, [2, 1], [3000, 1500], "packed", lead=2, tail=3)
    assert R.rbq_workspace_bytes(R.RBQ_OP_PREFILL, 2, 8, 2, 128, 3000, inp.T) > 0
    out, lse = inp.run(R, True)
    torch.cuda.synchronize()
    assert torch.all(out[:2] == 5.0) and torch.all(out[-3:] == 5.0) and torch.all(lse[:2] == 5.0) and torch.all(lse[-3:] == 5.0)
    check(inp, out, lse, True)


def test_lengths_beyond_the_buffers_are_clamped(R):
    """Device counts that pass max_k, the rows or the tokens read and write inside the buffers only: the results are those
    of the clamped lengths."""
    inp = Inputs(9, "bf16", 4, 2, 64, [40, 24], [100, 60], "cache")
    want = inp.run(R, False)
    inp.cu = i32([0, 40, 1000]), i32([0, 100, 160])
    got = inp.run(R, False)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    short = Inputs(9, "bf16", 4, 2, 64, [40, 24], [70, 60], "cache")
    short.K, short.V, short.lay = inp.K, inp.V, inp.lay
    want = short.run(R, False)
    inp.cu = i32([0, 40, 64]), i32([0, 100, 160])
    inp.max_k = 70
    got = inp.run(R, False)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_large_logits_and_a_rising_maximum(R):
    """Keys whose logits grow along the sequence (the running maximum moves at every step) and reach thousands."""
    inp = Inputs(10, "bf16", 4, 1, 128, [200], [900], "packed")
    inp.K.mul_(torch.linspace(0.1, 60.0, 900, device="cuda")[:, None, None].to(torch.bfloat16))
    out, lse = inp.run(R, True)
    torch.cuda.synchronize()
    check(inp, out, lse, True)


@pytest.mark.parametrize("qs,ks", [([90, 30], [90, 95]), ([2, 1], [3000, 2000])], ids=["whole", "split"])
def test_graph_replays_and_two_streams(R, qs, ks):
    inp = Inputs(11, "bf16", 8, 2, 128, qs, ks, "packed")
    want = [t.clone() for t in inp.run(R, True)]
    again = inp.run(R, True)
    torch.cuda.synchronize()
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])     # run to run
    ws = R.workspace(R.RBQ_OP_PREFILL, inp.B, 8, 2, 128, inp.max_k, inp.T)
    out, lse = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inp.run(R, True, ws=ws, out=out, lse=lse)
    for i in range(4):
        inp.q.copy_(torch.randn(inp.q.shape, device="cuda").to(inp.q.dtype))
        inp.cu[1].copy_(i32([0, ks[0] - i, sum(ks) - i]))
        graph.replay()
        eager = inp.run(R, True)
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    a = inp.run(R, True, stream=side, ws=ws, out=out, lse=lse)
    b = inp.run(R, True)
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dt,Hq,Hkv,D,qs,ks,layout", [
    ("bf16", 8, 2, 128, [300, 70], [300, 133], "packed"),
    ("bf16", 4, 4, 64, [150, 200], [150, 200], "cache"),
    ("bf16", 8, 1, 128, [40, 3], [3000, 2100], "packed"),      # keys split over blocks
    ("f32", 8, 2, 64, [90, 140], [120, 140], "packed"),
    ("f32", 4, 1, 128, [30, 7], [2001, 50], "cache"),
], ids=["bf16-D128", "bf16-D64", "bf16-split", "f32-D64", "f32-D128-split"])
def test_infinities_and_nan_reach_the_tokens_that_see_them_only(R, dt, Hq, Hkv, D, qs, ks, layout):
    """An infinity in one dimension of a value, a NaN in another value, a key of NaN, one after the other, and a query of
    NaN: tokens that see none of them, and dimensions that hold none, keep their results to the bit."""
    print("nan", dt, Hq, Hkv, D, qs, ks, layout, flush=True)
    inp = Inputs(23, dt, Hq, Hkv, D, qs, ks, layout)
    G = Hq // Hkv
    clean, clean_lse = (t.clone() for t in inp.run(R, True))
    marks = {}                       # sequence -> first tokens that see: the infinity, the NaN of a value, the key
    at = lambda t, b, j: t[b, -1, j] if layout == "cache" else t[inp.cu_k[b] + j, -1]  # noqa: E731  (the last KV head)
    for b in range(2):
        steps = sorted({qs[b] // 3, qs[b] // 2, qs[b] - 2})
        inf_t, nan_t, key_t = steps if len(steps) == 3 else (steps[0], steps[0], steps[-1])
        shift = ks[b] - qs[b]
        at(inp.V, b, inf_t + shift)[5] = -float("inf")
        at(inp.V, b, nan_t + shift)[D - 3] = float("nan")
        at(inp.K, b, key_t + shift)[7] = float("nan")
        marks[b] = inf_t, nan_t, key_t
    inp.q[inp.cu_q[0] + 1, 0, 3] = float("nan")
    out, lse = inp.run(R, True)
    torch.cuda.synchronize()
    assert torch.isnan(out[1, 0]).all() and torch.isnan(lse[1, 0])
    clean[1, 0], clean_lse[1, 0] = out[1, 0], lse[1, 0]
    if Hkv > 1:                       # the other KV heads' groups
        assert torch.equal(torch.nan_to_num(out[:, :-G]), torch.nan_to_num(clean[:, :-G]))
        assert torch.equal(torch.nan_to_num(lse[:, :-G]), torch.nan_to_num(clean_lse[:, :-G]))
    for b, (inf_t, nan_t, key_t) in marks.items():
        o, c = out[inp.cu_q[b]:inp.cu_q[b + 1], -G:], clean[inp.cu_q[b]:inp.cu_q[b + 1], -G:].clone()
        l, cl = lse[inp.cu_q[b]:inp.cu_q[b + 1], -G:], clean_lse[inp.cu_q[b]:inp.cu_q[b + 1], -G:].clone()
        c[inf_t:, :, 5] = -float("inf")
        c[nan_t:, :, D - 3] = float("nan")
        c[key_t:] = float("nan")
        cl[key_t:] = float("nan")
        if b == 0 and Hkv == 1:
            c[1, 0], cl[1, 0] = float("nan"), float("nan")
        same = (o == c) | (torch.isnan(o) & torch.isnan(c))
        assert same.all(), (b, (~same).nonzero()[:4])
        assert ((l == cl) | (torch.isnan(l) & torch.isnan(cl))).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_an_infinity_in_the_last_value_of_a_full_mask(R, dt):
    """Not causal, lengths that end inside a tile: every token gets the infinity, in its dimension alone."""
    inp = Inputs(24, dt, 4, 2, 64, [33, 5], [77, 33], "packed")
    want = inp.run(R, False)[0].clone()
    for b in range(2):
        inp.V[inp.cu_k[b + 1] - 1, :, 9] = float("inf")
    want[..., 9] = float("inf")
    got = inp.run(R, False)[0]
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_no_keys_at_all(R, dt):
    """max_k = 0, without K and V or with an empty one: every token of every sequence sees nothing."""
    q = torch.randn(5, 4, 64, device="cuda").to(DT[dt])
    empty = torch.empty(0, 2, 64, device="cuda", dtype=DT[dt])
    for causal in (False, True):
        out, lse = torch.full_like(q, 3.0), torch.full((5, 4), 3.0, device="cuda")
        R.rbq_prefill_attention(2, 4, 2, 64, q, 256, empty, empty, 128, 64, 0, 0, i32([0, 2, 5]), i32([0, 0, 0]), 5, 0, causal,
                                0.1, out, lse)
        torch.cuda.synchronize()
        assert torch.all(out == 0) and torch.all(lse == -float("inf"))


def test_plans_of_every_size_agree_with_whole_keys(R):
    """The number of splits goes by rules on the sizes: from one token to many, every plan gives the attention's value."""
    for tokens in (1, 2, 5, 17, 60, 150, 333):
        for keys in (64, 700, 2049):
            inp = Inputs(tokens + keys, "bf16", 8, 2, 64, [tokens], [max(keys, tokens)], "packed")
            out, lse = inp.run(R, True)
            torch.cuda.synchronize()
            check(inp, out, lse, True, heads=(0, 7))


@pytest.mark.parametrize("dt,Hq,Hkv,D,layout", [("bf16", 4, 1, 128, "packed"), ("f32", 2, 1, 64, "cache"), ("bf16", 6, 2, 64, "cache")])
def test_more_sequences_than_lanes_with_split_keys(R, dt, Hq, Hkv, D, layout):
    """Few tokens in each of many sequences, over anything from no keys to thousands: the keys are split, and every split of
    a tile runs, also behind its last key."""
    print("many split", dt, Hq, Hkv, D, layout, flush=True)
    rng = np.random.default_rng(12)
    qs = [int(v) for v in rng.integers(0, 3, 70)]
    ks = [int(v) for v in rng.choice([0, 1, 2, 63, 64, 65, 700, 1500, 2999, 4100], 70)]
    qs[:3], ks[:3], qs[-2:], ks[-2:] = [2, 2, 1], [0, 1, 4100], [1, 2], [4100, 2]
    inp = Inputs(31, dt, Hq, Hkv, D, qs, ks, layout)
    assert R.rbq_workspace_bytes(R.RBQ_OP_PREFILL, 70, Hq, Hkv, D, inp.max_k, inp.T) > 0
    for causal in (True, False):
        out, lse = inp.run(R, causal)
        torch.cuda.synchronize()
        check(inp, out, lse, causal)


def test_strides_of_single_tokens_and_rows(R):
    """One token of a long sequence of projections, one key row, one sequence of a cache: bitwise as contiguous."""
    from paper_2606_31519_amd import pipeline
    Hq, Hkv, D = 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(1, 1 << 15, Hq, D, device="cuda", generator=g).to(torch.bfloat16)
    K, V = (torch.randn(1, Hkv, 90, D, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    odd = [t.as_strided(t.shape, (0, 90 * D, D, 1)) for t in (K, V)]
    att = pipeline.PromptAttention(Hq, Hkv, D, [1], [90])
    got, want = att(x[:, 7], *odd), att(x[:, 7].contiguous(), K, V)
    k1, v1 = (t[0, :, 5:6].transpose(0, 1) for t in (K, V))
    one = pipeline.PromptAttention(Hq, Hkv, D, [1])
    a, b = one(x[:, 9], k1, v1), one(x[:, 9].contiguous(), k1.contiguous(), v1.contiguous())
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(a, b)
    assert torch.equal(a[0], v1[0].repeat_interleave(Hq // Hkv, dim=0))
