"""The 4-bit cache on the GPU: rows written (codes and words exactly those of the
definition), read back, and attended to, densely and sparsely, against 64 bits on the
values that the cache holds."""
import math

import numpy as np
import pytest
import torch

import kv4_util as ku
from kv8_util import attention

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def R():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2606_31519_amd import rbq
    return rbq


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def words(w):
    """Words [..][2] as a device tensor."""
    return dev(np.ascontiguousarray(w.astype(np.uint32)).view(np.int32))


def rows_like(rng, shape, dt):
    """Rows of all sizes: outlier channels, large and tiny tokens, rounded to the type; as float64."""
    x = rng.standard_normal(shape) * np.exp(rng.uniform(-3, 3, shape[:-1] + (1,)))
    x[..., rng.integers(0, shape[-1], 3)] *= 9.0
    return torch.from_numpy(x).to(DT[dt]).double().numpy()


def encoded(x, fmt):
    """Codes and words of rows x [..][D]."""
    flat = [ku.encode_row(r, fmt) for r in x.reshape(-1, x.shape[-1])]
    return (np.stack([c for c, _ in flat]).reshape(x.shape),
            np.array([w for _, w in flat], np.uint32).reshape(x.shape[:-1]))


# B, Hkv, D, cap, [(offset per sequence, rows per sequence), ...]: the writes one after another
WRITES = [
    (1, 2, 128, 300, [([0], [300])]),
    (1, 1, 64, 50, [([0], [1]), ([1], [1]), ([2], [15]), ([17], [33])]),
    (3, 2, 128, 200, [([0, 5, 64], [70, 0, 33]), ([70, 0, 97], [1, 3, 100])]),
    (2, 2, 64, 513, [([0, 0], [513, 1]), ([100, 1], [20, 130])]),                    # over rows already written
    (5, 1, 128, 257, [([0, 1, 0, 0, 0], [256, 0, 17, 1, 100])]),
]


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("case", WRITES, ids=[f"B{c[0]}-D{c[2]}-cap{c[3]}" for c in WRITES])
def test_rows_written_are_those_of_the_definition(R, case, dt, fmt):
    B, H, D, cap, writes = case
    print("write", case, dt, fmt, flush=True)
    rng = np.random.default_rng(cap + D)
    kv = rng.integers(0, 256, (B, H, cap, D)).astype(np.uint8)
    par = rng.integers(0, 1 << 31, (B, H, cap, 2)).astype(np.uint32)
    d_kv, d_par = dev(kv), words(par)
    for offs, cnts in writes:
        n = max(cnts)
        ld = n + 3
        x = [rows_like(rng, (B, H, ld, D), dt) for _ in range(2)]
        for b in range(B):
            if cnts[b] == 0:
                continue
            at = slice(offs[b], offs[b] + cnts[b])
            enc = [encoded(t[b, :, :cnts[b]], fmt) for t in x]
            kv[b, :, at] = ku.records(enc[0][0], enc[1][0], fmt)
            par[b, :, at, 0], par[b, :, at, 1] = enc[0][1], enc[1][1]
        one = len(set(offs)) == 1 and len(set(cnts)) == 1
        seqs = (None, None) if one else (dev(np.array(offs, np.int32)), dev(np.array(cnts, np.int32)))
        R.rbq_quantize_kv4(B, H, D, dev(x[0], DT[dt]), dev(x[1], DT[dt]), ld, n, max(offs), cap, R.KV4_FORMATS[fmt], d_kv,
                           d_par, *seqs)
    torch.cuda.synchronize()
    # every row, the ones that no write touched included (left as they were)
    assert np.array_equal(d_par.cpu().numpy().view(np.uint32), par)
    got = d_kv.cpu().numpy()
    if fmt == "fp4":   # (a zero may have either sign)
        fix = lambda a: np.where(ku.unpack(a, fmt) == 8, 0, ku.unpack(a, fmt))  # noqa: E731
        assert np.array_equal(fix(got), fix(kv))
    else:
        assert np.array_equal(got, kv)


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_finite_rows_of_every_size(R, D, dt, fmt):
    """Without an infinity or NaN near them (which take another way through the kernel): rows of any finite bits below a
    bound, for bounds from the least subnormal to the largest value; bounds, ties and values of one size, rows of each alone."""
    rng = np.random.default_rng(17)
    top = (1 << 15) if dt == "bf16" else (1 << 31)
    limit = 0x7F80 if dt == "bf16" else 0x7F800000                        # infinity's bits
    bounds = np.concatenate([np.geomspace(2, limit, 600).astype(np.int64), limit * np.arange(1, 256) // 255,
                             np.arange(1, 256) * (limit // 255) + (limit // 255) * 3 // 4])
    bounds = np.clip(np.repeat(bounds, 2), 2, limit)
    mag = rng.integers(0, bounds[:, None], (len(bounds), D))
    # half of the rows close to their bound in size, so that the codes spread
    near = np.maximum(bounds[:, None] - (rng.integers(0, 5, mag.shape) << (7 if dt == "bf16" else 23)) - rng.integers(1, 99, mag.shape), 0)
    mag = np.where(rng.random((len(bounds), 1)) < 0.5, mag, near)
    sign = np.where(rng.random((len(bounds), 1)) < 0.8, rng.integers(0, 2, mag.shape), rng.integers(0, 2, (len(bounds), 1)))
    bits = mag + sign * top
    x = (torch.from_numpy(bits.astype(np.uint16).view(np.int16)).view(torch.bfloat16) if dt == "bf16" else
         torch.from_numpy(bits.astype(np.uint32).view(np.float32)))
    same = [np.zeros(D), np.full(D, 0.1), np.full(D, -0.1), np.full(D, 2.0 ** 126), np.full(D, -2.0 ** 126), np.full(D, 1e-40),
            np.resize([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -0.75, -1.25, -2.5, -5.0], D),
            np.resize(np.arange(16) / 2.0, D), np.resize([1e6, 1e6 + 0.0625, 1e6 + 4], D), np.resize([-7.0, 0.0], D),
            np.resize([-2.0 ** 126, 2.0 ** 126, 1.0], D), np.resize([7 * 2.0 ** -126, 2.0 ** -127], D)]
    x = torch.cat([x, torch.from_numpy(np.repeat(np.stack(same), 8, axis=0)).to(DT[dt])])
    assert torch.all(torch.isfinite(x.float()))
    n = len(x)
    kv, par = torch.zeros(1, 1, n, D, dtype=torch.uint8, device="cuda"), torch.zeros(1, 1, n, 2, dtype=torch.int32, device="cuda")
    d = x.cuda().view(1, 1, n, D)
    R.rbq_quantize_kv4(1, 1, D, d, -d, n, n, 0, n, R.KV4_FORMATS[fmt], kv, par)
    got, p = kv.cpu().numpy()[0, 0], par.cpu().numpy().view(np.uint32)[0, 0]
    for k, v in ((0, x), (1, -x)):
        codes, word = encoded(v.double().numpy(), fmt)
        # (a base of zero may have either sign)
        zero = lambda a: np.where((a >> 16) == 0x8000, a & 0xFFFF, a) if fmt == "int4" else a  # noqa: E731
        assert np.array_equal(zero(p[:, k]), zero(word)), np.flatnonzero(zero(p[:, k]) != zero(word))[:5]
        c = ku.unpack(got[:, k * D // 2:(k + 1) * D // 2], fmt)
        if fmt == "fp4":
            c, codes = (np.where(a == 8, 0, a) for a in (c, codes))
        assert np.array_equal(c, codes), np.argwhere(c != codes)[:5]


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_extreme_values(R, D, dt, fmt):
    """Rows of zeros, of one value, of subnormals, at the type's largest and lowest value, at the format's borders and
    ties, with infinities and NaN beside ordinary values, and of nothing else; read back in both types."""
    big = float(torch.finfo(DT[dt]).max)
    rng = np.random.default_rng(3)
    rows = [np.zeros(D), np.full(D, 0.1), np.full(D, -0.1), np.full(D, big), np.full(D, -big)]
    for f in (7.0, 7.0 * 2.0 ** -9, 7.03125, 6.0, 1e-40, 2.0 ** -133, 2.0 ** -126, 2.0 ** 126, big / 2, big):
        u = rng.uniform(-1, 1, D)
        u[0] = 1.0
        rows.append(u * f)
    rows.append(np.resize([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -0.75, -1.25, -2.5, -5.0], D))   # ties of e2m1
    rows.append(np.resize(np.arange(16) / 2.0, D))                                                              # of int4
    rows.append(np.resize([1e6, 1e6 + 0.0625, 1e6 + 4], D))          # a narrow range far from 0
    rows.append(rng.uniform(0.5, 2.0, D) * 2.0 ** rng.integers(-120, 120, D))
    odd = rng.standard_normal(D)
    odd[:4] = [np.inf, -np.inf, np.nan, -np.nan]
    rows += [odd, np.resize([np.nan], D), np.resize([np.inf, -np.inf], D), np.where(np.arange(D) == 5, np.inf, 0.0),
             np.where(np.arange(D) == 9, np.nan, 3.0), -np.abs(odd)]
    x = torch.from_numpy(np.stack(rows)).to(DT[dt])
    n = len(rows)
    fc = R.KV4_FORMATS[fmt]
    kv, par = torch.zeros(1, 1, n, D, dtype=torch.uint8, device="cuda"), torch.zeros(1, 1, n, 2, dtype=torch.int32, device="cuda")
    d = x.cuda().view(1, 1, n, D)
    R.rbq_quantize_kv4(1, 1, D, d, d.flip(2).contiguous(), n, n, 0, n, fc, kv, par)
    codes, word = encoded(x.double().numpy(), fmt)
    got = kv.cpu().numpy()[0, 0]
    p = par.cpu().numpy().view(np.uint32)[0, 0]
    want = ku.row_values(codes, word, fmt)
    assert np.all(np.isfinite(want.astype(np.float32)))
    for i in range(n):
        for k, j in ((0, i), (1, n - 1 - i)):
            assert p[i, k] == word[j], (i, k, hex(p[i, k]), hex(word[j]))
            c = ku.unpack(got[i, k * D // 2:(k + 1) * D // 2], fmt)
            assert np.array_equal(ku.row_values(c, p[i, k], fmt), want[j]), (i, k)
    for out_t in (torch.float32, torch.bfloat16):
        back = [torch.full((1, 1, n, D), 7.0, dtype=out_t, device="cuda") for _ in range(2)]
        R.rbq_dequantize_kv4(1, 1, D, kv, par, fc, n, n, 0, *back, n)
        w = torch.from_numpy(want.astype(np.float32)).to(out_t)
        assert torch.equal(back[0][0, 0].cpu(), w) and torch.equal(back[1][0, 0].cpu(), w.flip(0))


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_rows_read_back(R, dt, fmt):
    """Every code under every kind of word, from ragged places; rows behind a sequence's own are left as they were."""
    B, H, D, cap = 3, 2, 128, 90
    rng = np.random.default_rng(7)
    (ck, wk), (cv, wv) = (ku.random_cache(rng, (B, H, cap), D, fmt) for _ in range(2))
    kv, par = dev(ku.records(ck, cv, fmt)), words(np.stack([wk, wv], axis=-1))
    offs, cnts = [0, 31, 40], [50, 17, 0]
    K, V = (torch.full((B, H, 53, D), 7.0, dtype=DT[dt], device="cuda") for _ in range(2))
    R.rbq_dequantize_kv4(B, H, D, kv, par, R.KV4_FORMATS[fmt], cap, 50, 40, K, V, 53, dev(np.array(offs, np.int32)),
                         dev(np.array(cnts, np.int32)))
    for got, c, w in ((K, ck, wk), (V, cv, wv)):
        want = torch.full((B, H, 53, D), 7.0, dtype=DT[dt])
        for b in range(B):
            at = slice(offs[b], offs[b] + cnts[b])
            want[b, :, :cnts[b]] = torch.from_numpy(ku.row_values(c[b, :, at], w[b, :, at], fmt).astype(np.float32)).to(DT[dt])
        assert torch.equal(got.cpu(), want)


# B, Hq, Hkv, D, cap, rows, window rows, share selected, window type
READS = [
    (1, 8, 2, 128, 3967, [3967], [129], 0.05, "bf16"),
    (2, 4, 4, 64, 1030, [1025, 1], [0, 1], 0.3, "f32"),                  # G = 1; one row; no window
    (3, 4, 2, 128, 500, [0, 500, 31], [0, 257, 4], 0.5, "bf16"),         # an empty sequence; a window of two splits
    (1, 16, 1, 128, 2100, [2049], [70], 0.02, "f32"),                    # G = 16
    (2, 16, 2, 64, 700, [640, 129], [17, 300], 0.9, "bf16"),             # G = 8, D = 64
    (2, 8, 2, 128, 40, [17, 33], [0, 0], 0.2, "bf16"),
    (1, 2, 1, 64, 64, [0], [5], 0.5, "f32"),                              # the window alone
    (1, 16, 1, 64, 300, [300], [40], 0.3, "bf16"),                        # G = 16, D = 64
    (9, 8, 2, 128, 33000, [33000, 3, 20000, 1024, 0, 15000, 777, 32768, 9], [0, 5, 64, 1, 0, 9, 3, 8, 2], 0.02, "bf16"),
]


class Reads:
    """A cache of every code, with rows that no call may read full of ones (fp4 words of them: NaN scales)."""

    def __init__(self, case, fmt):
        self.B, self.Hq, self.Hkv, self.D, self.cap, self.ns, self.ws, self.share, self.ldt = case
        B, Hq, Hkv, D, cap, ns, ws = self.B, self.Hq, self.Hkv, self.D, self.cap, self.ns, self.ws
        rng = self.rng = np.random.default_rng(cap + Hq)
        self.fmt, self.n, self.w, self.tau = fmt, max(ns), max(ws), 1.0 / math.sqrt(D)
        self.code = {k: ku.random_cache(rng, (B, Hkv, cap), D, fmt) for k in "KV"}
        self.q = rng.standard_normal((B, Hq, D)).astype(np.float32)
        self.win = {k: torch.from_numpy(rng.standard_normal((B, Hkv, self.w + 2, D))).to(DT[self.ldt]) for k in "KV"}
        rec = ku.records(self.code["K"][0], self.code["V"][0], fmt)
        par = np.stack([self.code["K"][1], self.code["V"][1]], axis=-1)
        for b in range(B):
            rec[b, :, ns[b]:] = 0xFF
            par[b, :, ns[b]:] = 0xFFFFFFFF
            for k in "KV":
                self.win[k][b, :, ws[b]:] = float("nan")
        self.kv, self.par, self.kw, self.vw = dev(rec), words(par), self.win["K"].cuda(), self.win["V"].cuda()
        self.dq = dev(self.q)
        keep = rng.random((B, Hq, cap)) < self.share
        for b in range(B):
            keep[b, :, ns[b]:] = False
        if ns[0] > 40:
            keep[0, 0] = False                       # a head that selects nothing
            keep[0, -1, :ns[0]] = True               # and, unless they are one group, a head that selects everything
        self.keep = keep
        sel = np.zeros((B, Hq, max(self.n, 1)), np.int32)
        cnt = keep.sum(axis=2).astype(np.int32)
        for b in range(B):
            for h in range(Hq):
                sel[b, h, :cnt[b, h]] = np.flatnonzero(keep[b, h])
        self.sel, self.cnt = dev(sel), dev(cnt)
        uniform = len(set(ns)) == 1 and len(set(ws)) == 1
        self.seqs = (None, None) if uniform else (dev(np.array(ns, np.int32)), dev(np.array(ws, np.int32)))

    def call(self, R, kind, out, lse, ws, stream=None):
        head = (self.B, self.Hq, self.Hkv, self.D, self.dq, self.kv, self.par, R.KV4_FORMATS[self.fmt], self.cap, self.n)
        loc = (self.kw, self.vw, self.w + 2, self.w, self.tau)
        if kind == "dense":
            R.rbq_dense_decode_kv4(*head, *loc, out, lse, ws, *self.seqs, stream=stream)
        else:
            R.rbq_sparse_decode_kv4(*head, self.sel, self.cnt, *loc, out, lse, ws, *self.seqs, stream=stream)

    def buffers(self, R):
        ws = R.workspace(R.RBQ_OP_DECODE_KV4, self.B, self.Hq, self.Hkv, self.D, self.n, self.w)
        ws.fill_(255)                                      # (NaN patterns: nothing is read before it is written)
        return (torch.full((self.B, self.Hq, self.D), 9.0, device="cuda"), torch.full((self.B, self.Hq), 9.0, device="cuda"),
                ws)

    def check(self, kind, out, lse, heads=None):
        G = self.Hq // self.Hkv
        for b in range(self.B):
            for h in (range(self.Hq) if heads is None else heads):
                rows = np.arange(self.ns[b]) if kind == "dense" else np.flatnonzero(self.keep[b, h])
                K, V, Kb, Vb = [], [], [], []
                for k, val, blk in (("K", K, Kb), ("V", V, Vb)):
                    c, w = (t[b, h // G][rows] for t in self.code[k])
                    x = self.win[k][b, h // G, :self.ws[b]].double().numpy()
                    val += [ku.exact_values(c, w, self.fmt), x]
                    blk += [ku.bulk(c, w, self.fmt), np.abs(x)]
                K, V, Kb, Vb = (np.concatenate(t) for t in (K, V, Kb, Vb))
                q = self.q[b, h].astype(np.float64)
                o, l = attention(q, K, V, self.tau)
                ot, lt = ku.attention_tolerance(q, K, V, Kb, Vb, self.tau)
                assert np.abs(out[b, h] - o).max() <= ot, (kind, b, h, np.abs(out[b, h] - o).max(), ot)
                assert (lse[b, h] == l if np.isinf(l) else abs(lse[b, h] - l) <= lt), (kind, b, h, lse[b, h], l, lt)


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("case", READS, ids=[f"B{c[0]}-G{c[1] // c[2]}-D{c[3]}-n{max(c[5])}" for c in READS])
def test_attention_over_the_cache(R, case, fmt):
    print("read", case, fmt, flush=True)
    inp = Reads(case, fmt)
    for kind in ("dense", "sparse"):
        out, lse, ws = inp.buffers(R)
        inp.call(R, kind, out, lse, ws)
        torch.cuda.synchronize()
        inp.check(kind, out.cpu().numpy(), lse.cpu().numpy(), (0, inp.Hq - 1) if inp.B > 4 else None)


@pytest.mark.parametrize("fmt", ku.FORMATS)
def test_a_selection_of_everything_is_the_dense_call(R, fmt):
    inp = Reads((1, 8, 2, 128, 777, [777], [33], 2.0, "bf16"), fmt)
    inp.keep[:] = True
    inp.sel = dev(np.tile(np.arange(777, dtype=np.int32), (1, 8, 1)))
    inp.cnt = dev(np.full((1, 8), 777, np.int32))
    for kind in ("dense", "sparse"):
        out, lse, ws = inp.buffers(R)
        inp.call(R, kind, out, lse, ws)
        inp.check(kind, out.cpu().numpy(), lse.cpu().numpy())


@pytest.mark.parametrize("fmt", ku.FORMATS)
def test_append_and_attend_in_a_graph_and_on_two_streams(R, fmt):
    """A token appended and attended to, captured once and replayed with new rows and queries (the program's own work
    between the replays), against the same calls made eagerly; and the same on a stream of its own beside another call."""
    B, Hq, Hkv, D, cap, n = 2, 8, 2, 64, 256, 100
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    K, V = rnd(B, Hkv, n, D), rnd(B, Hkv, n, D)
    fc = R.KV4_FORMATS[fmt]

    def fresh():
        kv, par = (torch.zeros(B, Hkv, cap, D, dtype=torch.uint8, device="cuda"),
                   torch.zeros(B, Hkv, cap, 2, dtype=torch.int32, device="cuda"))
        R.rbq_quantize_kv4(B, Hkv, D, K, V, n, n, 0, cap, fc, kv, par)
        return kv, par, torch.zeros(B, Hq, D, device="cuda"), torch.zeros(B, Hq, device="cuda"), \
            R.workspace(R.RBQ_OP_DECODE_KV4, B, Hq, Hkv, D, cap, 0)

    off = torch.full((B,), n, dtype=torch.int32, device="cuda")
    k1, v1, q = rnd(B, Hkv, 1, D), rnd(B, Hkv, 1, D), rnd(B, Hq, D)

    def token(st, stream=None):
        kv, par, out, lse, ws = st
        R.rbq_quantize_kv4(B, Hkv, D, k1, v1, 1, 1, cap - 1, cap, fc, kv, par, off, None, stream=stream)
        R.rbq_dense_decode_kv4(B, Hq, Hkv, D, q, kv, par, fc, cap, cap, None, None, 0, 0, 0.125, out, lse, ws, cnt, None,
                               stream=stream)

    cnt = off + 1
    ref, cap_st = fresh(), fresh()
    token(fresh())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token(cap_st)
    for i in range(5):
        k1.copy_(rnd(B, Hkv, 1, D) * 2.0 ** i)
        v1.copy_(rnd(B, Hkv, 1, D))
        q.copy_(rnd(B, Hq, D))
        off.fill_(n + i)
        cnt.fill_(n + i + 1)
        graph.replay()
        token(ref)
        torch.cuda.synchronize()
        for a, b in zip(ref[:4], cap_st[:4]):
            assert torch.equal(a, b)
    side = torch.cuda.Stream()
    a, b = fresh(), fresh()
    torch.cuda.synchronize()
    token(a, stream=side)
    token(b)
    torch.cuda.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(a[:4], b[:4]))


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("sparse", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,ldt", [(8, 2, 128, "bf16"), (16, 1, 64, "f32"), (2, 2, 128, "f32"), (16, 2, 64, "bf16"),
                                          (16, 1, 128, "bf16"), (4, 2, 64, "bf16"), (16, 2, 128, "f32")])
def test_short_contexts(R, Hq, Hkv, D, ldt, sparse, fmt):
    """Every group size, lengths from none to a few groups of rows, with and without a window; runs are bitwise alike."""
    for n, w in ((0, 0), (1, 0), (0, 1), (31, 3), (32, 0), (33, 1), (129, 17), (257, 0)):
        case = (1, Hq, Hkv, D, max(n, 1), [n], [w], 0.4, ldt)
        print("short", case, sparse, fmt, flush=True)
        inp = Reads(case, fmt)
        kind = "sparse" if sparse else "dense"
        res = []
        for _ in range(2):
            out, lse, ws = inp.buffers(R)
            inp.call(R, kind, out, lse, ws)
            torch.cuda.synchronize()
            res.append((out.cpu().numpy(), lse.cpu().numpy()))
        assert np.array_equal(res[0][0], res[1][0]) and np.array_equal(res[0][1], res[1][1])
        inp.check(kind, *res[0])


@pytest.mark.parametrize("fmt", ku.FORMATS)
@pytest.mark.parametrize("B,Hq,Hkv,D,n,w,ldt", [
    (2, 8, 2, 128, 700, 40, "bf16"),
    (2, 16, 2, 64, 700, 300, "f32"),
    (1, 16, 1, 128, 0, 17, "f32"),
    (2, 2, 2, 128, 100, 1, "bf16"),
    (1, 4, 2, 64, 60, 20, "f32"),
    (8, 32, 8, 64, 15700, 300, "bf16"),      # sparse: windows taken along by the last splits
    (8, 8, 8, 128, 15700, 200, "f32"),
])
def test_infinities_in_the_window(R, B, Hq, Hkv, D, n, w, ldt, fmt):
    """An infinity in a value of the window is the result in its dimension (one of each sign, or a NaN: NaN), and every
    other dimension, and every other KV head, keeps its bits; one in a key or a query gives its heads NaN."""
    print("inf", B, Hq, Hkv, D, n, w, ldt, fmt, flush=True)
    G, tau, cap = Hq // Hkv, 0.05, n + 1
    rng = np.random.default_rng(D + w)
    (ck, wk), (cv, wv) = (ku.random_cache(rng, (B, Hkv, cap), D, fmt) for _ in range(2))
    kv, par, fc = dev(ku.records(ck, cv, fmt)), words(np.stack([wk, wv], axis=-1)), R.KV4_FORMATS[fmt]
    q = dev(rng.standard_normal((B, Hq, D)).astype(np.float32))
    K, V = (dev(rng.standard_normal((B, Hkv, w, D)), DT[ldt]) for _ in range(2))
    sel = torch.arange(max(n, 1), dtype=torch.int32, device="cuda").expand(B, Hq, max(n, 1)).contiguous()
    cnt = torch.full((B, Hq), n // 3, dtype=torch.int32, device="cuda")
    seq_w = torch.full((B,), w, dtype=torch.int32, device="cuda")

    def run():
        res = []
        for sparse in (False, True):
            for ragged in (False, True):
                out, lse = torch.empty(B, Hq, D, device="cuda"), torch.empty(B, Hq, device="cuda")
                ws = R.workspace(R.RBQ_OP_DECODE_KV4, B, Hq, Hkv, D, n, w)
                head, loc = (B, Hq, Hkv, D, q, kv, par, fc, cap, n), (K, V, w, w, tau, out, lse, ws)
                seqs = (None, seq_w) if ragged else (None, None)
                if sparse:
                    R.rbq_sparse_decode_kv4(*head, sel, cnt, *loc, *seqs)
                else:
                    R.rbq_dense_decode_kv4(*head, *loc, *seqs)
                torch.cuda.synchronize()
                res.append((out, lse))
        return res

    same = lambda a, b: bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())  # noqa: E731
    inf, nan = float("inf"), float("nan")
    clean = run()
    b, hk = B - 1, Hkv - 1
    heads = slice(hk * G, (hk + 1) * G)
    V[b, hk, w // 2, 5], V[b, hk, w - 1, D - 1], V[b, hk, 0, 6] = inf, -inf, nan
    marks = {5: inf, D - 1: -inf, 6: nan}
    if w > 1:
        V[b, hk, 0, 7], V[b, hk, w - 1, 7] = inf, -inf
        marks[7] = nan
    if ldt == "f32":
        V[b, hk, w // 3, 8] = -3.4e38        # beyond bf16's range: counts as an infinity
        marks[8] = -inf
    got = run()
    for (out, lse), (o, l) in zip(got, clean):
        want = o.clone()
        for d, v in marks.items():
            want[b, heads, d] = v
        assert same(out, want) and torch.equal(lse, l)
    K[b, hk, w // 2, 3] = -inf
    q[0, 0, 1] = inf
    for (out, lse), (o, l) in zip(run(), got):
        want, wl = o.clone(), l.clone()
        for t in (want, wl):
            t[b, heads], t[0, 0] = nan, nan
        assert same(out, want) and same(lse, wl)


@pytest.mark.parametrize("fmt", ku.FORMATS)
def test_a_rising_maximum_and_rows_of_no_weight(R, fmt):
    """Logits that grow along the rows by hundreds, so that every group moves the maximum, and fall again; and rows whose
    step is zero or whose values are far from zero."""
    B, Hq, Hkv, D, n = 1, 4, 1, 128, 1500
    inp = Reads((B, Hq, Hkv, D, n, [n], [0], 0.5, "bf16"), fmt)
    rng = np.random.default_rng(2)
    q = np.abs(rng.standard_normal((B, Hq, D))).astype(np.float32)
    x = rng.standard_normal((2, n, D)) + np.sin(np.arange(n) / 200.0)[None, :, None] * np.array([4.0, 30.0])[:, None, None]
    x[1, 7] = 0.25                         # one value: a step of zero
    x[0, 9] = 0.0
    for i, k in enumerate("KV"):
        enc = [ku.encode_row(torch.from_numpy(r).bfloat16().double().numpy(), fmt) for r in x[i]]
        inp.code[k] = (np.stack([e[0] for e in enc])[None, None], np.array([e[1] for e in enc], np.uint32)[None, None])
    inp.kv = dev(ku.records(inp.code["K"][0], inp.code["V"][0], fmt))
    inp.par = words(np.stack([inp.code["K"][1], inp.code["V"][1]], axis=-1))
    inp.q, inp.dq, inp.tau = q, dev(q), 0.3
    for kind in ("dense", "sparse"):
        out, lse, ws = inp.buffers(R)
        inp.call(R, kind, out, lse, ws)
        inp.check(kind, out.cpu().numpy(), lse.cpu().numpy())
