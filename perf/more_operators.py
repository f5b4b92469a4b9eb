"""The measured operators of the 4-bit K/V cache.

A case is one call pattern (`kind`) at one shape:

  cache   new rows written into the 4-bit cache and read back
          (rbq_quantize_kv4, rbq_dequantize_kv4)
  dense   decode attention over every row of the 4-bit cache and a window of
          recent rows in full precision (rbq_dense_decode_kv4)
  sparse  the same over each head's selected rows (rbq_sparse_decode_kv4)
  chunk   attention of chunks of prompts over cached 4-bit rows and, causally,
          over the chunks' own rows in full precision (rbq_prefill_attention_kv4)

A cached row of one KV head is a record of D bytes, D / 2 of K's codes and D / 2 of V's,
and two 32-bit words of parameters, K's and V's:

  fp4   e2m1 codes, dimension d in bits 4 (d % 2) .. of byte d / 2; byte g of the word is the
        exponent of group g of D / 4 dimensions: a value is e2m1 * 2^(byte - 127)
  int4  whole numbers c of 0 to 15, dimension d in nibble (d % 8) / 2 + 4 (d % 2) of the 32-bit
        word d / 8; the word is a bf16 step s (low half) and a bf16 base m: a value is c s + m

Where `own` is false the operators run in their plain form, elementary torch
operations; where it is true, as a user of the library calls them. Inputs are
drawn on the GPU from the seed.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
TINY, MOST = 2.0 ** -126, 2.0 ** 126
# where the dimensions of eight lie among the nibbles of a word, int4
NIBBLE = [d // 2 + 4 * (d % 2) for d in range(8)]


def _cache(name, B, Hkv, D, new, held, fmt, kv="bf16", ragged=False):
    c = dict(kind="cache", B=B, Hkv=Hkv, D=D, new=new, held=held, fmt=fmt, kv=kv, ragged=ragged)
    return c if name is None else dict(c, name=name)


def _decode(name, kind, B, Hq, Hkv, D, n, w, fmt, kv="bf16", ragged=False, share=1.0):
    c = dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, D=D, n=n, w=w, fmt=fmt, kv=kv, ragged=ragged)
    if kind == "sparse":
        c["share"] = share   # of the keys that one head selects
    return c if name is None else dict(c, name=name)


def _chunk(name, B, Hq, Hkv, D, q, n, fmt, kv="bf16", causal=True):
    c = dict(kind="chunk", B=B, Hq=Hq, Hkv=Hkv, D=D, q=q, n=n, fmt=fmt, kv=kv, causal=causal)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the K and V of a 128K prompt (8 KV heads of 128) into an fp4 cache
        _cache("cache4_128k_fp4", 1, 8, 128, 130816, 0, "fp4"),
        # a serving batch whose windows are full: up to 256 rows each, behind contexts of any length, as int4
        _cache("cache4_16x256_int4", 16, 8, 128, 256, 4000, "int4", ragged=True),
        # one token for each of eight sequences, fp32 rows: the smallest call, all latency
        _cache("cache4_token_f32", 8, 2, 64, 1, 1000, "int4", kv="f32"),
        # one token of a chat, 32 query heads over 8 KV heads, a prompt of no particular length
        _decode("dense4_4k", "dense", 1, 32, 8, 128, 3967, 129, "fp4"),
        # the long-context token over everything: 128K rows and a 256-row window
        _decode("dense4_128k_int4", "dense", 1, 32, 8, 128, 130816, 256, "int4"),
        # a serving batch of 16 sequences of 2K to 32K, windows of their own
        _decode("dense4_ragged_16x32k", "dense", 16, 32, 8, 128, 32512, 256, "fp4", ragged=True),
        # the long-context token over a Top-p selection (a fifth of the keys per head, 59 % of the rows per group)
        _decode("sparse4_128k", "sparse", 1, 32, 8, 128, 130816, 256, "fp4", share=0.2),
        # head dimension 64, two percent of the keys, fp32 window
        _decode("sparse4_64k_d64_int4", "sparse", 1, 32, 8, 64, 65521, 97, "int4", kv="f32", share=0.02),
        # a serving batch of wide heads (64 over 8), sequences of 2K to 32K
        _decode("sparse4_ragged_8x32k_wide", "sparse", 8, 64, 8, 128, 32512, 200, "int4", ragged=True, share=0.03),
        # the next turn of a long chat: 2000 tokens over 30000 cached rows
        _chunk("chunk4_2000_30k", 1, 32, 8, 128, 2001, 30011, "fp4"),
        # drafted tokens of eight sequences, up to 7 each, checked against up to 8000 cached rows
        _chunk("chunk4_8x7_8k_int4", 8, 32, 8, 128, 7, 8000, "int4"),
        # chunks of two prompts over their cached rows, D = 64, fp32
        _chunk("chunk4_f32_d64_int4", 2, 8, 2, 64, 500, 6000, "int4", kv="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["cache", "dense", "sparse", "chunk"])
    D = rng.choice([128, 128, 64])
    kv = rng.choice(["bf16", "bf16", "f32"])
    fmt = rng.choice(["fp4", "int4"])
    Hkv = rng.choice([1, 2, 4, 8])
    Hq = Hkv * rng.choice([1, 2, 4, 8, 16])
    B = _log(rng, 1, 16)
    ragged = rng.random() < 0.5
    if kind == "cache":
        new = _log(rng, 1, max(2, 8 * 65536 // (B * Hkv)))
        held = _log(rng, 1, 5000) if rng.random() < 0.6 else 0
        return _cache(None, B, Hkv, D, new, held, fmt, kv, ragged)
    if kind in ("dense", "sparse"):
        n = _log(rng, 1, max(2, 8 * 131072 // (B * Hq)))
        w = rng.choice([0, _log(rng, 1, 512)])
        return _decode(None, kind, B, Hq, Hkv, D, n, w, fmt, kv, ragged, round(math.exp(rng.uniform(-6, -0.5)), 4))
    # queries x keys x heads, padded to the longest sequence, stay under a quarter of the largest listed case's
    most = 2001 * 32012 * 8 // (B * Hq)
    if kv == "f32":
        most //= 8
    q = _log(rng, 1, max(1, min(3000, math.isqrt(most))))
    n = rng.choice([0, _log(rng, 1, max(1, min(65536, most // q - q)))]) if most // q > q else 0
    return _chunk(None, B, Hq, Hkv, D, q, n, fmt, kv, rng.random() < 0.8)


# ---------------------------------------------------------------- lengths
def _spread(B, lo, hi, r):
    """B lengths spread evenly over [lo, hi], in the seed's order."""
    v = [int(round(lo + (hi - lo) * (i + 0.5) / B)) for i in range(B)]
    r.shuffle(v)
    return v


def _even(B, lo, hi):
    return _spread(B, lo, hi, random.Random(0))


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------- the 4-bit format, plain
def _encode(x, fmt):
    """Codes (uint8 of 0 to 15) and parameter words (int32) of rows x [..][D]."""
    D = x.shape[-1]
    x = x.float()
    fin = torch.isfinite(x)
    x = torch.nan_to_num(x, nan=0.0, posinf=math.inf, neginf=-math.inf)
    zero = torch.zeros((), device=DEV)
    if fmt == "fp4":
        amax = torch.where(fin, x.abs(), zero).unflatten(-1, (4, D // 4)).amax(dim=-1)
        m, e = torch.frexp(amax)                                   # amax = m 2^e, m in [0.5, 1); 7 = 0.875 * 2^3
        e = (e - 3 + (m > 0.875)).clamp(min=-126, max=125)
        byte = torch.where(amax > 0, e + 127, torch.zeros_like(e)).int()
        r = ((127 - e).int() << 23).view(torch.float32)            # 2^-e by its bits
        y = (x.unflatten(-1, (4, D // 4)) * r[..., None]).flatten(-2)
        y = torch.where((byte > 0)[..., None].expand(*byte.shape, D // 4).flatten(-2), y, zero)
        a = y.abs().clamp(max=6.0)
        step = torch.where(a >= 4, 2.0, torch.where(a >= 2, 1.0, 0.5))
        a = ((a / step).round() * step).clamp(max=6.0)
        code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4))   # 0 .5 1 1.5 2 3 4 6 -> 0 .. 7
        code = code.to(torch.uint8) + 8 * torch.signbit(y).to(torch.uint8)
        return code, byte[..., 0] | byte[..., 1] << 8 | byte[..., 2] << 16 | byte[..., 3] << 24
    lim = x.clamp(-MOST, MOST)
    lo = torch.where(fin, lim, torch.full_like(lim, math.inf)).amin(dim=-1)
    hi = torch.where(fin, lim, torch.full_like(lim, -math.inf)).amax(dim=-1)
    some = fin.any(dim=-1)
    lo, hi = torch.where(some, lo, zero), torch.where(some, hi, zero)
    u = lo.view(torch.int32)
    m = torch.where(u < 0, u + 0xFFFF, u) & -65536                 # to bf16, away from 0 where negative: down
    d = hi - m.view(torch.float32)
    u = (d / torch.full_like(d, 15.0)).clamp(min=TINY).view(torch.int32)   # (divided by a tensor: by a number, torch multiplies)
    s = torch.where(d > 0, (u + 0xFFFF) & -65536, torch.zeros_like(u))
    sf, mf = s.view(torch.float32), m.view(torch.float32)
    r = torch.where(sf > 0, 1.0 / sf, zero)
    y = torch.nan_to_num((x - mf[..., None]).double() * r[..., None].double(), nan=0.0, posinf=math.inf, neginf=-math.inf)
    return y.round().clamp(0, 15).to(torch.uint8), (s >> 16) & 0xFFFF | m


def _pack(code, fmt):
    """Codes [..][D] as bytes [..][D / 2]."""
    if fmt == "int4":
        code = code.unflatten(-1, (-1, 8))[..., [NIBBLE.index(p) for p in range(8)]].flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4


def _values(code, par, fmt):
    """The values, in 32 bits, that bytes [..][D / 2] and words [..] stand for."""
    n = torch.stack([code & 15, code >> 4], dim=-1).flatten(-2)
    D = n.shape[-1]
    if fmt == "fp4":
        a = (n & 7).float()
        a = torch.where(a < 4, a / 2, torch.where(a < 6, a - 2, 2 * a - 8))
        a = torch.where(n >= 8, -a, a)
        byte = torch.stack([(par >> 8 * g) & 255 for g in range(4)], dim=-1)
        s = (byte << 23).view(torch.float32)                       # 2^(byte - 127) by its bits (0 of a group of zeros)
        return (a.unflatten(-1, (4, D // 4)) * s[..., None]).flatten(-2)
    n = n.unflatten(-1, (-1, 8))[..., NIBBLE].flatten(-2)
    s, m = (par << 16).view(torch.float32), (par & -65536).view(torch.float32)
    return (n.double() * s[..., None].double() + m[..., None].double()).float()   # (one rounding)


def _filled(K, V, fmt):
    """The cache holding rows K, V [B][H][R][D]: records [B][H][R][D] bytes, words [B][H][R][2]."""
    B, H, R, D = K.shape
    codes = torch.empty(B, H, R, D, dtype=torch.uint8, device=DEV)
    par = torch.empty(B, H, R, 2, dtype=torch.int32, device=DEV)
    step = max(64, (1 << 24) // (H * D))
    for b in range(B):
        for r in range(0, R, step):
            for i, x in enumerate((K, V)):
                c, p = _encode(x[b, :, r:r + step], fmt)
                codes[b, :, r:r + step, i * D // 2:(i + 1) * D // 2] = _pack(c, fmt)
                par[b, :, r:r + step, i] = p
    return codes, par


def _cached(st, n):
    """K and V of rows [0, n) in 32 bits."""
    D, fmt = st["case"]["D"], st["case"]["fmt"]
    return [_values(st["kv4"][:, :, :n, i * D // 2:(i + 1) * D // 2], st["par"][:, :, :n, i], fmt) for i in range(2)]


# ---------------------------------------------------------------- inputs
def _rows(g, shape, dt):
    """Keys or values with four outlier channels and some tokens larger than the rest."""
    D = shape[-1]
    ch = torch.ones(D, device=DEV)
    ch[torch.randperm(D, device=DEV, generator=g)[:4]] = 4.0
    x = torch.empty(shape, dtype=dt, device=DEV)
    for b in range(shape[0]):
        tok = 1.0 + 2.0 * (torch.rand(shape[1:-1] + (1,), device=DEV, generator=g) < 0.02)
        x[b] = (torch.randn(shape[1:], device=DEV, generator=g) * ch * tok).to(dt)
    return x


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = random.Random(seed)
    B, Hkv, D, kind, dt, fmt = case["B"], case["Hkv"], case["D"], case["kind"], TYPE[case["kv"]], case["fmt"]
    st = {"case": case}
    if kind == "cache":
        new, held = case["new"], case["held"]
        offs = _spread(B, held / 16, held, r) if case["ragged"] else [held] * B
        cnts = _spread(B, new / 16, new, r) if case["ragged"] else [new] * B
        cnts = [max(1, c) for c in cnts]
        cap = held + new
        st.update(cap=cap, kv4=torch.zeros(B, Hkv, cap, D, dtype=torch.uint8, device=DEV),
                  par=torch.zeros(B, Hkv, cap, 2, dtype=torch.int32, device=DEV),
                  off=_i32(offs), cnt=_i32(cnts), host=(offs, cnts))
        for k in "KV":
            st[k] = _rows(g, (B, Hkv, new, D), dt)
            st[k + "_back"] = torch.zeros(B, Hkv, new, D, dtype=dt, device=DEV)
        return st
    Hq, n = case["Hq"], case["n"]
    K, V = (_rows(g, (B, Hkv, n, D), torch.bfloat16) for _ in range(2))
    st["kv4"], st["par"] = _filled(K, V, fmt)
    del K, V
    if kind == "chunk":
        qs = [max(1, v) for v in (_spread(B, case["q"] / 16, case["q"], r) if B > 1 else [case["q"]])]
        ns = _spread(B, n / 16, n, r) if B > 1 else [n]
        cu = np.cumsum([0] + qs).tolist()
        T = cu[-1]
        st.update(q=(1.2 * torch.randn(T, Hq, D, device=DEV, generator=g)).to(dt), K=_rows(g, (1, T, Hkv, D), dt)[0],
                  V=_rows(g, (1, T, Hkv, D), dt)[0], cu=_i32(cu), seq_n=_i32(ns), host=(qs, ns), T=T)
        return st
    w = case["w"]
    ns = [max(1, v) for v in _spread(B, n / 16, n, r)] if case["ragged"] else [n] * B
    ws = _spread(B, 0, w, r) if case["ragged"] else [w] * B
    for k in "KV":
        st[k + "w"] = _rows(g, (B, Hkv, max(w, 1), D), dt)
    st.update(q=1.2 * torch.randn(B, Hq, D, device=DEV, generator=g), host=(ns, ws), seq_n=_i32(ns), seq_w=_i32(ws))
    if kind == "sparse":
        live = torch.arange(n, device=DEV)[None, None, :] < st["seq_n"][:, None, None]
        keep = (torch.rand(B, Hq, n, device=DEV, generator=g) < case["share"]) & live
        keep[:, :, 0] = True
        cnt = keep.sum(dim=2)
        sel = torch.zeros(B, Hq, n, dtype=torch.int32, device=DEV)
        sel[torch.arange(n, device=DEV)[None, None, :] < cnt[:, :, None]] = keep.nonzero()[:, 2].int()
        st.update(sel_idx=sel, sel_count=cnt.int())
    return st


# ---------------------------------------------------------------- plain forms
def _run_cache(st):
    c = st["case"]
    D, fmt, new = c["D"], c["fmt"], c["new"]
    i = torch.arange(new, device=DEV)
    row = (st["off"][:, None] + i).long()                                   # cache rows of the new ones
    live = i[None] < st["cnt"][:, None]
    bi = torch.arange(c["B"], device=DEV)[:, None]
    was = (st["kv4"][bi, :, row], st["par"][bi, :, row])                    # [B][new][H][..]
    l4 = live[:, :, None, None]
    codes, words = [], []
    for k in "KV":
        code, par = _encode(st[k], fmt)
        codes.append(_pack(code, fmt))
        words.append(par)
    rec, wd = torch.cat(codes, dim=-1).transpose(1, 2), torch.stack(words, dim=-1).transpose(1, 2)
    st["kv4"][bi, :, row] = torch.where(l4, rec, was[0])
    st["par"][bi, :, row] = torch.where(l4, wd, was[1])
    rec, wd = st["kv4"][bi, :, row].transpose(1, 2), st["par"][bi, :, row].transpose(1, 2)
    res = {}
    for j, k in enumerate("KV"):
        val = _values(rec[..., j * D // 2:(j + 1) * D // 2], wd[..., j], fmt).to(TYPE[c["kv"]])
        res[k] = torch.where(live[:, None, :, None], val, torch.zeros_like(val))
    return res


def _attend(q, K, V, keep, tau):
    """q [..][M][D], K and V [..][N][D], keep [..][M][N]: softmax attention in 32 bits; rows that keep nothing give 0."""
    S = torch.matmul(q, K.transpose(-1, -2).contiguous()).mul_(tau).masked_fill_(~keep, -math.inf)
    m = S.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = S.sub_(m).exp_()
    l = P.sum(dim=-1, keepdim=True)
    out = torch.matmul(P, V) / l.clamp(min=1e-38)
    return out, (m + l.log())[..., 0]


def _run_decode(st):
    c = st["case"]
    B, Hq, Hkv, D, n, w = (c[k] for k in ("B", "Hq", "Hkv", "D", "n", "w"))
    G = Hq // Hkv
    pos = torch.arange(n, device=DEV)
    keep = (pos[None, :] < st["seq_n"][:, None])[:, None, None].expand(B, Hkv, G, n)
    if c["kind"] == "sparse":
        live = pos[None, None, :] < st["sel_count"][:, :, None]
        sel = torch.zeros(B, Hq, n + 1, dtype=torch.bool, device=DEV)
        sel.scatter_(2, torch.where(live, st["sel_idx"], n).long(), True)
        keep = sel[:, :, :n].view(B, Hkv, G, n)
    inw = (torch.arange(w, device=DEV)[None, :] < st["seq_w"][:, None])[:, None, None].expand(B, Hkv, G, w)
    keep = torch.cat([keep, inw], dim=3)
    kv = [torch.cat([x, st[k + "w"][:, :, :w].float()], dim=2) for x, k in zip(_cached(st, n), "KV")]
    out, lse = _attend(st["q"].view(B, Hkv, G, D), kv[0], kv[1], keep, 1.0 / math.sqrt(D))
    return {"out": out.reshape(B, Hq, D), "lse": lse.reshape(B, Hq)}


def _run_chunk(st):
    c = st["case"]
    B, Hq, Hkv, D, n = (c[k] for k in ("B", "Hq", "Hkv", "D", "n"))
    G, Lq = Hq // Hkv, max(st["host"][0])
    cu = st["cu"].long()
    nq, nk = cu[1:] - cu[:-1], st["seq_n"]
    i, j = torch.arange(Lq, device=DEV), torch.arange(n, device=DEV)
    tok = torch.where(i[None] < nq[:, None], cu[:-1, None] + i, 0)                        # [B][Lq]
    q = st["q"].float()[tok].view(B, Lq, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Lq, D)
    K, V = (torch.cat([x, st[k].float()[tok].transpose(1, 2)], dim=2) for x, k in zip(_cached(st, n), "KV"))
    mine = i[None, None] < nq[:, None, None]                                              # [B][1][Lq] of the chunk's own keys
    if c["causal"]:
        mine = mine & (i[None, None] <= i[None, :, None])
    keep = torch.cat([(j[None] < nk[:, None])[:, None].expand(B, Lq, n), mine.expand(B, Lq, Lq)], dim=2)
    keep = keep[:, None, None].expand(B, Hkv, G, Lq, n + Lq).reshape(B, Hkv, G * Lq, n + Lq)
    out, lse = _attend(q, K, V, keep, 1.0 / math.sqrt(D))
    # token t of the packed axis: its sequence and place there
    t = torch.arange(st["T"], device=DEV)
    b = torch.searchsorted(cu, t, right=True) - 1
    k = t - cu[b]
    out = out.view(B, Hkv, G, Lq, D).permute(0, 3, 1, 2, 4).reshape(B, Lq, Hq, D)[b, k]
    lse = lse.view(B, Hkv, G, Lq).permute(0, 3, 1, 2).reshape(B, Lq, Hq)[b, k]
    return {"out": out.to(TYPE[c["kv"]]), "lse": lse}


# ---------------------------------------------------------------- as a user calls them
def _own_cache(st):
    from paper_2606_31519_amd import rbq
    c = st["case"]
    B, Hkv, D, new, held = (c[k] for k in ("B", "Hkv", "D", "new", "held"))
    seqs = (st["off"], st["cnt"]) if c["ragged"] else (None, None)
    fmt = rbq.KV4_FORMATS[c["fmt"]]
    rbq.rbq_quantize_kv4(B, Hkv, D, st["K"], st["V"], new, new, held, st["cap"], fmt, st["kv4"], st["par"], *seqs)
    rbq.rbq_dequantize_kv4(B, Hkv, D, st["kv4"], st["par"], fmt, st["cap"], new, held, st["K_back"], st["V_back"], new,
                           *seqs)
    return {"K": st["K_back"], "V": st["V_back"]}


def _own_decode(st):
    from paper_2606_31519_amd import rbq
    c = st["case"]
    B, Hq, Hkv, D, n, w = (c[k] for k in ("B", "Hq", "Hkv", "D", "n", "w"))
    if "ws" not in st:   # a serving loop keeps its workspace and outputs
        st["ws"] = rbq.workspace(rbq.RBQ_OP_DECODE_KV4, B, Hq, Hkv, D, n, w)
        st["out"], st["lse"] = torch.empty(B, Hq, D, device=DEV), torch.empty(B, Hq, device=DEV)
    seqs = (st["seq_n"], st["seq_w"]) if c["ragged"] else (None, None)
    cache = (st["kv4"], st["par"], rbq.KV4_FORMATS[c["fmt"]], n, n)
    tail = (st["Kw"], st["Vw"], max(w, 1), w, 1.0 / math.sqrt(D), st["out"], st["lse"], st["ws"])
    if c["kind"] == "dense":
        rbq.rbq_dense_decode_kv4(B, Hq, Hkv, D, st["q"], *cache, *tail, *seqs)
    else:
        rbq.rbq_sparse_decode_kv4(B, Hq, Hkv, D, st["q"], *cache, st["sel_idx"], st["sel_count"], *tail, *seqs)
    return {"out": st["out"], "lse": st["lse"]}


def _own_chunk(st):
    from paper_2606_31519_amd import rbq
    c = st["case"]
    B, Hq, Hkv, D, n, T = c["B"], c["Hq"], c["Hkv"], c["D"], c["n"], st["T"]
    if "ws" not in st:
        st["ws"] = rbq.workspace(rbq.RBQ_OP_PREFILL_KV4, B, Hq, Hkv, D, n, T)
        st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty(T, Hq, device=DEV)
    # strides of a query's, and of a new K / V row and head; rows of the cache per sequence, and the most that one holds
    rbq.rbq_prefill_attention_kv4(B, Hq, Hkv, D, st["q"], Hq * D, st["K"], st["V"], Hkv * D, D, st["cu"], T, st["kv4"],
                                  st["par"], rbq.KV4_FORMATS[c["fmt"]], n, n, st["seq_n"], c["causal"], 1.0 / math.sqrt(D),
                                  st["out"], st["lse"], st["ws"])
    return {"out": st["out"], "lse": st["lse"]}


def run(state):
    kind = state["case"]["kind"]
    if kind == "cache":
        return _own_cache(state) if own else _run_cache(state)
    if kind == "chunk":
        return _own_chunk(state) if own else _run_chunk(state)
    return _own_decode(state) if own else _run_decode(state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    B, Hkv, D, kind = case["B"], case["Hkv"], case["D"], case["kind"]
    el = 2 if case["kv"] == "bf16" else 4
    if kind == "cache":
        cnts = [max(1, c) for c in _even(B, case["new"] / 16, case["new"])] if case["ragged"] else [case["new"]] * B
        new = sum(cnts) * Hkv
        # new rows in, their records and words out, the rows back
        return {"bytes": new * (2 * D * el + D + 8 + 2 * D * el), "flops": 2 * new * 2 * D * 2}
    Hq, n = case["Hq"], case["n"]
    if kind in ("dense", "sparse"):
        w = case["w"]
        ns = sum(max(1, v) for v in _even(B, n / 16, n)) if case["ragged"] else B * n
        ws = sum(_even(B, 0, w)) if case["ragged"] else B * w
        f = case.get("share", 1.0)
        union = 1.0 - (1.0 - f) ** (Hq // Hkv)
        by = Hkv * (ns * union * (D + 8) + 2 * ws * D * el) + B * Hq * D * 8 + B * Hq * 4
        if kind == "sparse":
            by += 4 * Hq * ns * f
        return {"bytes": int(by), "flops": int(4 * D * Hq * (ns * f + ws))}
    qs = [max(1, v) for v in (_even(B, case["q"] / 16, case["q"]) if B > 1 else [case["q"]])]
    ns = _even(B, n / 16, n) if B > 1 else [n]
    mean = sum(ns) / B                              # (their order goes by the seed)
    pairs = sum(a * (mean + ((a + 1) / 2 if case["causal"] else a)) for a in qs)
    by = (2 * sum(qs) * Hq * D + 2 * sum(qs) * Hkv * D) * el + 4 * sum(qs) * Hq + sum(ns) * Hkv * (D + 8)
    return {"bytes": int(by), "flops": int(4 * D * Hq * pairs)}


# ---------------------------------------------------------------- the same in 64 bits
def _pow2(e):
    """2^e of whole numbers e by its bits (the GPU's pow rounds)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _bf16_toward(x, up):
    """x, in 64 bits, on the grid of bf16's eight bits, rounded up or down."""
    a = x.abs().clamp(min=TINY)
    step = _pow2(torch.frexp(a)[1] - 8)
    return (torch.ceil(x / step) if up else torch.floor(x / step)) * step


def _exact_stored(x, fmt):
    """The values that finite rows x [..][D] (in 64 bits) are stored as."""
    if fmt == "fp4":
        y = x.unflatten(-1, (4, -1))
        amax = y.abs().amax(dim=-1, keepdim=True)
        e = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -130) / 7.0)).to(torch.int64).clamp(-126, 125)
        e = torch.where((e > -126) & (amax <= 7.0 * _pow2(e - 1)), e - 1, e)   # (where log2 rounded across a whole number)
        e = torch.where((e < 125) & (amax > 7.0 * _pow2(e)), e + 1, e)
        z = y / _pow2(e)
        grid = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
        mid = (grid[1:] + grid[:-1]) / 2
        k = torch.bucketize(z.abs().contiguous(), mid)                         # first midpoint that is not below
        tie = (k < 7) & (z.abs() == mid[k.clamp(max=6)]) & (k % 2 == 1)        # halfway and odd: to the even code above
        return (torch.sign(z) * grid[k + tie.long()] * _pow2(e)).flatten(-2)
    lo, hi = x.amin(dim=-1, keepdim=True), x.amax(dim=-1, keepdim=True)
    m = _bf16_toward(lo, False)
    d = (hi - m).float().double()
    s = torch.where(d > 0, _bf16_toward((d / 15.0).float().double(), True).clamp(min=TINY), torch.zeros_like(d))
    r = torch.where(s > 0, (1.0 / s).float().double(), torch.zeros_like(s))    # (held in 32 bits, as the difference is)
    return torch.round((x - m).float().double() * r).clamp(0, 15) * s + m


def _exact_values(code, par, fmt):
    """The values of records [..][D / 2] and words [..], in 64 bits."""
    if fmt == "fp4":
        grid = torch.tensor(E2M1 + [-v for v in E2M1], dtype=torch.float64, device=code.device)
        v = grid[torch.stack([code % 16, code // 16], dim=-1).long()].flatten(-2)
        byte = torch.stack([par.long() // 256 ** g % 256 for g in range(4)], dim=-1)
        return v * _pow2(byte - 127).repeat_interleave(v.shape[-1] // 4, dim=-1)
    w = code.contiguous().view(torch.int32).long()
    c = torch.stack([(w >> 4 * (d // 2 + 4 * (d % 2))) % 16 for d in range(8)], dim=-1).flatten(-2).double()
    s, m = ((par.long() % 65536 << 16).int().view(torch.float32), (par.long() // 65536 << 16).int().view(torch.float32))
    return c * s.double()[..., None] + m.double()[..., None]


def _exact_rows(q, K, V, keep, tau):
    """Attention of q [M][D] over K, V [N][D] with keep [M][N]."""
    lg = torch.matmul(q, K.t().contiguous()) * tau
    lg = torch.where(keep, lg, torch.full((), -math.inf, dtype=lg.dtype, device=DEV))
    L = torch.logsumexp(lg, dim=1)
    return torch.matmul(torch.exp(lg - L[:, None]), V), L


def exact(case, seed):
    st = prepare(case, seed)
    kind, B, Hkv, D, fmt = case["kind"], case["B"], case["Hkv"], case["D"], case["fmt"]
    if kind == "cache":
        res = {}
        for k in "KV":
            res[k] = torch.zeros(B, Hkv, case["new"], D, dtype=torch.float64, device=DEV)
            for b, cnt in enumerate(st["host"][1]):
                for lo in range(0, cnt, 8192):
                    hi = min(cnt, lo + 8192)
                    res[k][b, :, lo:hi] = _exact_stored(st[k][b, :, lo:hi].double(), fmt)
        return res
    Hq, tau = case["Hq"], float(np.float32(1.0 / math.sqrt(D)))
    G = Hq // Hkv

    def held(b, h, n):
        return [_exact_values(st["kv4"][b, h, :n, i * D // 2:(i + 1) * D // 2], st["par"][b, h, :n, i], fmt) for i in range(2)]

    if kind == "chunk":
        out = torch.empty(st["T"], Hq, D, dtype=torch.float64, device=DEV)
        lse = torch.empty(st["T"], Hq, dtype=torch.float64, device=DEV)
        t0 = 0
        for b, (nq, nb) in enumerate(zip(*st["host"])):
            i, j = torch.arange(nq, device=DEV)[:, None], torch.arange(nb + nq, device=DEV)[None]
            keep = (j <= i + nb) if case["causal"] else torch.ones(nq, nb + nq, dtype=torch.bool, device=DEV)
            for h in range(Hkv):
                K, V = (torch.cat([x, st[k][t0:t0 + nq, h].double()]) for x, k in zip(held(b, h, nb), "KV"))
                for g in range(h * G, h * G + G):
                    out[t0:t0 + nq, g], lse[t0:t0 + nq, g] = _exact_rows(st["q"][t0:t0 + nq, g].double(), K, V, keep, tau)
            t0 += nq
        return {"out": out, "lse": lse}
    out = torch.empty(B, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.empty(B, Hq, dtype=torch.float64, device=DEV)
    for b, (nb, wb) in enumerate(zip(*st["host"])):
        for h in range(Hkv):
            K, V = (torch.cat([x, st[k + "w"][b, h, :wb].double()]) for x, k in zip(held(b, h, nb), "KV"))
            at = slice(h * G, h * G + G)
            keep = torch.ones(G, nb + wb, dtype=torch.bool, device=DEV)
            if kind == "sparse":
                keep[:, :nb] = False
                for g in range(G):
                    keep[g, st["sel_idx"][b, h * G + g, :int(st["sel_count"][b, h * G + g])].long()] = True
            out[b, at], lse[b, at] = _exact_rows(st["q"][b, at].double(), K, V, keep, tau)
    return {"out": out, "lse": lse}
