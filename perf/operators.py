"""The measured operators of the 8-bit K/V cache and of the prompt's attention.

A case is one call pattern (`kind`) at one shape:

  cache   new rows written into the 8-bit cache (one scale per sequence, KV head
          and block of tokens) and the blocks they touch read back
          (rbq_quantize_kv, rbq_dequantize_kv)
  dense   decode attention over every row of the 8-bit cache and a window of
          recent rows in full precision (rbq_dense_decode_kv8)
  sparse  the same over each head's selected rows (rbq_sparse_decode_kv8)
  prompt  attention of whole prompts, or of chunks of them over cached rows
          (rbq_prefill_attention)

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
CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
TINY = 2.0 ** -126


def _cache(name, B, Hkv, D, new, held, block, fmt, kv="bf16", ragged=False):
    c = dict(kind="cache", B=B, Hkv=Hkv, D=D, new=new, held=held, block=block, fmt=fmt, kv=kv, ragged=ragged)
    return c if name is None else dict(c, name=name)


def _decode(name, kind, B, Hq, Hkv, D, n, w, block, fmt, kv="bf16", ragged=False, share=1.0):
    c = dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, D=D, n=n, w=w, block=block, fmt=fmt, kv=kv, ragged=ragged)
    if kind == "sparse":
        c["share"] = share   # of the keys that one head selects
    return c if name is None else dict(c, name=name)


def _prompt(name, B, Hq, Hkv, D, q, ctx, kv="bf16", causal=True, layout="packed"):
    c = dict(kind="prompt", B=B, Hq=Hq, Hkv=Hkv, D=D, q=q, ctx=ctx, kv=kv, causal=causal, layout=layout)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the K and V of a 128K prompt of the 8B-model shape (8 KV heads of 128) into an e4m3 cache
        _cache("cache_128k_e4m3", 1, 8, 128, 130816, 0, 64, "e4m3"),
        # a serving batch whose windows are full: up to 256 rows each, behind contexts of any length, as int8
        _cache("cache_16x256_int8", 16, 8, 128, 256, 4000, 32, "int8", ragged=True),
        # one token for each of eight sequences, fp32 rows: the smallest call, all latency
        _cache("cache_token_f32", 8, 2, 64, 1, 1000, 16, "e4m3", kv="f32"),
        # one token of a chat, 32 query heads over 8 KV heads, a prompt of no particular length
        _decode("dense_4k", "dense", 1, 32, 8, 128, 3967, 129, 64, "e4m3"),
        # the long-context token over everything: 128K rows and a 256-row window
        _decode("dense_128k", "dense", 1, 32, 8, 128, 130816, 256, 64, "e4m3"),
        # a serving batch of 16 sequences of 2K to 32K, windows of their own, int8
        _decode("dense_ragged_16x32k_int8", "dense", 16, 32, 8, 128, 32512, 256, 128, "int8", ragged=True),
        # the long-context token over a Top-p selection (a fifth of the keys per head, 59 % of the rows per group)
        _decode("sparse_128k", "sparse", 1, 32, 8, 128, 130816, 256, 64, "e4m3", share=0.2),
        # head dimension 64, two percent of the keys, fp32 window, int8
        _decode("sparse_64k_d64_int8", "sparse", 1, 32, 8, 64, 65521, 97, 32, "int8", kv="f32", share=0.02),
        # a serving batch of wide heads (64 over 8), sequences of 2K to 32K
        _decode("sparse_ragged_8x32k_wide", "sparse", 8, 64, 8, 128, 32512, 200, 16, "e4m3", ragged=True, share=0.03),
        # eight chat prompts of 43 to 650 tokens packed together
        _prompt("prompt_8x700", 8, 32, 8, 128, 701, 0),
        # one long prompt, whole
        _prompt("prompt_16k", 1, 32, 8, 128, 16001, 0),
        # chunks of two prompts over their cached rows, D = 64, fp32
        _prompt("prompt_chunks_f32_d64", 2, 8, 2, 64, 500, 6000, kv="f32", layout="cache"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["cache", "dense", "sparse", "prompt"])
    D = rng.choice([128, 128, 64])
    kv = rng.choice(["bf16", "bf16", "f32"])
    fmt = rng.choice(["e4m3", "int8"])
    block = rng.choice([16, 32, 64, 128, 256])
    Hkv = rng.choice([1, 2, 4, 8])
    Hq = Hkv * rng.choice([1, 2, 4, 8, 16])
    B = _log(rng, 1, 16)
    ragged = rng.random() < 0.5
    if kind == "cache":
        new = _log(rng, 1, max(2, 8 * 65536 // (B * Hkv)))
        held = _log(rng, 1, 5000) if rng.random() < 0.6 else 0
        return _cache(None, B, Hkv, D, new, held, block, fmt, kv, ragged)
    if kind in ("dense", "sparse"):
        n = _log(rng, 1, max(2, 8 * 131072 // (B * Hq)))
        w = rng.choice([0, _log(rng, 1, 512)])
        return _decode(None, kind, B, Hq, Hkv, D, n, w, block, fmt, kv, ragged, round(math.exp(rng.uniform(-6, -0.5)), 4))
    # queries x keys x heads, padded to the longest sequence, stay under an eighth of the largest listed case's
    most = 16001 * 16001 * 4 // (B * Hq)
    if kv == "f32":
        most //= 16
    q = _log(rng, 1, max(1, min(6000, math.isqrt(most))))
    ctx = rng.choice([0, _log(rng, 1, max(1, min(32768, most // q - q)))]) if most // q > q else 0
    return _prompt(None, B, Hq, Hkv, D, q, ctx, kv, rng.random() < 0.8, rng.choice(["packed", "cache"]))


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


# ---------------------------------------------------------------- the 8-bit cache, plain
def _e4m3_exponent(amax):
    """The smallest e with amax <= 448 * 2^e, at least -126 (amax = m 2^x, m in [0.5, 1); 448 = 0.875 2^9)."""
    m, x = torch.frexp(amax)
    return (x - 9 + (m > 0.875)).clamp(min=-126)


def _scale(amax, fmt):
    """Scale of a block whose largest magnitude is amax; 0 for a block of zeros."""
    if fmt == "e4m3":
        s = ((_e4m3_exponent(amax).int() + 127) << 23).view(torch.float32)   # 2^e by its bits
    else:
        s = (amax / torch.full_like(amax, 127.0)).clamp(min=TINY)   # (divided by a tensor: by a number, torch multiplies)
    return torch.where(amax > 0, s, torch.zeros_like(s))


def _encode(x, s, fmt):
    """Codes of x under scales s (broadcast), in x / s rounded once: products are exact in 64 bits."""
    r = torch.where(s > 0, 1.0 / s, torch.zeros_like(s)).double()
    y = torch.nan_to_num(x.double(), nan=0.0, posinf=math.inf, neginf=-math.inf) * r
    y = torch.nan_to_num(y, nan=0.0, posinf=math.inf, neginf=-math.inf)
    if fmt == "e4m3":
        return y.clamp(-448, 448).float().to(torch.float8_e4m3fn)
    return y.round().clamp(-127, 127).to(torch.int8)


def _recode(c, ratio, fmt):
    y = c.double() * ratio.double()
    return y.float().to(torch.float8_e4m3fn) if fmt == "e4m3" else y.round().to(torch.int8)


def _write(codes, scale, x, row, new, held, block, fmt):
    """Write the rows of x marked `new` [B][R] into the cache rows `row` [B][R] (R whole blocks), keeping rows `held`."""
    B, H, R, D = x.shape
    nb = R // block
    bi = torch.arange(B, device=DEV)[:, None]
    blk = row[:, ::block] // block                                             # [B][nb]
    was = codes.view(torch.int8)[bi, :, row].transpose(1, 2).view(codes.dtype)  # [B][H][R][D]
    n4, h4 = new[:, None, :, None], held[:, None, :, None]
    fin = torch.where(n4 & torch.isfinite(x), x.float(), torch.zeros((), device=DEV)).abs()
    need = _scale(fin.reshape(B, H, nb, block * D).amax(dim=3), fmt)
    has = held.view(B, nb, block).any(dim=2)                                   # blocks that hold rows already
    touched = new.view(B, nb, block).any(dim=2)
    old = scale[bi, :, blk].transpose(1, 2)                                    # [B][H][nb]
    kept = torch.where(has[:, None], old, torch.zeros_like(old))
    s = torch.maximum(need, kept)
    grow = torch.where(s > 0, kept / s, torch.ones_like(s))
    up = lambda t: t.repeat_interleave(block, dim=2)[..., None]  # noqa: E731
    enc = _encode(x.float(), up(s), fmt).view(torch.int8)
    rec = _recode(was, up(grow), fmt).view(torch.int8)
    out = torch.where(n4, enc, torch.where(h4, rec, was.view(torch.int8)))
    codes.view(torch.int8)[bi, :, row] = out.transpose(1, 2)
    scale[bi, :, blk] = torch.where(touched[:, None], s, old).transpose(1, 2)


def _values(codes, scale, block):
    """The values that cache rows [0, R) stand for, in 32 bits."""
    R = codes.shape[2]
    return codes.float() * scale.repeat_interleave(block, dim=2)[:, :, :R, None]


def _filled(x, block, fmt):
    """A cache holding the rows x [B][H][R][D] (R whole blocks)."""
    B, H, R, D = x.shape
    s = torch.empty(B, H, R // block, device=DEV)
    codes = torch.empty(B, H, R, D, dtype=torch.int8, device=DEV)
    step = max(block, (1 << 25) // (H * D) // block * block)
    for b in range(B):
        for r in range(0, R, step):
            v = x[b, :, r:r + step].float().view(H, -1, block * D)
            sc = _scale(v.abs().amax(dim=2), fmt)
            s[b, :, r // block:r // block + v.shape[1]] = sc
            codes[b, :, r:r + step] = _encode(v, sc[:, :, None], fmt).view(torch.int8).view(H, -1, D)
    return codes.view(CODE[fmt]), s


# ---------------------------------------------------------------- inputs
def _rows(g, shape, dt):
    """Keys or values with four outlier channels and some tokens larger than the rest."""
    D = shape[-1]
    ch = torch.ones(D, device=DEV)
    ch[torch.randperm(D, device=DEV, generator=g)[:4]] = 6.0
    x = torch.empty(shape, dtype=dt, device=DEV)
    for b in range(shape[0]):
        tok = 1.0 + 2.0 * (torch.rand(shape[1:-1] + (1,), device=DEV, generator=g) < 0.02)
        x[b] = (torch.randn(shape[1:], device=DEV, generator=g) * ch * tok).to(dt)
    return x


def _up(n, block):
    return (n + block - 1) // block * block


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = random.Random(seed)
    B, Hkv, D, kind, dt = case["B"], case["Hkv"], case["D"], case["kind"], TYPE[case["kv"]]
    st = {"case": case}
    if kind == "cache":
        new, held, block, fmt = case["new"], case["held"], case["block"], case["fmt"]
        offs = _spread(B, held / 16, held, r) if case["ragged"] else [held] * B
        cnts = _spread(B, new / 16, new, r) if case["ragged"] else [new] * B
        cnts = [max(1, c) for c in cnts]
        cap = _up(held + new + 2 * block, block)
        R = _up(block - 1 + new, block)           # rows of the blocks that one sequence's new rows can touch
        st.update(cap=cap, R=R)
        for k in ("K", "V"):
            codes, s = _filled(_rows(g, (B, Hkv, _up(held, block), D), torch.float32), block, fmt) if held else (None, None)
            st[k + "8"] = torch.zeros(B, Hkv, cap, D, dtype=torch.int8, device=DEV).view(CODE[fmt])
            st[k + "s"] = torch.zeros(B, Hkv, cap // block, device=DEV)
            if held:
                st[k + "8"].view(torch.int8)[:, :, :codes.shape[2]] = codes.view(torch.int8)
                st[k + "s"][:, :, :s.shape[2]] = s
            st[k] = _rows(g, (B, Hkv, new, D), dt)
            st[k + "_back"] = torch.zeros(B, Hkv, R, D, dtype=dt, device=DEV)
        first = [o // block * block for o in offs]
        st.update(off=_i32(offs), cnt=_i32(cnts), first=_i32(first), span=_i32([o + c - f for o, c, f in zip(offs, cnts, first)]),
                  host=(offs, cnts))
        return st
    if kind in ("dense", "sparse"):
        Hq, n, w, block, fmt = (case[k] for k in ("Hq", "n", "w", "block", "fmt"))
        ns = [max(1, v) for v in _spread(B, n / 16, n, r)] if case["ragged"] else [n] * B
        ws = _spread(B, 0, w, r) if case["ragged"] else [w] * B
        cap = _up(n, block)
        for k in ("K", "V"):
            st[k + "8"], st[k + "s"] = _filled(_rows(g, (B, Hkv, cap, D), torch.bfloat16), block, fmt)
            st[k + "w"] = _rows(g, (B, Hkv, max(w, 1), D), dt)
        st.update(cap=cap, q=1.2 * torch.randn(B, Hq, D, device=DEV, generator=g), host=(ns, ws), seq_n=_i32(ns), seq_w=_i32(ws))
        if kind == "sparse":
            live = torch.arange(n, device=DEV)[None, None, :] < st["seq_n"][:, None, None]
            keep = (torch.rand(B, Hq, n, device=DEV, generator=g) < case["share"]) & live
            keep[:, :, 0] = True
            cnt = keep.sum(dim=2)
            sel = torch.zeros(B, Hq, n, dtype=torch.int32, device=DEV)
            sel[torch.arange(n, device=DEV)[None, None, :] < cnt[:, :, None]] = keep.nonzero()[:, 2].int()
            st.update(sel_idx=sel, sel_count=cnt.int())
        return st
    Hq, lq, ctx = case["Hq"], case["q"], case["ctx"]
    qs = [max(1, v) for v in (_spread(B, lq / 16, lq, r) if B > 1 else [lq])]
    ks = [a + b for a, b in zip(qs, _spread(B, 0, ctx, r) if B > 1 else [ctx])]
    cu_q, cu_k = np.cumsum([0] + qs).tolist(), np.cumsum([0] + ks).tolist()
    T, cap = cu_q[-1], max(ks)
    shape = (1, cu_k[-1], Hkv, D) if case["layout"] == "packed" else (B, Hkv, cap, D)
    st.update(q=(1.2 * torch.randn(T, Hq, D, device=DEV, generator=g)).to(dt), K=_rows(g, shape, dt), V=_rows(g, shape, dt),
              cu_q=_i32(cu_q), cu_k=_i32(cu_k), host=(qs, ks), T=T, cap=cap)
    return st


# ---------------------------------------------------------------- plain forms
def _run_cache(st):
    c = st["case"]
    block, fmt, R = c["block"], c["fmt"], st["R"]
    new_src = torch.arange(c["new"], device=DEV)
    row = st["first"][:, None].long() + torch.arange(R, device=DEV)      # cache rows of the touched blocks
    src = row - st["off"][:, None]
    new = (src >= 0) & (src < st["cnt"][:, None])
    held = src < 0
    pick = src.clamp(0, len(new_src) - 1)
    bi = torch.arange(c["B"], device=DEV)[:, None]
    res = {}
    for k in ("K", "V"):
        x = st[k][bi, :, pick].transpose(1, 2)                             # [B][H][R][D]
        _write(st[k + "8"], st[k + "s"], x, row, new, held, block, fmt)
        codes = st[k + "8"].view(torch.int8)[bi, :, row].transpose(1, 2).contiguous().view(CODE[fmt])
        s = st[k + "s"][bi, :, row[:, ::block] // block].transpose(1, 2)
        val = _values(codes, s, block).to(TYPE[c["kv"]])
        res[k] = torch.where((new | held)[:, None, :, None], val, torch.zeros_like(val))
        res[k + "_scale"] = st[k + "s"]
    return res


def _attend(q, K, V, keep, tau):
    """q [..][G][D], K and V [..][N][D], keep [..][G][N]: softmax attention in 32 bits; rows that keep nothing give 0."""
    S = torch.matmul(q, K.transpose(-1, -2).contiguous()).mul_(tau).masked_fill_(~keep, -math.inf)
    m = S.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = S.sub_(m).exp_()
    l = P.sum(dim=-1, keepdim=True)
    out = torch.matmul(P, V) / l.clamp(min=1e-38)
    return out, (m + l.log())[..., 0]


def _run_decode(st):
    c = st["case"]
    B, Hq, Hkv, D, n, w, block = (c[k] for k in ("B", "Hq", "Hkv", "D", "n", "w", "block"))
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
    kv = [torch.cat([_values(st[k + "8"][:, :, :n], st[k + "s"], block), st[k + "w"][:, :, :w].float()], dim=2) for k in "KV"]
    out, lse = _attend(st["q"].view(B, Hkv, G, D), kv[0], kv[1], keep, 1.0 / math.sqrt(D))
    return {"out": out.reshape(B, Hq, D), "lse": lse.reshape(B, Hq)}


def _run_prompt(st):
    c = st["case"]
    B, Hq, Hkv, D = (c[k] for k in ("B", "Hq", "Hkv", "D"))
    G, Lq, Lk = Hq // Hkv, max(st["host"][0]), max(st["host"][1])
    cu_q, cu_k = st["cu_q"].long(), st["cu_k"].long()
    nq, nk = cu_q[1:] - cu_q[:-1], cu_k[1:] - cu_k[:-1]
    i, j = torch.arange(Lq, device=DEV), torch.arange(Lk, device=DEV)
    tok = torch.where(i[None] < nq[:, None], cu_q[:-1, None] + i, 0)                     # [B][Lq]
    q = st["q"].float()[tok].view(B, Lq, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Lq, D)
    if c["layout"] == "packed":
        at = torch.where(j[None] < nk[:, None], cu_k[:-1, None] + j, 0)
        K, V = (st[k][0].float()[at].transpose(1, 2).contiguous() for k in "KV")
    else:
        K, V = st["K"].float(), st["V"].float()
    keep = (j[None, None] < nk[:, None, None]) & (i[None, :, None] < nq[:, None, None])
    if c["causal"]:
        keep = keep & (j[None, None] <= i[None, :, None] + (nk - nq)[:, None, None])
    keep = keep[:, None, None].expand(B, Hkv, G, Lq, Lk)
    S = torch.matmul(q, K.transpose(-1, -2).contiguous()).view(B, Hkv, G, Lq, Lk)
    S.mul_(1.0 / math.sqrt(D)).masked_fill_(~keep, -math.inf)
    m = S.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = S.sub_(m).exp_()
    l = P.sum(dim=-1, keepdim=True)
    out = torch.matmul(P.view(B, Hkv, G * Lq, Lk), V).view(B, Hkv, G, Lq, D) / l.clamp(min=1e-38)
    lse = (m + l.log())[..., 0]
    # token t of the packed axis: its sequence and place there
    t = torch.arange(st["T"], device=DEV)
    b = torch.searchsorted(cu_q, t, right=True) - 1
    k = t - cu_q[b]
    out = out.permute(0, 3, 1, 2, 4).reshape(B, Lq, Hq, D)[b, k]
    return {"out": out.to(TYPE[c["kv"]]), "lse": lse.permute(0, 3, 1, 2).reshape(B, Lq, Hq)[b, k]}


# ---------------------------------------------------------------- as a user calls them
def _own_cache(st):
    from paper_2606_31519_amd import rbq
    c = st["case"]
    B, Hkv, D, new, held, block = (c[k] for k in ("B", "Hkv", "D", "new", "held", "block"))
    seqs = (st["off"], st["cnt"]) if c["ragged"] else (None, None)
    back = (st["first"], st["span"]) if c["ragged"] else (None, None)
    first = held // block * block
    rows = st["R"] if c["ragged"] else held + new - first
    rbq.rbq_quantize_kv(B, Hkv, D, st["K"], st["V"], new, new, held, st["cap"], block, st["K8"], st["V8"], st["Ks"], st["Vs"],
                        *seqs)
    rbq.rbq_dequantize_kv(B, Hkv, D, st["K8"], st["V8"], block, st["Ks"], st["Vs"], st["cap"], rows, first, st["K_back"],
                          st["V_back"], st["R"], *back)
    return {"K": st["K_back"], "K_scale": st["Ks"], "V": st["V_back"], "V_scale": st["Vs"]}


def _own_decode(st):
    from paper_2606_31519_amd import rbq
    c = st["case"]
    B, Hq, Hkv, D, n, w, block = (c[k] for k in ("B", "Hq", "Hkv", "D", "n", "w", "block"))
    if "ws" not in st:   # a serving loop keeps its workspace and outputs
        st["ws"] = rbq.workspace(rbq.RBQ_OP_DECODE_KV8, B, Hq, Hkv, D, n, w)
        st["out"], st["lse"] = torch.empty(B, Hq, D, device=DEV), torch.empty(B, Hq, device=DEV)
    seqs = (st["seq_n"], st["seq_w"]) if c["ragged"] else (None, None)
    cache = (st["K8"], st["V8"], block, st["Ks"], st["Vs"], st["cap"], n)
    tail = (st["Kw"], st["Vw"], max(w, 1), w, 1.0 / math.sqrt(D), st["out"], st["lse"], st["ws"])
    if c["kind"] == "dense":
        rbq.rbq_dense_decode_kv8(B, Hq, Hkv, D, st["q"], *cache, *tail, *seqs)
    else:
        rbq.rbq_sparse_decode_kv8(B, Hq, Hkv, D, st["q"], *cache, st["sel_idx"], st["sel_count"], *tail, *seqs)
    return {"out": st["out"], "lse": st["lse"]}


def _own_prompt(st):
    from paper_2606_31519_amd import rbq
    c = st["case"]
    B, Hq, Hkv, D, T, cap = c["B"], c["Hq"], c["Hkv"], c["D"], st["T"], st["cap"]
    if "ws" not in st:
        st["ws"] = rbq.workspace(rbq.RBQ_OP_PREFILL, B, Hq, Hkv, D, cap, T)
        st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty(T, Hq, device=DEV)
    # strides of a K / V row, head and sequence, and the rows that there are (of all sequences, or of each)
    lay = (Hkv * D, D, 0, st["K"].shape[1]) if c["layout"] == "packed" else (D, cap * D, Hkv * cap * D, cap)
    rbq.rbq_prefill_attention(B, Hq, Hkv, D, st["q"], Hq * D, st["K"], st["V"], *lay, st["cu_q"], st["cu_k"], T, cap,
                              c["causal"], 1.0 / math.sqrt(D), st["out"], st["lse"], st["ws"])
    return {"out": st["out"], "lse": st["lse"]}


def run(state):
    kind = state["case"]["kind"]
    if kind == "cache":
        return _own_cache(state) if own else _run_cache(state)
    if kind == "prompt":
        return _own_prompt(state) if own else _run_prompt(state)
    return _own_decode(state) if own else _run_decode(state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    B, Hkv, D, kind = case["B"], case["Hkv"], case["D"], case["kind"]
    el = 2 if case["kv"] == "bf16" else 4
    if kind == "cache":
        block = case["block"]
        offs = _even(B, case["held"] / 16, case["held"]) if case["ragged"] else [case["held"]] * B
        cnts = [max(1, c) for c in _even(B, case["new"] / 16, case["new"])] if case["ragged"] else [case["new"]] * B
        new = sum(cnts)
        kept = sum(o % block for o in offs)
        scales = sum((o + c + block - 1) // block - o // block for o, c in zip(offs, cnts))
        # new rows in and their codes out; rows and scales of the touched blocks read back
        by = 2 * Hkv * (new * D * (el + 1) + kept * D + scales * 4 + (new + kept) * D * el)
        return {"bytes": by, "flops": 2 * Hkv * (2 * new + kept) * D * 2}
    if kind in ("dense", "sparse"):
        Hq, n, w, block = (case[k] for k in ("Hq", "n", "w", "block"))
        ns = sum(max(1, v) for v in _even(B, n / 16, n)) if case["ragged"] else B * n
        ws = sum(_even(B, 0, w)) if case["ragged"] else B * w
        f = case.get("share", 1.0)
        union = 1.0 - (1.0 - f) ** (Hq // Hkv)
        touched = 1.0 - (1.0 - union) ** block      # blocks with a row that some head takes
        by = Hkv * (2 * ns * union * D + 2 * ws * D * el + 8 * ns * touched / block) + B * Hq * D * 8 + B * Hq * 4
        if kind == "sparse":
            by += 4 * Hq * ns * f
        return {"bytes": int(by), "flops": int(4 * D * Hq * (ns * f + ws))}
    Hq, lq, ctx = case["Hq"], case["q"], case["ctx"]
    qs = [max(1, v) for v in (_even(B, lq / 16, lq) if B > 1 else [lq])]
    cs = _even(B, 0, ctx) if B > 1 else [ctx]
    cs = [sum(cs) / B] * B                          # (their order goes by the seed)
    pairs = sum(a * (k + (a + 1) / 2 if case["causal"] else k + a) for a, k in zip(qs, cs))
    by = (2 * sum(qs) * Hq * D + 2 * (sum(qs) + sum(cs)) * Hkv * D) * el + 4 * sum(qs) * Hq
    return {"bytes": int(by), "flops": int(4 * D * Hq * pairs)}


# ---------------------------------------------------------------- the same in 64 bits
def _pow2(e):
    """2^e of whole numbers e by its bits (the GPU's pow rounds)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_scale(amax, fmt):
    if fmt == "e4m3":
        a = np.maximum(amax.cpu().numpy(), np.finfo(np.float64).tiny)
        e = np.ceil(np.log2(a / 448.0)).astype(np.int64)
        e -= np.ldexp(448.0, e - 1) >= a               # (where log2 rounded across a whole number)
        e += np.ldexp(448.0, e) < a
        s = _pow2(torch.from_numpy(np.maximum(e, -126)).to(amax.device))
    else:
        s = (amax / 127.0).float().double().clamp(min=TINY)            # the scale is held in 32 bits
    return torch.where(amax > 0, s, torch.zeros_like(s))


def _nearest(y, fmt):
    """The value of the format nearest to y, ties to even."""
    if fmt == "int8":
        return torch.round(y).clamp(-127, 127)
    a = y.abs().clamp(max=448.0)
    step = _pow2(torch.frexp(a.clamp(min=2.0 ** -6))[1] - 4)
    return torch.sign(y) * torch.round(a / step) * step


def _exact_cache(case, st):
    B, Hkv, D, block, fmt, R = case["B"], case["Hkv"], case["D"], case["block"], case["fmt"], st["R"]
    res = {}
    for k in ("K", "V"):
        back = torch.zeros(B, Hkv, R, D, dtype=torch.float64, device=DEV)
        scales = st[k + "s"].double()
        for b, (off, cnt) in enumerate(zip(*st["host"])):
            first, at = off // block * block, 0
            for lo in range(first, off + cnt, max(block, 8192 // block * block)):
                hi = min(off + cnt, lo + max(block, 8192 // block * block))
                m = _up(hi - lo, block)
                v = torch.zeros(Hkv, m, D, dtype=torch.float64, device=DEV)
                kept = max(0, off - lo) if lo == first else 0
                v[:, kept:hi - lo] = st[k][b, :, lo + kept - off:hi - off].double()
                need = _exact_scale(v.view(Hkv, m // block, block * D).abs().amax(dim=2), fmt)
                s = need.clone()
                if kept:
                    old = scales[b, :, lo // block].clone()
                    s[:, 0] = torch.maximum(need[:, 0], old)
                big = s.repeat_interleave(block, dim=1)[..., None]
                inv = torch.where(big > 0, (1.0 / big).float().double(), torch.zeros_like(big))
                q = _nearest(v * inv, fmt)
                if kept:
                    ratio = torch.where(s[:, 0] > 0, (old / s[:, 0]).float().double(), torch.ones_like(old))
                    c = st[k + "8"][b, :, lo:lo + kept].double()
                    q[:, :kept] = _nearest(c * ratio[:, None, None], fmt)
                back[b, :, at:at + hi - lo] = (q * big)[:, :hi - lo]
                scales[b, :, lo // block:lo // block + m // block] = s
                at += hi - lo
        res[k], res[k + "_scale"] = back, scales
    return res


def _exact_rows(q, K, V, keep, tau):
    """Attention of q [Hkv][M][D] over K, V [Hkv][N][D] with keep [Hkv or 1][M][N], head by head."""
    out, lse = [], []
    for h in range(q.shape[0]):
        lg = torch.matmul(q[h], K[h].t().contiguous()) * tau
        lg = torch.where(keep[h if keep.shape[0] > 1 else 0], lg, torch.full((), -math.inf, dtype=lg.dtype, device=DEV))
        L = torch.logsumexp(lg, dim=1)
        out.append(torch.matmul(torch.exp(lg - L[:, None]), V[h]))
        lse.append(L)
    return torch.stack(out), torch.stack(lse)


def exact(case, seed):
    st = prepare(case, seed)
    kind, B, Hkv, D = case["kind"], case["B"], case["Hkv"], case["D"]
    if kind == "cache":
        return _exact_cache(case, st)
    Hq, tau = case["Hq"], float(np.float32(1.0 / math.sqrt(D)))
    G = Hq // Hkv
    if kind in ("dense", "sparse"):
        block, outs, lses = case["block"], [], []
        for b, (nb, wb) in enumerate(zip(*st["host"])):
            kv = []
            for k in "KV":
                s = st[k + "s"][b].double()[:, torch.arange(nb, device=DEV) // block]
                kv.append(torch.cat([st[k + "8"][b, :, :nb].float().double() * s[..., None], st[k + "w"][b, :, :wb].double()], dim=1))
            keep = torch.ones(Hkv, G, nb + wb, dtype=torch.bool, device=DEV)
            if kind == "sparse":
                keep[:, :, :nb] = False
                for h in range(Hq):
                    keep[h // G, h % G, st["sel_idx"][b, h, :int(st["sel_count"][b, h])].long()] = True
            o, l = _exact_rows(st["q"][b].double().view(Hkv, G, D), kv[0], kv[1], keep, tau)
            outs.append(o.reshape(Hq, D))
            lses.append(l.reshape(Hq))
        return {"out": torch.stack(outs), "lse": torch.stack(lses)}
    out = torch.empty(st["T"], Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.empty(st["T"], Hq, dtype=torch.float64, device=DEV)
    tq = tk = 0
    for b, (nq, nk) in enumerate(zip(*st["host"])):
        K, V = (st[k][0, tk:tk + nk].transpose(0, 1) if case["layout"] == "packed" else st[k][b, :, :nk] for k in "KV")
        i, j = torch.arange(nq, device=DEV)[:, None], torch.arange(nk, device=DEV)[None]
        keep = (j <= i + nk - nq) if case["causal"] else torch.ones(nq, nk, dtype=torch.bool, device=DEV)
        for h in range(Hq):
            o, l = _exact_rows(st["q"][tq:tq + nq, h].double()[None], K[h // G].double()[None], V[h // G].double()[None],
                               keep[None], tau)
            out[tq:tq + nq, h], lse[tq:tq + nq, h] = o[0], l[0]
        tq, tk = tq + nq, tk + nk
    return {"out": out, "lse": lse}
