"""Device buffers of one decode workload and the calls of one decode step.

The KV cache of a (sequence, KV head) holds `cap` rows: rows [0, n) are
indexed (Algorithm 1), rows [n, n + w) are the local window of newest keys
that decode attends in full precision and that a lazy flush later appends to
the index (Section 3.4). torch only allocates memory and supplies the stream;
every step of the method runs in librbq.so's kernels.
"""
from __future__ import annotations

import math

import numpy as np
import torch

from . import rbq


def to_device_kv(arr: np.ndarray, kv_dtype: str, device) -> torch.Tensor:
    """Upload keys/values given as float32 or as bf16 bit patterns (uint16)."""
    if kv_dtype == "f32":
        return torch.from_numpy(np.ascontiguousarray(arr, dtype=np.float32)).to(device)
    t = torch.from_numpy(np.ascontiguousarray(arr).view(np.int16)).to(device)
    return t.view(torch.bfloat16)


class DecodeState:
    """Index + cache + per-step buffers for B sequences x Hkv KV heads."""

    def __init__(self, B, Hq, Hkv, D, cap, n, w, K, V, q, P, c_q=None, device="cuda", compact=False):
        """compact: the compact index (one fp16 factor per key in kfac16, no
        query centroid) and the *_f16 calls instead of the fp32 (f, g) index."""
        if compact and c_q is not None:
            raise ValueError("the compact index is built and read without a query centroid")
        self.compact = compact
        self.B, self.Hq, self.Hkv, self.D = B, Hq, Hkv, D
        self.cap, self.n, self.w = cap, n, w
        self.device = device
        self.K, self.V = K, V                       # [B][Hkv][cap][D]
        self.q = q                                  # [B][Hq][D] fp32
        self.P = P                                  # [D][D] fp32
        self.c_q = c_q                              # [B][Hkv][D] fp32 or None
        f32 = dict(dtype=torch.float32, device=device)
        self.c_k = torch.zeros(B, Hkv, D, **f32)
        self.codes = torch.zeros(B, Hkv, cap, D // 32, dtype=torch.int32, device=device)
        self.kfac = None if compact else torch.zeros(B, Hkv, cap, 2, **f32)
        self.kfac16 = torch.zeros(B, Hkv, cap, dtype=torch.float16, device=device) if compact else None
        self.qplanes = torch.zeros(B, Hq, 4, D // 32, dtype=torch.int32, device=device)
        self.qscal = torch.zeros(B, Hq, rbq.QSCAL_STRIDE, **f32)
        self.scores = torch.zeros(B, Hq, max(n, 1), **f32)
        self.sel_idx = torch.zeros(B, Hq, max(n, 1), dtype=torch.int32, device=device)
        self.sel_count = torch.zeros(B, Hq, dtype=torch.int32, device=device)
        self.out = torch.zeros(B, Hq, D, **f32)
        self.lse = torch.zeros(B, Hq, **f32)
        self.ws_encode = rbq.workspace(rbq.RBQ_OP_ENCODE, B, Hq, Hkv, D, max(n, w, 1), 0, device)
        self.ws_topp = rbq.workspace(rbq.RBQ_OP_TOPP, B, Hq, Hkv, D, n, 0, device)
        self.ws_decode = rbq.workspace(rbq.RBQ_OP_SPARSE_DECODE, B, Hq, Hkv, D, n, w, device)
        self.ws_step = rbq.workspace(rbq.RBQ_OP_DECODE_STEP, B, Hq, Hkv, D, n, w, device)
        self.sm_scale = 1.0 / math.sqrt(D)

    @classmethod
    def from_workload(cls, wl, device="cuda", c_q: bool = True, compact: bool = False):
        K = to_device_kv(wl.K, wl.kv_dtype, device)
        V = to_device_kv(wl.V, wl.kv_dtype, device)
        q = torch.from_numpy(np.ascontiguousarray(wl.q)).to(device)
        P = torch.from_numpy(np.ascontiguousarray(wl.P)).to(device)
        cq = torch.from_numpy(np.ascontiguousarray(wl.c_q)).to(device) if c_q and not compact else None
        return cls(wl.B, wl.Hq, wl.Hkv, wl.D, wl.N, wl.n_index, wl.w, K, V, q, P, cq, device, compact)

    def _window(self, t):
        """Rows [n, cap) of a cache (the local window), in HBM or mapped host memory."""
        return t.rows(self.n, self.D) if isinstance(t, rbq.MappedHost) else t[:, :, self.n:]

    # ---------------------------------------------------------------- the five calls
    def build_index(self, stream=None, rot_out=None, alpha_out=None):
        """Prefill index construction over rows [0, n), setting c_k (Algorithm 1)."""
        if self.compact:
            rbq.rbq_encode_keys_f16(self.B, self.Hkv, self.D, self.K, self.cap, self.n, 0, self.cap, self.P,
                                    self.c_k, self.codes, self.kfac16, rbq.RBQ_ENCODE_SET_CENTROID, self.ws_encode,
                                    stream)
            return
        rbq.rbq_encode_keys(self.B, self.Hkv, self.D, self.K, self.cap, self.n, 0, self.cap, self.P, self.c_q,
                            self.c_k, self.codes, self.kfac, rbq.RBQ_ENCODE_SET_CENTROID, alpha_out,
                            self.ws_encode, stream, rot_out=rot_out)

    def flush_window(self, stream=None):
        """Lazy update: encode the w window rows into index rows [n, n + w) with
        the prefill centroid (Section 3.4). The index size used by scoring is
        left at n, so repeated steps stay identical."""
        if self.w == 0:
            return
        K_win = self._window(self.K)
        if self.compact:
            rbq.rbq_encode_keys_f16(self.B, self.Hkv, self.D, K_win, self.cap, self.w, self.n, self.cap, self.P,
                                    self.c_k, self.codes, self.kfac16, 0, None, stream)
            return
        rbq.rbq_encode_keys(self.B, self.Hkv, self.D, K_win, self.cap, self.w, self.n, self.cap, self.P, self.c_q,
                            self.c_k, self.codes, self.kfac, 0, None, None, stream)

    def quantize(self, stream=None, qrot_out=None):
        rbq.rbq_quantize_query(self.B, self.Hq, self.Hkv, self.D, self.q, self.P, self.c_q, self.c_k,
                               self.qplanes, self.qscal, stream, qrot_out=qrot_out)

    def score(self, stream=None):
        if self.compact:
            rbq.rbq_score_f16(self.B, self.Hq, self.Hkv, self.D, self.n, self.cap, self.codes, self.kfac16,
                              self.qplanes, self.qscal, self.scores, stream)
            return
        rbq.rbq_score(self.B, self.Hq, self.Hkv, self.D, self.n, self.cap, self.codes, self.kfac, self.qplanes,
                      self.qscal, self.scores, stream)

    def select(self, p, stream=None):
        rbq.rbq_topp_select(self.B, self.Hq, self.n, self.scores, p, self.sm_scale, self.sel_idx, self.sel_count,
                            self.ws_topp, stream)

    def sparse_decode(self, stream=None):
        K_loc = self._window(self.K) if self.w else None
        V_loc = self._window(self.V) if self.w else None
        rbq.rbq_sparse_decode(self.B, self.Hq, self.Hkv, self.D, self.q, self.K, self.V, self.cap, self.n,
                              self.sel_idx, self.sel_count, K_loc, V_loc, self.cap, self.w, self.sm_scale, self.out,
                              self.lse, self.ws_decode, stream)

    def dense_decode(self, out=None, lse=None, stream=None):
        K_loc = self._window(self.K) if self.w else None
        V_loc = self._window(self.V) if self.w else None
        rbq.rbq_dense_decode(self.B, self.Hq, self.Hkv, self.D, self.q, self.K, self.V, self.cap, self.n, K_loc,
                             V_loc, self.cap, self.w, self.sm_scale, self.out if out is None else out,
                             self.lse if lse is None else lse, self.ws_decode, stream)

    def step(self, p, stream=None, flush=True):
        """One decode step of the whole path with rbq_decode_step: quantize ->
        score -> Top-p -> sparse attention (index selection + window), and the
        lazy flush of the window into index rows [n, n + w) (which this step's
        scoring does not read), in one call with fewer launches."""
        if self.compact:
            rbq.rbq_decode_step_f16(self.B, self.Hq, self.Hkv, self.D, self.q, self.P, self.c_k, self.K, self.V,
                                    self.cap, self.n, self.w, self.codes, self.kfac16, flush, p, self.sm_scale,
                                    self.qplanes, self.qscal, self.scores, self.sel_idx, self.sel_count, self.out,
                                    self.lse, self.ws_step, stream)
            return
        rbq.rbq_decode_step(self.B, self.Hq, self.Hkv, self.D, self.q, self.P, self.c_q, self.c_k, self.K, self.V,
                            self.cap, self.n, self.w, self.codes, self.kfac, flush, p, self.sm_scale, self.qplanes,
                            self.qscal, self.scores, self.sel_idx, self.sel_count, self.out, self.lse, self.ws_step,
                            stream)

    def step_calls(self, p, stream=None, flush=True):
        """The same step as the five separate calls (bitwise the same outputs)."""
        self.quantize(stream)
        self.score(stream)
        self.select(p, stream)
        self.sparse_decode(stream)
        if flush:
            self.flush_window(stream)

    # ---------------------------------------------------------------- ragged batches
    # seq_n / seq_w / seq_p: per-sequence indexed keys, window rows (the cache
    # tail after them) and p, as int32 / int32 / float32 device tensors [B]; the
    # state's n and w are the largest counts (n + w <= cap).
    def build_index_ragged(self, seq_n_host, stream=None):
        """Index construction of a ragged batch: sequence b over its rows
        [0, seq_n_host[b]) with its own centroid (a sequence without keys keeps a
        zero centroid)."""
        for b, nb in enumerate(seq_n_host):
            nb = min(int(nb), self.n)
            if nb > 0 and self.compact:
                rbq.rbq_encode_keys_f16(1, self.Hkv, self.D, self.K[b:b + 1], self.cap, nb, 0, self.cap, self.P,
                                        self.c_k[b:b + 1], self.codes[b:b + 1], self.kfac16[b:b + 1],
                                        rbq.RBQ_ENCODE_SET_CENTROID, self.ws_encode, stream)
            elif nb > 0:
                rbq.rbq_encode_keys(1, self.Hkv, self.D, self.K[b:b + 1], self.cap, nb, 0, self.cap, self.P,
                                    None if self.c_q is None else self.c_q[b:b + 1], self.c_k[b:b + 1],
                                    self.codes[b:b + 1], self.kfac[b:b + 1], rbq.RBQ_ENCODE_SET_CENTROID, None,
                                    self.ws_encode, stream)

    def step_ragged(self, seq_n, seq_w, seq_p, stream=None, flush=True):
        """One decode step of a ragged batch (rbq_decode_step_varlen)."""
        if self.compact:
            rbq.rbq_decode_step_varlen_f16(self.B, self.Hq, self.Hkv, self.D, self.q, self.P, self.c_k, self.K,
                                           self.V, self.cap, self.n, self.w, seq_n, seq_w, self.codes, self.kfac16,
                                           flush, seq_p, self.sm_scale, self.qplanes, self.qscal, self.scores,
                                           self.sel_idx, self.sel_count, self.out, self.lse, self.ws_step, stream)
            return
        rbq.rbq_decode_step_varlen(self.B, self.Hq, self.Hkv, self.D, self.q, self.P, self.c_q, self.c_k, self.K,
                                   self.V, self.cap, self.n, self.w, seq_n, seq_w, self.codes, self.kfac, flush,
                                   seq_p, self.sm_scale, self.qplanes, self.qscal, self.scores, self.sel_idx,
                                   self.sel_count, self.out, self.lse, self.ws_step, stream)

    def sparse_decode_ragged(self, seq_n, seq_w, stream=None):
        rbq.rbq_sparse_decode_varlen(self.B, self.Hq, self.Hkv, self.D, self.q, self.K, self.V, self.cap, self.n,
                                     self.w, seq_n, seq_w, self.sel_idx, self.sel_count, self.sm_scale, self.out,
                                     self.lse, self.ws_decode, stream)

    def dense_decode_ragged(self, seq_n, seq_w, out=None, lse=None, stream=None):
        rbq.rbq_dense_decode_varlen(self.B, self.Hq, self.Hkv, self.D, self.q, self.K, self.V, self.cap, self.n,
                                    self.w, seq_n, seq_w, self.sm_scale, self.out if out is None else out,
                                    self.lse if lse is None else lse, self.ws_decode, stream)


KV8_DTYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


class Kv8Cache:
    """K and V rows in 8 bits ("e4m3" or "int8"), one scale per (sequence, KV head,
    block of `block` tokens): the buffers and the calls that write and read them."""

    def __init__(self, B, Hkv, D, cap, fmt="e4m3", block=64, device="cuda"):
        if fmt not in KV8_DTYPES:
            raise ValueError(f"unknown 8-bit format {fmt!r} (one of {sorted(KV8_DTYPES)})")
        self.B, self.Hkv, self.D, self.cap, self.fmt, self.block = B, Hkv, D, cap, fmt, block
        self.K8, self.V8 = (torch.zeros(B, Hkv, cap, D, dtype=torch.int8, device=device).view(KV8_DTYPES[fmt])
                            for _ in range(2))
        blocks = (cap + block - 1) // block
        self.k_scale, self.v_scale = (torch.zeros(B, Hkv, blocks, dtype=torch.float32, device=device) for _ in range(2))

    def append(self, K, V, ld, rows, offset, seq_off=None, seq_rows=None, stream=None):
        """Rows [0, rows) of K / V [B][Hkv][ld][D] as cache rows [offset, offset + rows) (rbq_quantize_kv)."""
        rbq.rbq_quantize_kv(self.B, self.Hkv, self.D, K, V, ld, rows, offset, self.cap, self.block, self.K8, self.V8,
                            self.k_scale, self.v_scale, seq_off, seq_rows, stream)

    def read(self, K, V, ld, rows, offset=0, seq_off=None, seq_rows=None, stream=None):
        """Cache rows [offset, offset + rows) as rows [0, rows) of K / V (rbq_dequantize_kv)."""
        rbq.rbq_dequantize_kv(self.B, self.Hkv, self.D, self.K8, self.V8, self.block, self.k_scale, self.v_scale, self.cap,
                              rows, offset, K, V, ld, seq_off, seq_rows, stream)


class Kv4Cache:
    """K and V rows in 4 bits ("fp4" or "int4"), each row with scales of its own: the buffers and the calls that
    write and read them."""

    def __init__(self, B, Hkv, D, cap, fmt="fp4", device="cuda"):
        if fmt not in rbq.KV4_FORMATS:
            raise ValueError(f"unknown 4-bit format {fmt!r} (one of {sorted(rbq.KV4_FORMATS)})")
        self.B, self.Hkv, self.D, self.cap, self.fmt, self.code = B, Hkv, D, cap, fmt, rbq.KV4_FORMATS[fmt]
        self.kv4 = torch.zeros(B, Hkv, cap, D, dtype=torch.uint8, device=device)
        self.par = torch.zeros(B, Hkv, cap, 2, dtype=torch.int32, device=device)

    def append(self, K, V, ld, rows, offset, seq_off=None, seq_rows=None, stream=None):
        """Rows [0, rows) of K / V [B][Hkv][ld][D] as cache rows [offset, offset + rows) (rbq_quantize_kv4)."""
        rbq.rbq_quantize_kv4(self.B, self.Hkv, self.D, K, V, ld, rows, offset, self.cap, self.code, self.kv4, self.par,
                             seq_off, seq_rows, stream)

    def read(self, K, V, ld, rows, offset=0, seq_off=None, seq_rows=None, stream=None):
        """Cache rows [offset, offset + rows) as rows [0, rows) of K / V (rbq_dequantize_kv4)."""
        rbq.rbq_dequantize_kv4(self.B, self.Hkv, self.D, self.kv4, self.par, self.code, self.cap, rows, offset, K, V, ld,
                               seq_off, seq_rows, stream)


class PromptAttention:
    """The attention of a batch of prompts, or of chunks of them behind rows that are
    cached (rbq_prefill_attention): q_lens tokens and k_lens keys per sequence
    (k_lens None: the prompts themselves), the lengths' device arrays and the
    workspace kept for every call (one per layer; calls that overlap in time, on
    several streams, need plans of their own)."""

    def __init__(self, Hq, Hkv, D, q_lens, k_lens=None, causal=True, device="cuda"):
        k_lens = q_lens if k_lens is None else k_lens
        if len(q_lens) != len(k_lens) or not len(q_lens) or min(min(q_lens), min(k_lens)) < 0:
            raise ValueError("one length of at least 0 per sequence, for the queries and for the keys")
        self.B, self.Hq, self.Hkv, self.D, self.causal = len(q_lens), Hq, Hkv, D, causal
        if max(sum(map(int, q_lens)), sum(map(int, k_lens))) >= 1 << 31:   # (the call counts in int32)
            raise ValueError("2^31 tokens or keys and more")
        cu_q, cu_k = (np.concatenate([[0], np.cumsum(v)]).astype(np.int32) for v in (q_lens, k_lens))
        self.total_q, self.total_k, self.max_k = int(cu_q[-1]), int(cu_k[-1]), int(max(k_lens))
        self.cu_q, self.cu_k = (torch.from_numpy(c).to(device) for c in (cu_q, cu_k))
        self.ws = rbq.workspace(rbq.RBQ_OP_PREFILL, self.B, Hq, Hkv, D, self.max_k, self.total_q, device)
        self.sm_scale = 1.0 / math.sqrt(D)

    def _strides(self, t):
        """Of K or V: from a row, a head and a sequence to the next (0: packed, or the only sequence). A dimension of one
        entry has no stride that means anything, so it takes that of contiguous rows."""
        rows = 0 if t.dim() == 3 else 2
        row = t.stride(rows) if t.shape[rows] > 1 else self.D if rows else self.Hkv * self.D
        return row, t.stride(1) if self.Hkv > 1 else self.D, t.stride(0) if rows and self.B > 1 else 0

    def __call__(self, q, K, V, out=None, lse=None, stream=None):
        """q [total_q][Hq][D]; K, V packed [total_k][Hkv][D] or in a cache [B][Hkv][cap][D] (rows from 0, of each sequence
        its own: a cache expanded over several is refused); any strides whose last dimension (of q: two) is contiguous.
        Returns out [total_q][Hq][D] in q's type."""
        D = self.D
        if tuple(q.shape[1:]) != (self.Hq, D) or q.shape[0] < self.total_q:
            raise ValueError(f"q is {tuple(q.shape)}, the plan needs ({self.total_q}, {self.Hq}, {D})")
        packed = K.dim() == 3
        want = (self.total_k, self.Hkv, D) if packed else (self.B, self.Hkv, self.max_k, D)
        rows = 0 if packed else 2
        if (K.shape != V.shape or K.dim() not in (3, 4) or K.shape[rows] < want[rows]
                or tuple(K.shape[:rows]) != want[:rows] or tuple(K.shape[rows + 1:]) != want[rows + 1:]
                or self._strides(K) != self._strides(V)):
            raise ValueError(f"K and V are {tuple(K.shape)} and {tuple(V.shape)}, the plan needs {want} and equal strides")
        if q.stride(2) != 1 or (self.Hq > 1 and q.stride(1) != D) or K.stride(-1) != 1 or V.stride(-1) != 1:
            raise ValueError("the head dimension (and the heads of q) must be contiguous")
        if not packed and self.B > 1 and K.stride(0) == 0:   # (the call takes a stride of 0 for packed rows)
            raise ValueError("K and V are expanded over the sequences: each needs rows of its own")
        q_ld = q.stride(0) if self.total_q > 1 else self.Hq * D
        out = torch.empty(self.total_q, self.Hq, D, dtype=q.dtype, device=q.device) if out is None else out
        if not out.is_contiguous() or (lse is not None and not lse.is_contiguous()):
            raise ValueError("out and lse must be contiguous")
        rbq.rbq_prefill_attention(self.B, self.Hq, self.Hkv, D, q, q_ld, K, V, *self._strides(K), K.shape[rows], self.cu_q,
                                  self.cu_k, self.total_q, self.max_k, self.causal, self.sm_scale, out, lse, self.ws, stream)
        return out


class ChunkAttention:
    """The attention of chunks of prompts whose earlier rows are in a Kv4Cache (rbq_prefill_attention_kv4): q_lens tokens
    and n_lens cached rows per sequence of the cache; the lengths' device arrays and the workspace are kept for every
    call (calls that overlap in time, on several streams, need plans of their own). Rows that are not in the cache yet,
    as a session's window, go before the new tokens' among q, K and V (DecodeSession.turn does so)."""

    def __init__(self, Hq, cache, q_lens, n_lens, causal=True):
        if len(q_lens) != cache.B or len(n_lens) != cache.B or min(min(q_lens), min(n_lens)) < 0:
            raise ValueError("one length of at least 0 per sequence of the cache, for the tokens and for the cached rows")
        if max(n_lens) > cache.cap:
            raise ValueError(f"{max(n_lens)} cached rows, the cache holds {cache.cap}")
        if sum(map(int, q_lens)) >= 1 << 31:   # (the call counts in int32)
            raise ValueError("2^31 tokens and more")
        self.cache, self.Hq, self.causal, device = cache, Hq, causal, cache.kv4.device
        cu = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
        self.total_q, self.n = int(cu[-1]), int(max(n_lens))
        self.cu_q, self.seq_n = (torch.from_numpy(np.asarray(v, np.int32)).to(device) for v in (cu, n_lens))
        self.ws = rbq.workspace(rbq.RBQ_OP_PREFILL_KV4, cache.B, Hq, cache.Hkv, cache.D, self.n, self.total_q, device)
        self.sm_scale = 1.0 / math.sqrt(cache.D)

    def _strides(self, t):
        """Of K or V, from a row and a head to the next (a dimension of one entry has no stride that means anything)."""
        c = self.cache
        return t.stride(0) if self.total_q > 1 else c.Hkv * c.D, t.stride(1) if c.Hkv > 1 else c.D

    def __call__(self, q, K, V, out=None, lse=None, stream=None):
        """q [total_q][Hq][D]; K, V [total_q][Hkv][D], the chunks' own rows; any strides whose last dimension (of q: two)
        is contiguous. Returns out [total_q][Hq][D] in q's type."""
        c, T = self.cache, self.total_q
        if tuple(q.shape[1:]) != (self.Hq, c.D) or q.shape[0] < T:
            raise ValueError(f"q is {tuple(q.shape)}, the plan needs ({T}, {self.Hq}, {c.D})")
        if (K.shape != V.shape or tuple(K.shape[1:]) != (c.Hkv, c.D) or K.shape[0] < T
                or self._strides(K) != self._strides(V)):
            raise ValueError(f"K and V are {tuple(K.shape)} and {tuple(V.shape)}, the plan needs ({T}, {c.Hkv}, {c.D}) and "
                             "equal strides")
        if q.stride(2) != 1 or (self.Hq > 1 and q.stride(1) != c.D) or K.stride(2) != 1 or V.stride(2) != 1:
            raise ValueError("the head dimension (and the heads of q) must be contiguous")
        q_ld = q.stride(0) if T > 1 else self.Hq * c.D
        kv_ld, kv_head = self._strides(K)
        out = torch.empty(T, self.Hq, c.D, dtype=q.dtype, device=q.device) if out is None else out
        if not out.is_contiguous() or (lse is not None and not lse.is_contiguous()):
            raise ValueError("out and lse must be contiguous")
        rbq.rbq_prefill_attention_kv4(c.B, self.Hq, c.Hkv, c.D, q, q_ld, K, V, kv_ld, kv_head, self.cu_q, T, c.kv4, c.par,
                                      c.code, c.cap, self.n, self.seq_n, self.causal, self.sm_scale, out, lse, self.ws, stream)
        return out


class DecodeSession:
    """A decode loop over one growing cache: the lazy index update of Section
    3.4 as a serving loop would run it. The cache holds `cap` rows per (sequence,
    KV head). The prefill rows [0, n) are indexed once (with their centroid);
    each generated token's key and value are appended to the window after the
    indexed rows, each step attends over the Top-p selection of the index plus
    the whole window (one rbq_decode_step), and the step that finds the window
    full also flushes it into the index (encoded with the prefill centroid), so
    the next step scores n + window keys. Buffers and workspaces are sized once,
    for the largest index the cache can hold.

    K, V: [B][Hkv][cap][D] device tensors holding the prefill rows; P: the
    rotation; c_q: query centroids or None; compact: the fp16-factor index
    (then without c_q).

    kv8 ("e4m3" or "int8"): the indexed rows are kept in 8 bits (kv8_block tokens per
    scale), the window in K's type in buffers of its own; K and V [B][Hkv][at least
    n_prefill][D] are then read here only, and every step is one rbq_decode_step_kv8.

    kv4 ("fp4" or "int4"): the same in 4 bits, every step one rbq_decode_step_kv4. turn() takes a further turn's tokens at
    once."""

    def __init__(self, B, Hq, Hkv, D, cap, n_prefill, window, K, V, P, c_q=None, device="cuda", compact=False, kv8=None,
                 kv8_block=64, kv4=None):
        if kv8 is not None and kv4 is not None:
            raise ValueError("the indexed rows are kept in 8 bits or in 4, not both")
        if not 0 < window <= rbq.RBQ_MAX_WINDOW or n_prefill + window > cap:
            raise ValueError("the window must fit after the prefill rows (n_prefill + window <= cap)")
        q = torch.zeros(B, Hq, D, dtype=torch.float32, device=device)
        # Every flush adds a whole window to the index, and append() keeps
        # n + w <= cap, so the index sizes a step can see are n_prefill + k * window
        # up to cap (the last one may leave less than a window of room, and the
        # steps after it run with that index and a partial window).
        self.n_sizes = list(range(n_prefill, cap + 1, window))
        self.n_max = self.n_sizes[-1]
        # sized for the largest index: the scores, selections and per-row workspaces grow with n
        self.kv8 = self.kv4 = None
        src, src_ld = K, cap          # the prefill rows and their number per block
        if kv8 is not None or kv4 is not None:
            src_ld = K.shape[2]
            if src_ld < n_prefill or not (K.is_contiguous() and V.is_contiguous() and K.shape == V.shape):
                raise ValueError("K and V must be contiguous, of one shape, and hold the prefill rows")
            if kv8 is not None:
                self.kv8 = Kv8Cache(B, Hkv, D, cap, kv8, kv8_block, device)
            else:
                self.kv4 = Kv4Cache(B, Hkv, D, cap, kv4, device)
            (self.kv8 or self.kv4).append(K, V, src_ld, n_prefill, 0)
            self.K_win, self.V_win = (torch.zeros(B, Hkv, window, D, dtype=K.dtype, device=device) for _ in range(2))
            K = V = None              # (the state's calls over a full-precision cache have none to read)
        self.state = DecodeState(B, Hq, Hkv, D, cap, self.n_max, window, K, V, q, P, c_q, device, compact)
        self.n, self.w, self.window = n_prefill, 0, window
        st = self.state
        # the step workspace is not monotonic in n (smaller indexes may take more,
        # shorter decode splits): size it for every index size the loop will pass;
        # for a given n it grows with the window rows, so the full window bounds it
        op = (rbq.RBQ_OP_DECODE_STEP_KV8 if kv8 is not None else
              rbq.RBQ_OP_DECODE_STEP_KV4 if kv4 is not None else rbq.RBQ_OP_DECODE_STEP)
        need = max(rbq.rbq_workspace_bytes(op, B, Hq, Hkv, D, m, window) for m in self.n_sizes)
        if need > st.ws_step.numel():
            st.ws_step = torch.empty(need, dtype=torch.uint8, device=device)
        if compact:
            rbq.rbq_encode_keys_f16(B, Hkv, D, src, src_ld, n_prefill, 0, cap, P, st.c_k, st.codes, st.kfac16,
                                    rbq.RBQ_ENCODE_SET_CENTROID, st.ws_encode)
        else:
            rbq.rbq_encode_keys(B, Hkv, D, src, src_ld, n_prefill, 0, cap, P, c_q, st.c_k, st.codes, st.kfac,
                                rbq.RBQ_ENCODE_SET_CENTROID, None, st.ws_encode)

    def append(self, k: torch.Tensor, v: torch.Tensor):
        """Append one token's key and value ([B][Hkv][D]) to the window."""
        if self.w == self.window:
            raise RuntimeError("the window is full: run step() first (it flushes the window)")
        if self.n + self.w >= self.state.cap:
            raise RuntimeError("the cache is full")
        if self.kv8 is not None or self.kv4 is not None:
            self.K_win[:, :, self.w].copy_(k)
            self.V_win[:, :, self.w].copy_(v)
        else:
            r = self.n + self.w
            self.state.K[:, :, r].copy_(k)
            self.state.V[:, :, r].copy_(v)
        self.w += 1

    def step(self, q: torch.Tensor, p: float, stream=None) -> bool:
        """One decode step for the query q [B][Hq][D] at Top-p p; returns whether
        the window was flushed into the index. The outputs are state.out and
        state.lse; the selection is state.sel_idx / state.sel_count (row stride:
        the n of this step, self.n before a flush)."""
        st = self.state
        if self.n > self.n_max or self.n + self.w > st.cap:
            raise RuntimeError(f"index of {self.n} keys + {self.w} window rows exceeds the session's buffers "
                               f"({self.n_max} keys, cap {st.cap})")
        st.q.copy_(q)
        flush = self.w == self.window
        if self.kv8 is not None:
            c = self.kv8
            rbq.rbq_decode_step_kv8(st.B, st.Hq, st.Hkv, st.D, st.q, st.P, st.c_q, st.c_k, c.K8, c.V8, c.block, c.k_scale,
                                    c.v_scale, st.cap, self.n, self.K_win, self.V_win, self.window, self.w, st.codes, st.kfac,
                                    st.kfac16, flush, p, st.sm_scale, st.qplanes, st.qscal, st.scores, st.sel_idx,
                                    st.sel_count, st.out, st.lse, st.ws_step, stream)
        elif self.kv4 is not None:
            c = self.kv4
            rbq.rbq_decode_step_kv4(st.B, st.Hq, st.Hkv, st.D, st.q, st.P, st.c_q, st.c_k, c.kv4, c.par, c.code, st.cap, self.n,
                                    self.K_win, self.V_win, self.window, self.w, st.codes, st.kfac, st.kfac16, flush, p,
                                    st.sm_scale, st.qplanes, st.qscal, st.scores, st.sel_idx, st.sel_count, st.out, st.lse,
                                    st.ws_step, stream)
        elif st.compact:
            rbq.rbq_decode_step_f16(st.B, st.Hq, st.Hkv, st.D, st.q, st.P, st.c_k, st.K, st.V, st.cap, self.n,
                                    self.w, st.codes, st.kfac16, flush, p, st.sm_scale, st.qplanes, st.qscal,
                                    st.scores, st.sel_idx, st.sel_count, st.out, st.lse, st.ws_step, stream)
        else:
            rbq.rbq_decode_step(st.B, st.Hq, st.Hkv, st.D, st.q, st.P, st.c_q, st.c_k, st.K, st.V, st.cap, self.n,
                                self.w, st.codes, st.kfac, flush, p, st.sm_scale, st.qplanes, st.qscal, st.scores,
                                st.sel_idx, st.sel_count, st.out, st.lse, st.ws_step, stream)
        self.last_n, self.last_w = self.n, self.w
        if flush:
            self.n += self.w
            self.w = 0
        return flush

    def turn(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> torch.Tensor:
        """A further turn of T tokens a sequence, over a 4-bit cache: their attention, causal, over every row that the
        session holds, the window's among them, and then their rows entered as append() and step() enter them, whole
        windows into the cache and the index, up to `window` rows kept in the window. q [B][T][Hq][D], k and v
        [B][T][Hkv][D] in the window's type; returns [B][T][Hq][D]. On the current stream."""
        st, c = self.state, self.kv4
        if c is None:
            raise ValueError("a turn attends over a 4-bit cache: the session needs kv4")
        T = q.shape[1]
        if tuple(q.shape) != (st.B, T, st.Hq, st.D) or tuple(k.shape) != (st.B, T, st.Hkv, st.D) or v.shape != k.shape:
            raise ValueError(f"q, k and v are {tuple(q.shape)}, {tuple(k.shape)} and {tuple(v.shape)}")
        if not q.dtype == k.dtype == v.dtype == self.K_win.dtype:
            raise ValueError(f"q, k and v are {q.dtype}, {k.dtype} and {v.dtype}, the window {self.K_win.dtype}")
        rows = self.w + T
        if self.n + rows > st.cap:
            raise RuntimeError(f"{self.n + rows} rows exceed the cache's {st.cap}")
        if T == 0:
            return torch.empty_like(q)
        # The window's rows are the first of the chunk's own; their queries are zeros, and what those give is not used.
        own = [torch.cat([win[:, :, :self.w], x.transpose(1, 2)], dim=2).contiguous()
               for win, x in ((self.K_win, k), (self.V_win, v))]
        K, V = (x.transpose(1, 2).reshape(st.B * rows, st.Hkv, st.D) for x in own)
        q = torch.cat([q.new_zeros(st.B, self.w, st.Hq, st.D), q], dim=1).reshape(st.B * rows, st.Hq, st.D)
        out = ChunkAttention(st.Hq, c, [rows] * st.B, [self.n] * st.B)(q, K, V)
        out = out.view(st.B, rows, st.Hq, st.D)[:, self.w:]
        flush = (rows - 1) // self.window * self.window
        if flush > 0:
            if st.compact:
                rbq.rbq_encode_keys_f16(st.B, st.Hkv, st.D, own[0], rows, flush, self.n, st.cap, st.P, st.c_k, st.codes,
                                        st.kfac16, 0, None)
            else:
                rbq.rbq_encode_keys(st.B, st.Hkv, st.D, own[0], rows, flush, self.n, st.cap, st.P, st.c_q, st.c_k, st.codes,
                                    st.kfac, 0, None, None)
            c.append(*own, rows, flush, self.n)
        for win, x in ((self.K_win, own[0]), (self.V_win, own[1])):
            win[:, :, :rows - flush].copy_(x[:, :, flush:])
        self.n, self.w = self.n + flush, rows - flush
        return out
