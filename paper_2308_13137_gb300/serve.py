"""Serving a calibrated block in 8 bits, on torch tensors.

The functions check their arguments and pass them to the entry points of include/omq.h on the
current stream; outputs that are not given are allocated by torch.  Rows of activations may be
strided views (the last dimension contiguous).

* rmsnorm_quant  residual addition, RMSNorm with the folded gain and bias, per-token 8-bit codes
* qgemm          product of 8-bit codes with a step and zero point per token and output channel
* kv_append      rotary positions, the [Q, K] scale, and the write into an 8-bit paged cache
* kv_attention   attention of every sequence's newest tokens over that cache
* KVCache        the cache's tensors and the handle the calls take
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import _lib

F32, BF16 = torch.float32, torch.bfloat16
HEAD_DIM = 128
_DTYPE = {F32: 0, BF16: 1}
_cfgs = {}


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _rows(t, what: str, dtypes, cols: Optional[int] = None, rows: Optional[int] = None):
    """Row stride of a 2-D device tensor with contiguous rows."""
    if (t.dim() != 2 or t.dtype not in dtypes or (t.stride(1) != 1 and t.shape[1] > 1) or not t.is_cuda or
            (cols is not None and t.shape[1] != cols) or (rows is not None and t.shape[0] != rows)):
        want = "/".join(str(d).replace("torch.", "") for d in dtypes)
        raise ValueError(f"{what}: a device tensor [{rows if rows is not None else 'n'}, {cols if cols is not None else 'n'}] "
                         f"of {want} with contiguous rows, got {t.dtype} {tuple(t.shape)}")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _vec(t, what: str, dtype, n: int):
    if t is not None and (t.dtype != dtype or t.numel() != n or not t.is_contiguous()):
        raise ValueError(f"{what}: {n} contiguous values of {str(dtype).replace('torch.', '')}, got {t.dtype} {tuple(t.shape)}")


def _cfg(bits: int, h_eps: float):
    c = _cfgs.get((bits, h_eps))
    if c is None:
        c = _cfgs[(bits, h_eps)] = _lib.make_cfg(16, bits, 0, 0, h_eps)
    return c


class QuantRows(NamedTuple):
    """Quantized rows: uint8 codes [T, C], step h [T] and zero point z [T] (int32); optionally the bf16
    values (codes - z) h and the residual stream after the addition."""
    codes: Optional[torch.Tensor]
    h: Optional[torch.Tensor]
    z: Optional[torch.Tensor]
    values: Optional[torch.Tensor] = None
    residual: Optional[torch.Tensor] = None


def rmsnorm_quant(x, r=None, gain=None, bias=None, bits: int = 8, rms_eps: float = 1e-6, h_eps: float = 1e-5,
                  values: bool = False, out: Optional[QuantRows] = None) -> QuantRows:
    """t = x + r; y = t / sqrt(mean(t^2) + rms_eps) * gain + bias; codes, h, z = the per-token MinMax
    quantizer of y (omq_rmsnorm_quant).  x [T, C] fp32 or bf16; r [T, C] fp32 or bf16 or None; gain,
    bias [C] fp32 or None.  out: buffers to fill (its residual may be r); else they are allocated, the bf16
    values only with values=True and the residual sum only with r."""
    ldx = _rows(x, "x", (F32, BF16))
    T, C = x.shape
    if out is None:
        new = lambda dt, *s: torch.empty(*s, dtype=dt, device=x.device)  # noqa: E731
        quant = bits < 16
        out = QuantRows(new(torch.uint8, T, C) if quant else None, new(F32, T) if quant else None,
                        new(torch.int32, T) if quant else None, new(BF16, T, C) if values or not quant else None,
                        torch.empty(T, C, dtype=r.dtype, device=x.device) if r is not None else None)
    codes, h, z, vals, res = out
    r_dtype, ldr = 0, C
    if r is not None:
        ldr = _rows(r, "r", (F32, BF16), C, T)
        r_dtype = _DTYPE[r.dtype]
    if res is not None:
        ld = _rows(res, "residual", (F32, BF16), C, T)
        _need(r is None or (res.dtype == r.dtype and (ld == ldr or T == 1)), "residual: the type and row stride of r")
        r_dtype, ldr = _DTYPE[res.dtype], ld
    _vec(gain, "gain", F32, C)
    _vec(bias, "bias", F32, C)
    _vec(codes, "codes", torch.uint8, T * C)
    _vec(h, "h", F32, T)
    _vec(z, "z", torch.int32, T)
    _vec(vals, "values", BF16, T * C)
    _lib.omq_rmsnorm_quant(T, C, x, _DTYPE[x.dtype], ldx, r, res, r_dtype, ldr, gain, bias, rms_eps, codes, vals, h, z,
                           _cfg(bits, h_eps))
    return out


def qgemm(a, a_h, a_z, w, w_h, w_z, bias=None, out=None, out_dtype=F32, status=None):
    """Y[m, n] = a_h[m] w_h[n] sum_k (a[m, k] - a_z[m]) (w[n, k] - w_z[n]) + bias[n] (omq_qgemm_i8).
    a [M, K], w [N, K] uint8 codes; steps fp32; zero points int32 or None (= 128)."""
    lda = _rows(a, "a", (torch.uint8,))
    M, K = a.shape
    ldw = _rows(w, "w", (torch.uint8,), K)
    N = w.shape[0]
    _need(a_h is not None and w_h is not None, "a_h, w_h: the steps are required")
    _vec(a_h, "a_h", F32, M)
    _vec(w_h, "w_h", F32, N)
    _vec(a_z, "a_z", torch.int32, M)
    _vec(w_z, "w_z", torch.int32, N)
    _vec(bias, "bias", F32, N)
    if out is None:
        out = torch.empty(M, N, dtype=out_dtype, device=a.device)
    ldc = _rows(out, "out", (F32, BF16), N, M)
    f32 = out.dtype == F32
    need = _lib.omq_qgemm_i8_workspace_size(M, N, K)
    ws = torch.empty(need, dtype=torch.uint8, device=a.device) if need else None
    _lib.omq_qgemm_i8(M, N, K, a, lda, a_h, a_z, w, ldw, w_h, w_z, bias, out if f32 else None, None if f32 else out, ldc,
                      ws, status)
    return out


class KVCache:
    """The pages of an 8-bit key / value cache and what the calls need to find a sequence in them.

    k, v [n_pages, n_kv, page, 128] uint8 codes and k_scale, v_scale [n_pages, n_kv] fp32: a value is
    (code - 128) scale.  table [B, max_pages] int32 page ids, kv_len [B] int32 tokens of every sequence
    (those of the next call included).  The tensors are the caller's and stay alive with the handle; table
    and kv_len may be refilled in place between calls."""

    def __init__(self, k, v, k_scale, v_scale, table, kv_len):
        n_pages, n_kv, page, hd = k.shape
        _need(k.dim() == 4 and hd == HEAD_DIM and v.shape == k.shape, "k, v: [n_pages, n_kv, page, 128]")
        _need(page in (16, 32, 64, 128), "page: 16, 32, 64 or 128 tokens")
        for t, name, dt in ((k, "k", torch.uint8), (v, "v", torch.uint8), (k_scale, "k_scale", F32),
                            (v_scale, "v_scale", F32), (table, "table", torch.int32), (kv_len, "kv_len", torch.int32)):
            _need(t.is_cuda and t.is_contiguous() and t.dtype == dt, f"{name}: contiguous device tensor of {dt}")
        _need(k_scale.shape == (n_pages, n_kv) and v_scale.shape == (n_pages, n_kv), "scales: [n_pages, n_kv]")
        _need(table.dim() == 2 and kv_len.dim() == 1 and kv_len.shape[0] == table.shape[0], "table [B, n], kv_len [B]")
        self.k, self.v, self.k_scale, self.v_scale, self.table, self.kv_len = k, v, k_scale, v_scale, table, kv_len
        self.n_kv, self.page, self.B = n_kv, page, table.shape[0]
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self.handle = _lib.omq_kv_cache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                                        table.data_ptr(), kv_len.data_ptr(), n_pages, n_kv, page, table.shape[1], self.B)

    @classmethod
    def empty(cls, n_pages: int, n_kv: int, page: int, B: int, max_pages: int, device="cuda") -> "KVCache":
        new = lambda dt, *s: torch.zeros(*s, dtype=dt, device=device)  # noqa: E731
        return cls(new(torch.uint8, n_pages, n_kv, page, HEAD_DIM), new(torch.uint8, n_pages, n_kv, page, HEAD_DIM),
                   new(F32, n_pages, n_kv), new(F32, n_pages, n_kv), new(torch.int32, B, max_pages),
                   new(torch.int32, B))

    def check(self, stream=None):
        """Raises when a call met a page id or length out of range (waits for the stream)."""
        code = _lib.omq_stream_status(self.status, stream)
        if code:
            self.status.zero_()
            raise _lib.OmqError("KVCache", code)


def _row_map(cache, rows: int, cu_q, max_q):
    if cu_q is None:
        _need(rows % cache.B == 0 and max_q in (None, rows // cache.B), "rows: the same number for every sequence without cu_q")
        return rows // cache.B
    _need(max_q is not None, "max_q: needed with cu_q")
    _vec(cu_q, "cu_q", torch.int32, cache.B + 1)
    return max_q


def rope_table(n_pos: int, theta: float = 10000.0, device="cuda"):
    """Interleaved (cos, sin) of every position and frequency, [n_pos, 64, 2] fp32."""
    out = torch.empty(n_pos, HEAD_DIM // 2, 2, dtype=F32, device=device)
    _lib.omq_rope_table(n_pos, theta, out)
    return out


def kv_append(cache: KVCache, qkv, rope, n_heads: int, cu_q=None, max_q: Optional[int] = None, sa=None, q_out=None,
              k_out=None, v_out=None):
    """Turns the new rows' q and k, scales them by 1 / sa and sa, writes k and v into the cache and returns q
    in bf16 (omq_kv_append).  qkv [rows, (n_heads + 2 n_kv) 128] fp32 or bf16.  k_out, v_out [rows, n_kv*128]
    bf16 receive the values that the new codes stand for."""
    G = cache.n_kv
    ld = _rows(qkv, "qkv", (F32, BF16), (n_heads + 2 * G) * HEAD_DIM)
    rows = qkv.shape[0]
    max_q = _row_map(cache, rows, cu_q, max_q)
    _need(rope.dim() == 3 and rope.shape[1:] == (64, 2) and rope.dtype == F32, "rope: [n_pos, 64, 2] fp32")
    _vec(sa, "sa", F32, G * HEAD_DIM)
    if q_out is None:
        q_out = torch.empty(rows, n_heads * HEAD_DIM, dtype=BF16, device=qkv.device)
    ldq = _rows(q_out, "q_out", (BF16,), n_heads * HEAD_DIM, rows)
    ldkv = 0
    if k_out is not None or v_out is not None:
        _need(k_out is not None and v_out is not None, "k_out, v_out: both or neither")
        ldkv = _rows(k_out, "k_out", (BF16,), G * HEAD_DIM, rows)
        _need(_rows(v_out, "v_out", (BF16,), G * HEAD_DIM, rows) == ldkv, "v_out: the row stride of k_out")
    _lib.omq_kv_append(cache.handle, rows, max_q, cu_q, n_heads, qkv, _DTYPE[qkv.dtype], ld, rope, rope.shape[0], sa,
                       q_out, ldq, k_out, v_out, ldkv, cache.status)
    return q_out


def kv_attention(cache: KVCache, q, n_heads: int, cu_q=None, max_q: Optional[int] = None, max_kv: Optional[int] = None,
                 out=None, out_dtype=BF16, lse=None):
    """Causal attention of the rows q [rows, n_heads*128] bf16 over the cache (omq_kv_attention): row i of a
    sequence sees every key up to its own token.  max_kv: a bound of kv_len (default: what the table can
    hold).  lse [rows, n_heads] fp32 receives the base-2 log-sum-exp."""
    ldq = _rows(q, "q", (BF16,), n_heads * HEAD_DIM)
    rows = q.shape[0]
    max_q = _row_map(cache, rows, cu_q, max_q)
    if max_kv is None:
        max_kv = cache.table.shape[1] * cache.page
    if out is None:
        out = torch.empty(rows, n_heads * HEAD_DIM, dtype=out_dtype, device=q.device)
    ldo = _rows(out, "out", (F32, BF16), n_heads * HEAD_DIM, rows)
    _vec(lse, "lse", F32, rows * n_heads)
    need = _lib.omq_kv_attention_workspace_size(cache.B, rows, max_q, max_kv, n_heads, cache.n_kv)
    ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    f32 = out.dtype == F32
    _lib.omq_kv_attention(cache.handle, rows, max_q, cu_q, max_kv, n_heads, q, ldq, out if f32 else None,
                          None if f32 else out, ldo, lse, ws, cache.status)
    return out
