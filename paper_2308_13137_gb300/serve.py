"""Serving a calibrated block in 8 bits, on torch tensors.

The functions check their arguments and pass them to the entry points of include/omq.h on the
current stream; outputs that are not given are allocated by torch.  Rows of activations may be
strided views (the last dimension contiguous).

* rmsnorm_quant  residual addition, RMSNorm with the folded gain and bias, per-token 8-bit codes
* qgemm          product of 8-bit codes with a step and zero point per token and output channel
* kv_append      rotary positions, the [Q, K] scale, and the write into an 8-bit paged cache
* kv_attention   attention of every sequence's newest tokens over that cache
* KVCache        the cache's tensors and the handle the calls take

Tokens that a smaller model has drafted are checked as a tree of new rows in one step:

* draft_tree     depths and visible rows of the trees, for kv_append and kv_attention (tree=...)
* verify_drafts  the walk that accepts drafted tokens against the target's probabilities, and the new token
* kv_keep        the accepted rows to the front of the newest tokens in every layer's cache
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Sequence, Union

import torch

from . import _lib

F32, BF16 = torch.float32, torch.bfloat16
HEAD_DIM = 128


def _load_bind():
    """The compiled module of the calls; it links libomq.so, so both come from one build."""
    _lib.lib()
    from . import _bind
    return _bind


class _Calls:
    """The module's functions, loaded on first use (importing this file needs no build)."""

    def __getattr__(self, name):
        b = _load_bind()
        for f in ("rmsnorm_quant", "qgemm", "kv_append", "kv_attention", "draft_tree", "kv_append_tree", "kv_attention_tree",
                  "verify_drafts", "kv_keep"):
            setattr(self, f, getattr(b, f))
        return self.__dict__[name]


_calls = _Calls()


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


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
    if out is None:
        _need(x.dim() == 2, "x: [T, C]")
        T, C = x.shape
        new = lambda dt, *s: torch.empty(*s, dtype=dt, device=x.device)  # noqa: E731
        quant = bits < 16
        out = QuantRows(new(torch.uint8, T, C) if quant else None, new(F32, T) if quant else None,
                        new(torch.int32, T) if quant else None, new(BF16, T, C) if values or not quant else None,
                        torch.empty_strided(r.shape, r.stride(), dtype=r.dtype, device=x.device) if r is not None else None)
    codes, h, z, vals, res = out
    code = _calls.rmsnorm_quant(x, r, gain, bias, bits, rms_eps, h_eps, codes, h, z, vals, res)
    if code:
        _lib.check("omq_rmsnorm_quant", code)
    return out


def qgemm(a, a_h, a_z, w, w_h, w_z, bias=None, out=None, out_dtype=F32, status=None):
    """Y[m, n] = a_h[m] w_h[n] sum_k (a[m, k] - a_z[m]) (w[n, k] - w_z[n]) + bias[n] (omq_qgemm_i8).
    a [M, K], w [N, K] uint8 codes; steps fp32; zero points int32 or None (= 128).  status: an int32 device word
    that is set when a wait of the kernel ran out and the output is unfinished (a KVCache's serves: its check
    raises then)."""
    if out is None:
        out = torch.empty(a.shape[0], w.shape[0], dtype=out_dtype, device=a.device)
    code = _calls.qgemm(a, a_h, a_z, w, w_h, w_z, bias, out, status)
    if code:
        _lib.check("omq_qgemm_i8", code)
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
        _need(table.dim() == 2 and kv_len.dim() == 1 and kv_len.shape[0] == table.shape[0] and table.shape[0] > 0,
              "table [B, n], kv_len [B], B at least 1")
        self.k, self.v, self.k_scale, self.v_scale, self.table, self.kv_len = k, v, k_scale, v_scale, table, kv_len
        self.n_kv, self.page, self.B = n_kv, page, table.shape[0]
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self.handle = _lib.omq_kv_cache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                                        table.data_ptr(), kv_len.data_ptr(), n_pages, n_kv, page, table.shape[1], self.B)
        self.address = ctypes.addressof(self.handle)
        self.capacity = table.shape[1] * page            # tokens that a row of the table can name

    @classmethod
    def empty(cls, n_pages: int, n_kv: int, page: int, B: int, max_pages: int, device="cuda") -> "KVCache":
        new = lambda dt, *s: torch.zeros(*s, dtype=dt, device=device)  # noqa: E731
        return cls(new(torch.uint8, n_pages, n_kv, page, HEAD_DIM), new(torch.uint8, n_pages, n_kv, page, HEAD_DIM),
                   new(F32, n_pages, n_kv), new(F32, n_pages, n_kv), new(torch.int32, B, max_pages),
                   new(torch.int32, B))

    def check(self, stream=None):
        """Raises when a call that reports to this cache met a page id or length out of range, or a wait of its
        kernels ran out (waits for the stream)."""
        code = _lib.omq_stream_status(self.status, stream)
        if code:
            self.status.zero_()
            raise _lib.OmqError("KVCache", code)


def rope_table(n_pos: int, theta: float = 10000.0, device="cuda"):
    """Interleaved (cos, sin) of every position and frequency, [n_pos, 64, 2] fp32."""
    out = torch.empty(n_pos, HEAD_DIM // 2, 2, dtype=F32, device=device)
    _lib.omq_rope_table(n_pos, theta, out)
    return out


class DraftTree(NamedTuple):
    """The trees of a step's rows: parent [rows] int32, and what draft_tree makes of it, depth [rows] and the bits of
    the visible rows, seen [rows, words] (int32 words).  cu_q and max_q as in kv_append.  For attention alone the bits may
    be any."""
    parent: torch.Tensor
    depth: torch.Tensor
    seen: torch.Tensor
    cu_q: Optional[torch.Tensor]
    max_q: int


class Verified(NamedTuple):
    """tokens [B, steps] int32: every sequence's accepted tokens and the new one, -1 behind; path [B, steps]: the
    accepted rows (row 0 first), -1 behind; count [B]: how many."""
    tokens: torch.Tensor
    path: torch.Tensor
    count: torch.Tensor


def draft_tree(parent, cu_q=None, max_q: Optional[int] = None, out: Optional[DraftTree] = None, status=None) -> DraftTree:
    """Depths and visible rows of trees of drafted tokens (omq_draft_tree), once per step for all layers.  parent: int32,
    the row of every row's parent within its sequence (before its own; -1 at row 0); [rows] with cu_q and max_q, or
    [B, n] for n rows of every sequence.  out: a DraftTree whose depth and seen are filled; its parent, cu_q and max_q may be
    another step's, and what comes back has this call's.  status: an int32 device word that is set where a parent is out of
    range (a KVCache's serves)."""
    if cu_q is None:
        _need(parent.dim() == 2 and (max_q is None or max_q == parent.shape[1]), "parent: [B, n] without cu_q")
        max_q, parent = parent.shape[1], parent.reshape(-1)
    else:
        _need(parent.dim() == 1 and max_q is not None, "parent: [rows], and max_q, with cu_q")
    if out is None:
        new = lambda *s: torch.empty(*s, dtype=torch.int32, device=parent.device)  # noqa: E731
        out = DraftTree(parent, new(parent.shape[0]), new(parent.shape[0], (max_q + 31) // 32), cu_q, max_q)
    code = _calls.draft_tree(parent, cu_q, max_q, out.depth, out.seen, status)
    if code:
        _lib.check("omq_draft_tree", code)
    if out.max_q != max_q or not _same(out.parent, parent) or not _same(out.cu_q, cu_q):
        out = DraftTree(parent, out.depth, out.seen, cu_q, max_q)
    return out


def _same(a: Optional[torch.Tensor], b: Optional[torch.Tensor]) -> bool:
    """The same int32 values in the same place, whichever tensor objects name them (b has passed the call's checks)."""
    return a is b or (a is not None and b is not None and a.data_ptr() == b.data_ptr() and a.shape == b.shape and
                      a.dtype == b.dtype and a.device == b.device and a.is_contiguous())


def _rows_of(tree: Optional[DraftTree], cu_q, max_q):
    if tree is None:
        return cu_q, max_q
    _need(cu_q is None and max_q is None, "cu_q, max_q: the tree's")
    return tree.cu_q, tree.max_q


def kv_append(cache: KVCache, qkv, rope, n_heads: int, cu_q=None, max_q: Optional[int] = None, sa=None, q_out=None,
              k_out=None, v_out=None, tree: Optional[DraftTree] = None):
    """Turns the new rows' q and k, scales them by 1 / sa and sa, writes k and v into the cache and returns q
    in bf16 (omq_kv_append).  qkv [rows, (n_heads + 2 n_kv) 128] fp32 or bf16.  k_out, v_out [rows, n_kv*128]
    bf16 receive the values that the new codes stand for.  tree: the rows are drafted tokens, at the positions of
    their depths (omq_kv_append_tree); cu_q and max_q are its own then."""
    if q_out is None:
        q_out = torch.empty(qkv.shape[0], n_heads * HEAD_DIM, dtype=BF16, device=qkv.device)
    cu_q, max_q = _rows_of(tree, cu_q, max_q)
    if tree is not None:
        code = _calls.kv_append_tree(cache.address, qkv, rope, n_heads, cu_q, max_q, sa, q_out, k_out, v_out, cache.status,
                                     tree.depth)
        if code:
            _lib.check("omq_kv_append_tree", code)
        return q_out
    code = _calls.kv_append(cache.address, qkv, rope, n_heads, cu_q, max_q, sa, q_out, k_out, v_out, cache.status)
    if code:
        _lib.check("omq_kv_append", code)
    return q_out


def kv_attention(cache: KVCache, q, n_heads: int, cu_q=None, max_q: Optional[int] = None, max_kv: Optional[int] = None,
                 out=None, out_dtype=BF16, lse=None, tree: Optional[DraftTree] = None):
    """Causal attention of the rows q [rows, n_heads*128] bf16 over the cache (omq_kv_attention): row i of a
    sequence sees every key up to its own token.  max_kv: a bound of kv_len (default: what the table can
    hold); the work is cut by it, so give one near the lengths where the table is much longer.  lse [rows, n_heads] fp32 receives the base-2 log-sum-exp.
    tree: row i sees the tokens before its sequence's rows, and of the rows those that its bits name
    (omq_kv_attention_tree); cu_q and max_q are the tree's own then."""
    if out is None:
        out = torch.empty(q.shape[0], n_heads * HEAD_DIM, dtype=out_dtype, device=q.device)
    cu_q, max_q = _rows_of(tree, cu_q, max_q)
    if tree is not None:
        code = _calls.kv_attention_tree(cache.address, q, n_heads, cu_q, max_q, cache.capacity if max_kv is None else max_kv, out,
                                        lse, cache.status, tree.seen)
        if code:
            _lib.check("omq_kv_attention_tree", code)
        return out
    code = _calls.kv_attention(cache.address, q, n_heads, cu_q, max_q, cache.capacity if max_kv is None else max_kv, out, lse,
                               cache.status)
    if code:
        _lib.check("omq_kv_attention", code)
    return out


def verify_drafts(tree: DraftTree, tokens, probs, u, draft_probs=None, steps: Optional[int] = None,
                  out: Optional[Verified] = None, status=None) -> Verified:
    """Walks every sequence's tree from row 0 and accepts drafted tokens so that what comes out is distributed as if drawn
    from the target (omq_verify_drafts).  tokens [rows] int32; probs [rows, V] fp32 or bf16: the target's
    distribution after every row; draft_probs, of the same type: the one from which a row's children were drawn, or
    None where they were chosen (the likeliest, say); u [rows] fp32: uniform numbers in [0, 1), a drafted row's for its test
    and row 0's for the new token.  steps: columns of the outputs, the most rows of a path (default: max_q).
    status: an int32 device word that is set where a parent or token is out of range, or a row that the new token would be
    drawn from adds up to nothing or to 8 and more (a KVCache's serves)."""
    if out is None:
        B = tree.cu_q.shape[0] - 1 if tree.cu_q is not None else tree.parent.shape[0] // tree.max_q
        n = tree.max_q if steps is None else steps
        new = lambda *s: torch.empty(*s, dtype=torch.int32, device=probs.device)  # noqa: E731
        out = Verified(new(B, n), new(B, n), new(B))
    _need(steps is None or out.path.shape[1] == steps, "steps: the columns of out")
    code = _calls.verify_drafts(tree.parent, tree.cu_q, tree.max_q, tokens, probs, draft_probs, u, out.tokens, out.path, out.count,
                                status)
    if code:
        _lib.check("omq_verify_drafts", code)
    return out


def kv_keep(caches: Union[KVCache, Sequence[KVCache]], tree: DraftTree, path, count):
    """Moves the accepted rows of every sequence to the front of its newest tokens, in one cache or every layer's
    (omq_kv_keep): row path[b, j] to place j, for j < count[b], as verify_drafts gives them.  The lengths stay: what follows
    sets kv_len to kv_len - rows + count."""
    caches = (caches,) if isinstance(caches, KVCache) else caches
    code = _calls.kv_keep(tuple(c.address for c in caches), tuple(c.status for c in caches), tree.parent.shape[0], tree.cu_q,
                          tree.max_q, path, count)
    if code:
        _lib.check("omq_kv_keep", code)
