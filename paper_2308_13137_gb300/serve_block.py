"""A calibrated decoder block run in 8 bits: the packed form of BlockState.fold_pack as it is, over an
8-bit paged cache.

One call of ServedBlock.forward takes any number of new tokens of every sequence (a prompt, one token
each, or several to verify) through

    norm + codes -> q|k|v product -> rotary, cache write -> attention over the cache -> codes ->
    o product -> residual, norm + codes -> gate|up product -> silu(gate) up -> codes -> down product

with the entry points of include/omq.h; torch adds silu(gate) up.  `python -m
paper_2308_13137_gb300.serve_block` packs a random LLaMA-7B-shaped block, writes a prompt and decodes.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import _lib, serve

F32, BF16, U8, I32 = torch.float32, torch.bfloat16, torch.uint8, torch.int32


def unpack_codes(packed: torch.Tensor, bits: int) -> torch.Tensor:
    """uint8 codes [rows, cols] of the little-endian bit stream that fold_pack writes per row (code i at
    bits [bits i, bits i + bits))."""
    if bits == 8:
        return packed
    rows, nbytes = packed.shape
    b = (packed[:, :, None] >> torch.arange(8, dtype=U8, device=packed.device)) & 1
    b = b.reshape(rows, nbytes * 8 // bits, bits).to(I32)
    return (b << torch.arange(bits, dtype=I32, device=packed.device)).sum(-1).to(U8)


class ServedBlock:
    """Weights of one calibrated block (wbits 2..8, one group per output channel) for 8-bit serving."""

    def __init__(self, shape, packed, wbits: int, abits: int = 8, device: str = "cuda"):
        if not 2 <= wbits <= 8 or not 2 <= abits <= 8:
            raise ValueError("wbits, abits: 2 to 8")
        self.shape, self.abits, self.device = shape, abits, device
        dev = lambda t: t.to(device).contiguous()  # noqa: E731
        self.w = {}
        for k in ("qkv", "o", "gu", "d"):
            if packed["h_" + k].shape[1] != 1:
                raise ValueError("weight groups: the 8-bit product takes one step per output channel")
            self.w[k] = (unpack_codes(dev(packed["codes_" + k]), wbits), dev(packed["h_" + k]).view(-1),
                         dev(packed["z_" + k]).view(-1))
        get = lambda n: dev(packed[n]) if n in packed else None  # noqa: E731
        self.bias = dict(qkv=get("b_qkv"), o=get("b_o"), gu=get("b_gu"), d=None)
        self.ln = [(get(f"ln{i}_gain"), get(f"ln{i}_bias")) for i in (1, 2)]
        self.sa = get("sa")
        self.cfg = _lib.make_cfg(16, abits, 0, 0, 1e-5)

    @classmethod
    def from_state(cls, st, abits: int = 8) -> "ServedBlock":
        """The block of a calibrated BlockState."""
        return cls(st.shape, st.fold_pack(), st.wbits, abits, st.device)

    def cache(self, B: int, max_tokens: int, page: int = 64) -> serve.KVCache:
        """A cache of B sequences of up to max_tokens tokens on the block's device, its pages in order."""
        per = -(-max_tokens // page)
        c = serve.KVCache.empty(B * per, self.shape.n_kv, page, B, per, device=self.device)
        c.table.copy_(torch.arange(B * per, dtype=I32).view(B, per))
        return c

    def _product(self, name: str, rows: serve.QuantRows, status, out_dtype=F32):
        w, h, z = self.w[name]
        return serve.qgemm(rows.codes, rows.h, rows.z, w, h, z, bias=self.bias[name], out_dtype=out_dtype, status=status)

    def _norm(self, i: int, x, r=None) -> serve.QuantRows:
        g, b = self.ln[i]
        return serve.rmsnorm_quant(x, r, g, b, bits=self.abits, rms_eps=self.shape.rms_eps)

    def _codes(self, x) -> serve.QuantRows:
        T, C = x.shape
        new = lambda dt, *s: torch.empty(*s, dtype=dt, device=x.device)  # noqa: E731
        q = serve.QuantRows(new(U8, T, C), new(F32, T), new(I32, T), new(BF16, T, C))
        _lib.omq_act_quant_per_token(T, C, x, None, None, q.values, q.codes, q.h, q.z, new(I32, T), new(I32, T), self.cfg)
        return q

    def forward(self, h, cache: serve.KVCache, rope, delta=None, cu_q=None, max_q: Optional[int] = None,
                max_kv: Optional[int] = None):
        """h [rows, d] fp32: the residual stream of the new tokens; delta [rows, d]: the previous block's
        output still to be added to it (fused into this block's first norm).  Returns (h, delta) for the next
        block; the block's output is their sum.  cache.kv_len counts the new tokens already.  cache.check() raises
        when a call met a page id or length out of range, or a wait of any kernel ran out."""
        sh = self.shape
        self.cfg.dev_status = cache.status.data_ptr()    # the quantizer's waits
        n1 = self._norm(0, h) if delta is None else self._norm(0, delta, h)
        if delta is not None:
            h = n1.residual
        qkv = self._product("qkv", n1, cache.status)
        q = serve.kv_append(cache, qkv, rope, sh.n_heads, cu_q=cu_q, max_q=max_q, sa=self.sa)
        o = serve.kv_attention(cache, q, sh.n_heads, cu_q=cu_q, max_q=max_q, max_kv=max_kv, out_dtype=F32)
        n2 = self._norm(1, self._product("o", self._codes(o), cache.status), h)
        gu = self._product("gu", n2, cache.status)
        m = torch.nn.functional.silu(gu[:, :sh.ffn]) * gu[:, sh.ffn:]
        return n2.residual, self._product("d", self._codes(m), cache.status)


def main():
    import argparse
    import time

    from . import inputs as I
    from .block import BlockState
    ap = argparse.ArgumentParser(description="8-bit serving of one packed block: a prompt, then single tokens")
    ap.add_argument("--prompt", type=int, default=2048)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--batch", type=int, default=8)
    a = ap.parse_args()
    shape = I.BlockShape("served", T=128, d=4096, n_heads=32, n_kv=32, ffn=11008, wbits=8, abits=8, group=0, let=1)
    W = I.make_block_weights(shape, seed=0)
    x = I.make_block_input(shape, sample=0, weight_seed=0)
    blk = ServedBlock.from_state(BlockState(shape, W, I.make_block_theta(shape, W, x, seed=0)))
    B, n = a.batch, a.prompt + a.tokens
    cache, rope = blk.cache(B, n), serve.rope_table(n)
    g = torch.Generator(device="cuda").manual_seed(0)
    prompt = torch.randn(B * a.prompt, shape.d, generator=g, device="cuda")
    token = torch.randn(B, shape.d, generator=g, device="cuda")
    for k in range(2):                                   # the first pass warms up
        cache.kv_len.fill_(a.prompt)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        blk.forward(prompt, cache, rope, max_kv=a.prompt)
        torch.cuda.synchronize()
        t1 = time.perf_counter()
        for i in range(a.tokens):
            cache.kv_len.fill_(a.prompt + i + 1)
            blk.forward(token, cache, rope, max_kv=n)
        torch.cuda.synchronize()
        t2 = time.perf_counter()
    cache.check()
    print(f"one LLaMA-7B-shaped block, {B} sequences: {a.prompt}-token prompts {1e3 * (t1 - t0):.2f} ms "
          f"({B * a.prompt / (t1 - t0):.0f} tokens/s), then {1e6 * (t2 - t1) / a.tokens:.0f} us per step of one token each")


if __name__ == "__main__":
    main()
