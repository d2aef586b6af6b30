"""What the tensor calls of the serving module refuse: wrong devices, types, shapes and strides are a
ValueError, what the C entry point refuses an OmqError, and nothing is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16, U8, I32 = torch.float32, torch.bfloat16, torch.uint8, torch.int32


def _new(dt, *s):
    return torch.zeros(*s, dtype=dt, device="cuda")


def _launches():
    from paper_2308_13137_gb300 import _lib
    return _lib.omq_launch_count()


def _refused(call, kind=ValueError):
    before = _launches()
    with pytest.raises(kind):
        call()
    assert _launches() == before


def test_norm(cuda_lib):
    from paper_2308_13137_gb300 import _lib, serve
    x, r, g = _new(F32, 4, 64), _new(F32, 4, 64), _new(F32, 64)
    for bad in (dict(x=x.cpu()), dict(x=x.half()), dict(x=x[0]), dict(x=x.t()), dict(r=_new(F32, 4, 72)), dict(r=r.double()),
                dict(gain=_new(F32, 63)), dict(gain=g.to(BF16)), dict(gain=g.cpu()), dict(bias=_new(F32, 128)[::2])):
        kw = dict(dict(x=x, r=r, gain=g, bias=None), **bad)
        _refused(lambda: serve.rmsnorm_quant(kw["x"], kw["r"], kw["gain"], kw["bias"]))
    out = serve.QuantRows(_new(U8, 4, 64), _new(F32, 4), _new(I32, 4), None, _new(BF16, 4, 64))
    _refused(lambda: serve.rmsnorm_quant(x, r, out=out))                         # residual of another type than r
    _refused(lambda: serve.rmsnorm_quant(x, r, out=out._replace(residual=None, codes=_new(U8, 4, 65))))
    _refused(lambda: serve.rmsnorm_quant(_new(F32, 4, 60)), _lib.OmqError)       # not a multiple of 8
    _refused(lambda: serve.rmsnorm_quant(x, bits=9), _lib.OmqError)


def test_gemm(cuda_lib):
    from paper_2308_13137_gb300 import _lib, serve
    a, w, ah, wh, z = _new(U8, 4, 64), _new(U8, 16, 64), _new(F32, 4), _new(F32, 16), _new(I32, 4)
    base = dict(a=a, a_h=ah, a_z=None, w=w, w_h=wh, w_z=None, bias=None, out=None)
    for bad in (dict(a=a.cpu()), dict(a=a.to(torch.int8)), dict(w=_new(U8, 16, 48)), dict(a_h=None), dict(w_h=_new(F32, 15)),
                dict(a_z=z.to(torch.int64)), dict(w_z=z), dict(bias=ah), dict(out=_new(F32, 4, 24)), dict(out=_new(F32, 16, 4).t()),
                dict(out=_new(torch.float16, 4, 16)), dict(a=a.t())):
        kw = dict(base, **bad)
        _refused(lambda: serve.qgemm(**kw))
    _refused(lambda: serve.qgemm(**dict(base, a=a[:, :56], w=w[:, :56])), _lib.OmqError)
    _refused(lambda: serve.qgemm(**dict(base, w=_new(U8, 12, 64), w_h=_new(F32, 12))), _lib.OmqError)


def test_cache(cuda_lib):
    from paper_2308_13137_gb300 import _lib, serve
    c = serve.KVCache.empty(4, 2, 16, 3, 2)
    c.kv_len.fill_(1)
    rope, qkv, q, cu = serve.rope_table(32), _new(F32, 3, 8 * 128), _new(BF16, 3, 4 * 128), torch.tensor([0, 1, 2, 3], dtype=I32, device="cuda")
    for f in (lambda: serve.kv_append(c, qkv, rope, 5), lambda: serve.kv_append(c, qkv[:2], rope, 4),
              lambda: serve.kv_append(c, qkv, rope[:, :32], 4), lambda: serve.kv_append(c, qkv, rope, 4, cu_q=cu),
              lambda: serve.kv_append(c, qkv, rope, 4, cu_q=cu[:3], max_q=1), lambda: serve.kv_append(c, qkv, rope, 4, max_q=2),
              lambda: serve.kv_append(c, qkv, rope, 4, k_out=_new(BF16, 3, 256)),
              lambda: serve.kv_append(c, qkv, rope, 4, q_out=_new(F32, 3, 512)),
              lambda: serve.kv_append(c, qkv, rope, 4, sa=_new(F32, 128)), lambda: serve.kv_append(c, qkv.cpu(), rope, 4),
              lambda: serve.kv_attention(c, q, 5), lambda: serve.kv_attention(c, q.float(), 4),
              lambda: serve.kv_attention(c, q, 4, out=_new(BF16, 2, 512)), lambda: serve.kv_attention(c, q, 4, lse=_new(F32, 3)),
              lambda: serve.kv_attention(c, q.cpu(), 4), lambda: serve.kv_attention(c, q, 4, cu_q=cu.long(), max_q=1)):
        _refused(f)
    _refused(lambda: serve.kv_attention(c, q, 4, max_kv=0), _lib.OmqError)
    _refused(lambda: serve.kv_attention(c, _new(BF16, 3, 3 * 128), 3), _lib.OmqError)        # 3 heads over 2 KV heads
    for bad in (lambda: serve.KVCache(c.k, c.v, c.k_scale, c.v_scale, c.table.long(), c.kv_len),
                lambda: serve.KVCache(c.k[:, :, :8], c.v[:, :, :8], c.k_scale, c.v_scale, c.table, c.kv_len),
                lambda: serve.KVCache(c.k.cpu(), c.v, c.k_scale, c.v_scale, c.table, c.kv_len),
                lambda: serve.KVCache(c.k, c.v, c.k_scale[:, :1], c.v_scale, c.table, c.kv_len),
                lambda: serve.KVCache(c.k, c.v, c.k_scale, c.v_scale, c.table, c.kv_len[:2])):
        _refused(bad)
