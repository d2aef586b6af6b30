"""The ends of what the serving calls take."""
import ctypes

import pytest
import torch

import _serve_ref as REF

pytestmark = pytest.mark.gpu
F32, BF16, U8, I32 = torch.float32, torch.bfloat16, torch.uint8, torch.int32


def _new(dt, *s):
    return torch.zeros(*s, dtype=dt, device="cuda")


def test_empty_batch_is_refused(cuda_lib):
    """A table of no sequences is a ValueError when the cache is made, and in the calls themselves."""
    from paper_2308_13137_gb300 import _lib, serve
    c = serve.KVCache.empty(4, 2, 16, 3, 2)
    with pytest.raises(ValueError):
        serve.KVCache(c.k, c.v, c.k_scale, c.v_scale, c.table[:0], c.kv_len[:0])
    with pytest.raises(ValueError):
        serve.KVCache.empty(4, 2, 16, 0, 2)
    none = _lib.omq_kv_cache.from_buffer_copy(c.handle)
    none.B = 0
    at, bind, rope = ctypes.addressof(none), serve._load_bind(), serve.rope_table(32)
    for n in (0, 3):
        qkv, q = _new(F32, n, 8 * 128), _new(BF16, n, 4 * 128)
        for cu, most in ((None, None), (_new(I32, 1), 1)):
            with pytest.raises(ValueError):
                bind.kv_append(at, qkv, rope, 4, cu, most, None, q, None, None, c.status)
            with pytest.raises(ValueError):
                bind.kv_attention(at, q, 4, cu, most, 32, q, None, c.status)


@pytest.mark.parametrize("M,N,K", [(400, 776, 2064), (2048, 4096, 4096), (300, 2056, 8192)])
def test_every_launch_of_a_product_is_counted(cuda_lib, M, N, K):
    """omq_launch_count: the widening launch, the product, and the joining launch where K is split: the workspace has room for
    partial sums then, beyond the widened codes and their sums.  (Few rows: one launch, no workspace.)"""
    from paper_2308_13137_gb300 import _lib, serve
    a, w = _new(U8, M, K), _new(U8, N, K)
    ah, wh = _new(F32, M), _new(F32, N)
    need = _lib.omq_qgemm_i8_workspace_size(M, N, K)
    want = 1 if need == 0 else (3 if need > 2 * M * K + 4 * (M + 3) else 2)      # the register form: one
    before = _lib.omq_launch_count()
    serve.qgemm(a, ah, None, w, wh, None)
    assert _lib.omq_launch_count() - before == want


@pytest.mark.parametrize("M,N,K", [(65535 * 32, 8, 16), (65535 * 32 + 40, 8, 16), (2200000, 128, 128), (3000000, 64, 256)])
def test_many_rows_of_a_small_product(cuda_lib, M, N, K):
    """More rows than the register form's grid has room for; every output equals the exact one."""
    from paper_2308_13137_gb300 import serve
    g = torch.Generator(device="cuda").manual_seed(M % 1000)
    a = torch.randint(0, 256, (M, K), generator=g, device="cuda", dtype=torch.int32).to(U8)
    w = torch.randint(0, 256, (N, K), generator=g, device="cuda", dtype=torch.int32).to(U8)
    ah, wh = torch.rand(M, generator=g, device="cuda") + 0.5, torch.rand(N, generator=g, device="cuda") + 0.5
    az = torch.randint(0, 256, (M,), generator=g, device="cuda", dtype=torch.int32)
    wz = torch.randint(0, 256, (N,), generator=g, device="cuda", dtype=torch.int32)
    status = _new(I32, 1)
    got = serve.qgemm(a, ah, az, w, wh, wz, status=status)
    assert int(status) == 0
    for lo in range(0, M, 1 << 19):
        s = slice(lo, lo + (1 << 19))
        assert torch.equal(got[s], REF.int_product(a[s], az[s], w, wz).float() * ah[s, None] * wh)


def test_a_prompt_of_many_row_tiles(cuda_lib):
    """1024 query heads on one KV head, 8200 new tokens: 65600 tiles of 128 rows.  Only the newest 40 tokens are in
    the cache, so the rows before them are empty."""
    from paper_2308_13137_gb300 import serve
    heads, rows, held = 1024, 8200, 40
    g = torch.Generator(device="cuda").manual_seed(1)
    c = serve.KVCache.empty(4, 1, 16, 1, 4)
    c.table.copy_(torch.tensor([[2, 0, 3, 1]], dtype=I32))
    c.kv_len.fill_(held)
    for t in (c.k, c.v):
        t.copy_((torch.randn(t.shape, generator=g, device="cuda") * 35 + 128).round().clamp(1, 255))
    c.k_scale.fill_(0.03)
    c.v_scale.fill_(0.03)
    q = _new(BF16, rows, heads * 128)
    q[-held - 1:] = torch.randn(held + 1, heads * 128, generator=g, device="cuda").to(BF16)
    lse = torch.zeros(rows, heads, device="cuda")
    out = serve.kv_attention(c, q, heads, lse=lse)
    c.check()
    assert bool((out[:-held] == 0).all()) and bool((lse[:-held] == -float("inf")).all())
    O, L, top = REF.attention(c, q[-held:], heads, [(0, held)])
    got = out[-held:].double().view(O.shape)
    # weights in fp16, the output in bf16
    assert bool(((got - O).abs() <= 1.5 * 2.0 ** -11 * top[..., None] + 2.0 ** -8 * O.abs()).all())
    assert bool(((lse[-held:].double() - L).abs() <= 1e-4).all())


def test_a_workspace_that_does_not_fit(cuda_lib):
    """A torch.OutOfMemoryError, which a serving loop catches to make room; nothing is launched.  Partial results for
    a bound of 2^30 tokens and 1024 heads are 34 GB, the process is held to 14."""
    from paper_2308_13137_gb300 import _lib, serve
    heads, most = 1024, 1 << 30
    c = serve.KVCache.empty(1, heads, 16, 1, 1)
    c.kv_len.fill_(1)
    q, out = _new(BF16, 1, heads * 128), _new(BF16, 1, heads * 128)
    assert _lib.omq_kv_attention_workspace_size(1, 1, 1, most, heads, heads) > 30e9
    serve._load_bind()
    before = _lib.omq_launch_count()
    torch.cuda.set_per_process_memory_fraction(14e9 / torch.cuda.get_device_properties(0).total_memory)
    try:
        with pytest.raises(torch.cuda.OutOfMemoryError):
            serve.kv_attention(c, q, heads, max_kv=most, out=out)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert _lib.omq_launch_count() == before
    out.fill_(1)
    serve.kv_attention(c, q, heads, max_kv=16, out=out)
    c.check()
    assert bool((out == 0).all())
