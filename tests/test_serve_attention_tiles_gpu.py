"""Cache attention of many rows: odd and even numbers of 64-token tiles, whose two accumulators end on different
phases, in each of the forms for 24, 48 and 112 rows per KV head, many CTAs of each."""
import pytest
import torch

import _serve_ref as REF

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.mark.parametrize("heads,n_q", [(8, 3), (16, 3), (16, 7)])
@pytest.mark.parametrize("tiles", [1, 2, 3, 4, 5, 7, 8, 9])
def test_tile_counts(cuda_lib, heads, n_q, tiles):
    from paper_2308_13137_gb300 import serve
    B, page = 48, 64
    g = torch.Generator(device="cuda").manual_seed(tiles * 100 + heads + n_q)
    c = serve.KVCache.empty(B * tiles, 1, page, B, tiles)
    c.table.copy_(torch.randperm(B * tiles, generator=torch.Generator().manual_seed(tiles)).view(B, tiles))
    lens = [tiles * 64 - b for b in range(B)]                 # the last tile full, and short by up to 47 tokens
    c.kv_len.copy_(torch.tensor(lens, dtype=I32))
    for t in (c.k, c.v):
        t.copy_((torch.randn(t.shape, generator=g, device="cuda") * 35 + 128).round().clamp(1, 255))
    c.k_scale.copy_(torch.exp(0.3 * torch.randn(c.k_scale.shape, generator=g, device="cuda")) / 30)
    c.v_scale.copy_(torch.exp(torch.randn(c.v_scale.shape, generator=g, device="cuda")) / 30)
    q = torch.randn(B * n_q, heads * 128, generator=g, device="cuda").to(BF16)
    lse = torch.empty(B * n_q, heads, device="cuda")
    out = serve.kv_attention(c, q, heads, out_dtype=F32, lse=lse)
    c.check()
    rows = [(b * n_q, n_q) for b in range(B)]
    O, L, top = REF.attention(c, q, heads, rows)
    # weights are rounded to fp16, everything else to fp32
    assert bool(((out.double().view(O.shape) - O).abs() <= 1.5 * 2.0 ** -11 * top[..., None]).all())
    assert bool(((lse.double() - L).abs() <= 1e-4).all())
    for _ in range(5):
        assert torch.equal(serve.kv_attention(c, q, heads, out_dtype=F32), out)
