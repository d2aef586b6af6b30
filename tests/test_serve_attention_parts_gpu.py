"""Cache attention whose tokens are split over CTAs, with scores so large that a part's log-sum-exp in fp32 has no bits for its
sum (omq_kv_attention), against float64."""
import pytest
import torch

import test_serve_attention_scales_gpu as S

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("heads,n_q", S.ROWS)
@pytest.mark.parametrize("page,n_pages", [(64, 20), (16, 300), (128, 70)])
@pytest.mark.parametrize("size", [2.0 ** 8, 2.0 ** 12, 2.0 ** 24, -2.0 ** 24, 2.0 ** 110])
def test_parts_with_unequal_numbers_of_top_tokens(cuda_lib, heads, n_q, page, n_pages, size):
    """Keys of four levels: the top one's tokens stand in all parts, more and more of them towards the end.  Each weighs the
    same; the bounds are S._check's."""
    c = S._cache(n_pages, page, seed=heads + page, tail=5)
    g = torch.Generator(device="cuda").manual_seed(7)
    n = c.k.shape[0]
    level = torch.randint(30, 33, c.k.shape[:3], generator=g, device="cuda")
    chance = torch.arange(n, 0, -1, device="cuda")[:, None, None] / n          # (the pool holds the pages in reversed order)
    top = torch.rand(c.k.shape[:3], generator=g, device="cuda") < 0.2 * chance ** 3
    level[top] = 33 if size > 0 else 29
    c.k.copy_((128 + level)[..., None].expand(c.k.shape))
    q = torch.full((n_q, heads * 128), size, device="cuda").to(BF16)
    S._check(c, heads, n_q, q)
