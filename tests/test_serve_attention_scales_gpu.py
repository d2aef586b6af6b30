"""Cache attention where scores and value scales are far apart (omq_kv_attention), against float64.

Keys are constant per page and queries a power of two, so that every score is exact up to its three fp32
scalings; the bounds follow from that and from the fp16 rounding of the weights."""
import math

import pytest
import torch

import _serve_ref as REF

pytestmark = pytest.mark.gpu
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32

# (query heads of one KV head, new tokens): 1, 12, 24, 48 and 112 rows per KV head
ROWS = [(1, 1), (4, 3), (8, 3), (16, 3), (16, 7)]


def _cache(n_pages, page, seed, tail=0):
    """One sequence of n_pages pages (the last without its `tail` newest slots), its pages in reversed order; keys
    1 everywhere, bell-shaped values, scales 1 and 1 / 30."""
    from paper_2308_13137_gb300 import serve
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = serve.KVCache.empty(n_pages, 1, page, 1, n_pages)
    c.table.copy_(torch.arange(n_pages - 1, -1, -1, dtype=I32)[None])
    c.kv_len.fill_(n_pages * page - tail)
    c.k.fill_(129)
    c.v.copy_((torch.randn(c.v.shape, generator=g, device="cuda") * 35 + 128).round().clamp(1, 255))
    c.k_scale.fill_(1.0)
    c.v_scale.fill_(1.0 / 30)
    return c


def _at(c, i):
    """Pool index of the sequence's page i."""
    return int(c.table[0, i])


def _run(c, heads, n_q, q):
    from paper_2308_13137_gb300 import serve
    lse = torch.empty(n_q, heads, device="cuda")
    out = serve.kv_attention(c, q, heads, out_dtype=F32, lse=lse)
    c.check()
    return out, lse


def _check(c, heads, n_q, q):
    """Weights are rounded to fp16 (2^-11 relative each) and everything else to fp32: an output is within 1.5
    2^-11 of the largest |v| that the row sees.  The log-sum-exp is a score of four fp32 roundings and a
    logarithm of a sum."""
    out, lse = _run(c, heads, n_q, q)
    O, L, top = REF.attention(c, q, heads, [(0, n_q)])
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    assert bool(((out.double().view(O.shape) - O).abs() <= 1.5 * 2.0 ** -11 * top[..., None]).all())
    assert bool(((lse.double() - L).abs() <= 1e-5 + 8 * 2.0 ** -24 * L.abs()).all())
    return out, O


@pytest.mark.parametrize("heads,n_q", ROWS)
@pytest.mark.parametrize("page,n_pages,where", [(16, 12, 0), (16, 12, 5), (64, 5, 1), (128, 40, 3), (16, 40, 38)])
@pytest.mark.parametrize("v_scale", [0.0, 1e-38])
def test_top_score_on_a_page_of_vanishing_values(cuda_lib, heads, n_q, page, n_pages, where, v_scale):
    """The row's top score lies on a page whose V scale is zero (or next to it), the other pages' scores lie a
    gap below it, in log2 units: from weights that still count to ones far below the smallest fp32 number."""
    for gap in (40.0, 100.0, 119.0, 121.0, 135.0, 200.0, 300.0):
        c = _cache(n_pages, page, seed=heads + n_pages)
        q = torch.ones(n_q, heads * 128, device="cuda").to(BF16)
        # score of a key of all ones, scale s: 128 s log2(e) / sqrt(128)
        unit = 128 * math.log2(math.e) / math.sqrt(128)
        c.k_scale.fill_(1e-3 / unit)
        c.k_scale[_at(c, where)] = gap / unit
        c.v_scale[_at(c, where)] = v_scale
        _check(c, heads, n_q, q)


@pytest.mark.parametrize("heads,n_q", ROWS)
@pytest.mark.parametrize("v_scale", [0.04, 4096.0])
@pytest.mark.parametrize("size", [2.0 ** 24, -2.0 ** 24, -2.0 ** 99, -2.0 ** 110, 2.0 ** 99, 2.0 ** 110])
def test_scores_of_any_size(cuda_lib, heads, n_q, v_scale, size):
    """Scores of one sign and any size below the largest fp32 number, no visible score near zero: the row is
    not empty.  Keys differ between tokens by whole codes, so scores that are not equal are far apart."""
    page = 16
    c = _cache(20, page, seed=heads, tail=5)
    g = torch.Generator(device="cuda").manual_seed(3)
    level = torch.randint(20, 120, c.k.shape[:3], generator=g, device="cuda")
    c.k.copy_((128 + level)[..., None].expand(c.k.shape))
    c.v_scale.fill_(v_scale)
    c.v_scale[_at(c, 7)] = v_scale / 512
    q = torch.full((n_q, heads * 128), size, device="cuda").to(BF16)
    out, O = _check(c, heads, n_q, q)
    assert float(O.abs().max()) > 0
    # and beside ordinary scores: half of the pages have keys next to zero
    c.k_scale[: 10] = 2.0 ** -100
    _check(c, heads, n_q, q)
