"""Attention of draft trees where scores and value scales are far apart (omq_kv_attention_tree), against float64: the
causal attention's hard inputs in all forms of the trees' kernels, and the log-sum-exp beside pages of vanishing values."""
import math

import pytest
import torch

import _drafts_ref as D
import test_serve_attention_scales_gpu as S

pytestmark = pytest.mark.gpu
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32

CHAIN, STAR = (lambda n: list(range(-1, n - 1))), (lambda n: [-1] + [0] * (n - 1))
# 1, 12, 24, 48 and 112 rows per KV head: 8 and 16 rows at a time, four, two copies of a row and one
ROWS = S.ROWS


def _run(c, heads, parent, q):
    from paper_2308_13137_gb300 import serve
    n = len(parent)
    tree = serve.draft_tree(torch.tensor([parent], dtype=I32, device="cuda"))
    lse = torch.empty(n, heads, device="cuda")
    out = serve.kv_attention(c, q, heads, tree=tree, out_dtype=F32, lse=lse)
    c.check()
    O, L, top = D.attention(c, q, heads, [(0, n)], [D.ancestors(parent)])
    return out.double().view(O.shape), lse.double(), O, L, top


def _check(c, heads, parent, q):
    """As for the causal form: weights in fp16 (2^-11 relative each), all else fp32; the log-sum-exp is a score of four
    roundings, a logarithm of a sum, and, where a page's factor is in the exponent, two roundings of 2^-19."""
    out, lse, O, L, top = _run(c, heads, parent, q)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    assert bool(((out - O).abs() <= 1.5 * 2.0 ** -11 * top[..., None]).all())
    assert bool(((lse - L).abs() <= 1e-5 + 8 * 2.0 ** -24 * L.abs()).all())
    return O


@pytest.mark.parametrize("heads,n", ROWS)
@pytest.mark.parametrize("kind", [CHAIN, STAR])
@pytest.mark.parametrize("page,n_pages,where", [(16, 12, 0), (16, 12, 5), (32, 9, 2), (64, 5, 1), (128, 40, 3), (16, 40, 38)])
@pytest.mark.parametrize("v_scale", [0.0, 1e-38])
def test_top_score_on_a_page_of_vanishing_values(cuda_lib, heads, n, kind, page, n_pages, where, v_scale):
    """The row's top score lies on a page whose V scale is zero (or next to it), the other pages' scores lie a
    gap below it: on both sides of every bound that the tiles' two ways have."""
    unit = 128 * math.log2(math.e) / math.sqrt(128)
    for gap in (20.0, 40.0, 63.0, 65.0, 100.0, 119.0, 121.0, 135.0, 200.0, 300.0):
        c = S._cache(n_pages, page, seed=heads + n_pages)
        q = torch.ones(n, heads * 128, device="cuda").to(BF16)
        c.k_scale.fill_(1e-3 / unit)
        c.k_scale[S._at(c, where)] = gap / unit
        c.v_scale[S._at(c, where)] = v_scale
        _check(c, heads, kind(n), q)


@pytest.mark.parametrize("heads,n", ROWS)
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("v_scale", [0.04, 4096.0])
@pytest.mark.parametrize("size", [2.0 ** 24, -2.0 ** 24, -2.0 ** 99, -2.0 ** 110, 2.0 ** 99, 2.0 ** 110])
def test_scores_of_any_size(cuda_lib, heads, n, page, v_scale, size):
    """Scores of one sign and any size below the largest fp32 number, no visible score near zero: the row is
    not empty.  Keys differ between tokens by whole codes, so scores that are not equal are far apart."""
    c = S._cache(20, page, seed=heads, tail=5)
    g = torch.Generator(device="cuda").manual_seed(3)
    level = torch.randint(20, 120, c.k.shape[:3], generator=g, device="cuda")
    c.k.copy_((128 + level)[..., None].expand(c.k.shape))
    c.v_scale.fill_(v_scale)
    c.v_scale[S._at(c, 7)] = v_scale / 512
    q = torch.full((n, heads * 128), size, device="cuda").to(BF16)
    for parent in (CHAIN(n), STAR(n)):
        O = _check(c, heads, parent, q)
        assert float(O.abs().max()) > 0
    # and beside ordinary scores: half of the pages have keys next to zero
    c.k_scale[: 10] = 2.0 ** -100
    _check(c, heads, CHAIN(n), q)


@pytest.mark.parametrize("heads,n", ROWS)
@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("low", [-20, -50, -75, -90, -100, -120])
def test_log_sum_exp_beside_vanishing_values(cuda_lib, heads, n, page, low):
    """Half of the pages have scores of 35 to 61 (in bits) and values of the order 2^low, the others 2 less and ordinary values.
    The value scales are no part of the log-sum-exp: it holds to the roundings of its own size, however far the scales lie apart.

    Scores are whole numbers times a power of two and the constant log2(e) / sqrt(128), which lies within 1e-8 of its
    value in fp32 (9.1e-9, relative).  Roundings of 2^-19 (numbers from 32 to 64): a score, the log-sum-exp of a part of the tokens,
    and of the row; where a page's factor is in the exponent, that factor less the reference, and the exponent.  The logarithm, the
    exponentials and the sums: 2^-20."""
    worst = 0.0
    for i, code in enumerate((80, 108, 110, 112, 80, 71, 97, 119) * 3):
        c = S._cache(10, page, seed=i, tail=3)
        c.k_scale.fill_(2.0 ** -5)
        c.v_scale.fill_(1.0)
        for p in range(0, 10, 2):
            c.k[S._at(c, p)] = 128 + code
            c.k[S._at(c, p + 1)] = 128 + code - 4
            c.v_scale[S._at(c, p)] = 2.0 ** low * (1 + i / 24)
        q = torch.ones(n, heads * 128, device="cuda").to(BF16)
        _, lse, _, L, _ = _run(c, heads, STAR(n), q)
        worst = max(worst, float((lse - L).abs().max()))
    together = abs(low) < 50                  # the factor of a page, low + 10, and that less the reference lie below 64
    assert worst <= (5 if together else 3) * 2.0 ** -19 + 2.0 ** -20 + 1e-8 * 64, worst


@pytest.mark.parametrize("drawn", [True, False])
def test_the_token_after_an_accepted_draft_is_distributed_as_its_row(cuda_lib, drawn):
    """60000 sequences over 6 tokens: enough of them accept the first draft, and the next token has the frequencies of that
    draft's row; a count of n draws strays by sqrt(n p (1 - p)), five of these are allowed.  Chosen drafts: the first one is accepted
    with the target's probability."""
    from paper_2308_13137_gb300 import serve
    from test_serve_drafts_gpu import _dev, _dists
    B, V, n = 60000, 6, 6
    parent = [-1, 0, 0, 0, 1, 1]
    P1, Q1 = _dists(n, V, 11, spread=1.0, apart=1.0)
    g = torch.Generator(device="cuda").manual_seed(9)
    if drawn:
        up = _dev([0, 0, 0, 0, 1, 1], torch.int64)
        tok = torch.multinomial(Q1[up].repeat(B, 1), 1, generator=g)[:, 0].to(I32)
    else:
        tok = _dev([0, int(P1[0].argmax()), 1, 2, 0, 5]).repeat(B)
    got = serve.verify_drafts(serve.draft_tree(_dev(parent).repeat(B).view(B, n)), tok, P1.repeat(B, 1),
                              torch.rand(B * n, generator=g, device="cuda"), draft_probs=Q1.repeat(B, 1) if drawn else None, steps=3)
    took = (got.count >= 2) & (got.path[:, 1] == 1)
    p, q = P1[0].double(), Q1[0].double()
    chance = float(torch.minimum(p, q).sum()) if drawn else float(p.max())
    assert abs(int(took.sum()) - B * chance) <= 5 * math.sqrt(B * chance * (1 - chance)) + 1
    rows = got.tokens[:, 1][took]
    assert rows.numel() >= 1000
    count, p, m = torch.bincount(rows.long(), minlength=V).double(), P1[1].double(), rows.numel()
    assert bool(((count - m * p).abs() <= 5 * (m * p * (1 - p)).sqrt() + 1).all())
