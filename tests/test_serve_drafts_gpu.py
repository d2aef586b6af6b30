"""Drafted tokens over the 8-bit cache: trees, the append at their positions, attention along their branches, verification
against the target's probabilities, and the accepted path in the cache; each against its plain form."""
import math

import numpy as np
import pytest
import torch

import _drafts_ref as D
import _serve_ref as REF
from test_serve_cache_gpu import _cache, _cu

pytestmark = pytest.mark.gpu
F32, BF16, F64, U8, I32 = torch.float32, torch.bfloat16, torch.float64, torch.uint8, torch.int32


def _dev(a, dt=I32):
    return torch.as_tensor(np.asarray(a)).to("cuda", dt)


def _trees(n_q, seed, **kw):
    r = np.random.RandomState(seed)
    return [D.random_tree(n, r, **kw) if n else [] for n in n_q]


def _tree(parents, **kw):
    """serve.draft_tree of a list of parents per sequence."""
    from paper_2308_13137_gb300 import serve
    n_q = [len(p) for p in parents]
    return serve.draft_tree(_dev(sum(parents, [])), _cu(n_q), max(n_q), **kw)


# ------------------------------------------------------------------------------------------------
# trees
# ------------------------------------------------------------------------------------------------

CHAIN, STAR = (lambda n: list(range(-1, n - 1))), (lambda n: [-1] + [0] * (n - 1))


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 65, 509, 1024])
@pytest.mark.parametrize("kind", ["chain", "star", "random", "forest"])
def test_tree(cuda_lib, n, kind):
    parent = {"chain": CHAIN, "star": STAR, "forest": lambda n: [-1 if i % 3 == 0 else i - 1 for i in range(n)],
              "random": lambda n: D.random_tree(n, np.random.RandomState(n), depth=40, width=3)}[kind](n)
    t = _tree([parent, [], parent[:n // 2], [-1]])
    want = [D.ancestors(p) for p in (parent, parent[:n // 2], [-1])]
    assert t.depth.tolist() == sum(((m.sum(1) - 1).tolist() for m in want), [])
    assert np.array_equal(t.seen.cpu().numpy(), np.concatenate([D.words_of(m, t.seen.shape[1]) for m in want]))


def test_tree_of_equal_rows_and_wide_words(cuda_lib):
    """[B, n] parents without cu_q; words beyond the needed ones are zero; buffers are filled in place."""
    from paper_2308_13137_gb300 import serve
    parent = _dev([CHAIN(5), STAR(5), [-1, 0, 0, 1, 1]])
    out = serve.DraftTree(parent.view(-1), torch.full((15,), 7, dtype=I32, device="cuda"),
                          torch.full((15, 3), 7, dtype=I32, device="cuda"), None, 5)
    t = serve.draft_tree(parent, out=out)
    assert t is out and t.depth.tolist() == [0, 1, 2, 3, 4, 0, 1, 1, 1, 1, 0, 1, 1, 2, 2]
    assert t.seen[:, 0].tolist() == [1, 3, 7, 15, 31, 1, 3, 5, 9, 17, 1, 3, 5, 11, 19] and not t.seen[:, 1:].any()


def test_tree_bad_parents_and_rows(cuda_lib):
    """A parent that is not before its child is reported and the row counts as a root; sequences whose bounds are out of
    range are left out, and rows behind the last sequence stay as they were."""
    from paper_2308_13137_gb300 import _lib, serve
    status = torch.zeros(1, dtype=I32, device="cuda")
    t = serve.draft_tree(_dev([-1, 1, 0, 7, -2, 2]), _cu([6]), 6, status=status)
    assert int(status) == 1
    assert t.depth.tolist() == [0, 0, 1, 0, 0, 2] and t.seen[:, 0].tolist() == [1, 2, 5, 8, 16, 37]
    status.zero_()
    out = serve.DraftTree(None, torch.full((9,), -5, dtype=I32, device="cuda"), torch.full((9, 1), -5, dtype=I32, device="cuda"), None, 3)
    serve.draft_tree(_dev([-1, 0, 1] * 3), _dev([0, 3, 7, 6, 3]), 3, out=out, status=status)      # 4 rows, -1 rows, -3
    assert int(status) == 1 and out.depth.tolist() == [0, 1, 2] + [-5] * 6 and out.seen[:, 0].tolist() == [1, 3, 7] + [-5] * 6
    before = _lib.omq_launch_count()
    for bad in (lambda: serve.draft_tree(_dev([[-1] * 1025])), lambda: serve.draft_tree(torch.zeros(0, 4, dtype=I32, device="cuda")),
                lambda: serve.draft_tree(_dev([-1, 0]), _cu([2]), 0), lambda: serve.draft_tree(_dev([-1, 0]), _cu([2]), 3)):
        with pytest.raises((ValueError, _lib.OmqError)):
            bad()
    assert _lib.omq_launch_count() == before


# ------------------------------------------------------------------------------------------------
# append
# ------------------------------------------------------------------------------------------------

def _pair(lens, n_kv, page, seed):
    return _cache(lens, n_kv, page, seed=seed), _cache(lens, n_kv, page, seed=seed)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_append_of_chains_is_the_plain_append(cuda_lib, page, dt):
    """Depth i at row i: bit for bit what kv_append writes and returns."""
    from paper_2308_13137_gb300 import serve
    lens, n_q, heads, n_kv = [40, 7, 130, 16, 200], [7, 7, 1, 0, 150], 6, 2
    a, b = _pair(lens, n_kv, page, 3)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(sum(n_q), (heads + 2 * n_kv) * 128, generator=g, device="cuda").to(dt)
    sa = torch.exp(0.2 * torch.randn(n_kv * 128, generator=g, device="cuda"))
    rope = serve.rope_table(300)
    outs = []
    for c, kw in ((a, dict(cu_q=_cu(n_q), max_q=150)), (b, dict(tree=_tree([CHAIN(n) if n else [] for n in n_q])))):
        k, v = (torch.empty(sum(n_q), n_kv * 128, dtype=BF16, device="cuda") for _ in range(2))
        outs.append((serve.kv_append(c, x, rope, heads, sa=sa, k_out=k, v_out=v, **kw), k, v, c.k, c.v, c.k_scale, c.v_scale))
        c.check()
    for t, w in zip(*outs):
        assert torch.equal(t.view(torch.uint8), w.view(torch.uint8))


@pytest.mark.parametrize("page", [16, 64])
def test_append_at_depths(cuda_lib, page):
    """q of every row is bit for bit what a sequence of one row at that position gets; k within half a step of its
    page's scale (and fp32 rounding) of the turned k in double, v as without a tree."""
    from paper_2308_13137_gb300 import serve
    n_q, start, heads, n_kv = [13, 1, 40, 5], [30, 0, 101, 15], 4, 2
    lens = [s + n for s, n in zip(start, n_q)]
    parents = _trees(n_q, 5)
    tree = _tree(parents)
    c = _cache(lens, n_kv, page, seed=2)
    rows = sum(n_q)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(rows, (heads + 2 * n_kv) * 128, generator=g, device="cuda")
    sa = torch.exp(0.2 * torch.randn(n_kv * 128, generator=g, device="cuda"))
    rope = serve.rope_table(256)
    k, v = (torch.empty(rows, n_kv * 128, dtype=BF16, device="cuda") for _ in range(2))
    q = serve.kv_append(c, x, rope, heads, sa=sa, k_out=k, v_out=v, tree=tree)
    c.check()
    pos = torch.repeat_interleave(_dev(start, torch.int64), _dev(n_q, torch.int64)) + tree.depth
    one = serve.KVCache.empty(rows * 16, n_kv, 16, rows, 16)
    one.table.copy_(torch.arange(rows * 16, dtype=I32).view(rows, 16))
    one.kv_len.copy_(pos + 1)
    assert torch.equal(q, serve.kv_append(one, x, rope, heads, sa=sa))
    one.check()
    want = REF.turned(x.double()[:, heads * 128:(heads + n_kv) * 128].view(rows, n_kv, 128), rope, pos) * sa.double().view(n_kv, 128)
    cu = _cu(n_q).tolist()
    for b in range(4):
        got = REF.dequant(c, "k", b, lens[b])[start[b]:]
        sc = c.k_scale[c.table[b].long().clamp_min(0)][torch.arange(start[b], lens[b], device="cuda") // page].double()[..., None]
        ref = want[cu[b]:cu[b + 1]]
        # four fp32 roundings before the code, one of the quotient: 2^-21 of the largest magnitude is ample
        assert bool(((got - ref).abs() <= 0.5 * sc + 2.0 ** -21 * ref.abs().max()).all())


def test_append_bad_depths(cuda_lib):
    """A depth outside the table is reported; the row is turned to its root's position."""
    from paper_2308_13137_gb300 import serve
    rope = serve.rope_table(20)
    c = _cache([20], 1, 16, seed=1)
    x = torch.randn(4, 3 * 128, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    tree = serve.DraftTree(_dev([-1, 0, 1, 2]), _dev([0, 3, 4, -1]), _dev([[1], [3], [7], [15]]), _cu([4]), 4)
    q = serve.kv_append(c, x, rope, 1, tree=tree)
    assert int(c.status) == 1
    c.status.zero_()
    good = serve.kv_append(c, x, rope, 1, tree=tree._replace(depth=_dev([0, 3, 0, 0])))
    c.check()
    assert torch.equal(q, good)


# ------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------

def _seen_tree(masks, n_q, words=None):
    """A DraftTree with given visible rows (no parents)."""
    from paper_2308_13137_gb300 import serve
    words = words or (max(n_q) + 31) // 32
    bits = [D.words_of(m, words) for m in masks if len(m)]
    z = torch.zeros(sum(n_q), dtype=I32, device="cuda")
    return serve.DraftTree(z, z, _dev(np.concatenate(bits)), _cu(n_q), max(n_q))


def _attend(c, n_q, heads, masks, seed=1, q=None, tree=None, out_dtype=F32, **kw):
    from paper_2308_13137_gb300 import serve
    if q is None:
        q = (torch.randn(sum(n_q), heads * 128, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * 1.5).to(BF16)
    lse = torch.full((sum(n_q), heads), 7.0, device="cuda")
    out = serve.kv_attention(c, q, heads, tree=tree or _seen_tree(masks, n_q), lse=lse, out_dtype=out_dtype, **kw)
    c.check()
    return q, out, lse


def _check(c, n_q, heads, masks, q, out, lse):
    """Weights in fp16 (2^-11 relative each), all else fp32: within 2^-11 of the largest |v| that the row sees,
    half as much again for the fp32 parts."""
    cu = _cu(n_q).tolist()
    O, L, top = D.attention(c, q, heads, [(cu[b], n) for b, n in enumerate(n_q)], masks)
    got = out.double().view(O.shape)
    slack = 0 if out.dtype == F32 else 2.0 ** -8 * O.abs()
    assert bool(((got - O).abs() <= 1.5 * 2.0 ** -11 * top[..., None] + slack).all()), \
        float(((got - O).abs() / top[..., None].clamp_min(1e-30)).max())
    empty = torch.isinf(L)
    assert torch.equal(torch.isinf(lse), empty) and bool((got[empty] == 0).all())
    assert bool(((lse.double() - L)[~empty].abs() <= 1e-4).all())


LAYOUTS = [(1, 1), (4, 4), (8, 1), (6, 2), (16, 2)]


@pytest.mark.parametrize("heads,n_kv", LAYOUTS)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_trees_over_contexts_of_every_kind(cuda_lib, heads, n_kv, page):
    """Trees that start at a page's and a tile's edges, alone in the cache, and over several pages."""
    start = [0, 1, 15, 16, 17, page - 1, page, page + 1, 63, 64, 100, 700]
    for n in (1, 2, 5, 9, 16):
        n_q = [n] * len(start)
        parents = _trees(n_q, n + page)
        c = _cache([s + n for s in start], n_kv, page, seed=heads + page + n)
        masks = [D.ancestors(p) for p in parents]
        _check(c, n_q, heads, masks, *_attend(c, n_q, heads, masks, tree=_tree(parents)))


@pytest.mark.parametrize("heads,n_kv", LAYOUTS)
@pytest.mark.parametrize("n_q", [[2, 5, 1, 3], [17, 0, 33, 9], [64, 40, 7, 65], [130, 1, 200, 12]])
def test_ragged_trees(cuda_lib, heads, n_kv, n_q):
    """Rows of unequal number, none at all, and sequences with fewer tokens than rows."""
    lens = [n_q[0] + 301, max(0, n_q[1] - 3), n_q[2] + 70, n_q[3]]
    parents = _trees(n_q, sum(n_q) + heads, depth=9)
    masks = [D.ancestors(p) if p else np.zeros((0, 0), bool) for p in parents]
    c = _cache(lens, n_kv, 32, seed=heads + sum(n_q))
    _check(c, n_q, heads, masks, *_attend(c, n_q, heads, masks, tree=_tree(parents)))


@pytest.mark.parametrize("heads,n_kv,n", [(2, 2, 12), (8, 1, 7), (4, 1, 40), (2, 1, 300)])
def test_any_bits(cuda_lib, heads, n_kv, n):
    """Bits that are no tree's: rows that see later ones, not themselves, nothing at all; bits beyond the sequence's rows
    are set and count for nothing, and there are more words than are needed."""
    r = np.random.RandomState(n)
    start, n_q = [0, 37, 0, 500], [n, n, max(1, n // 2), n]
    masks = [r.rand(k, k) < 0.3 for k in n_q]
    masks[0][::3] = False                                      # no context: these rows are empty
    masks[2][:] = False
    masks[1][1] = False                                        # only the context
    words = (n + 31) // 32 + 2
    tree = _seen_tree(masks, n_q, words)
    at = 0
    bits = tree.seen.cpu().numpy().view(np.uint32).reshape(-1, words).copy()
    for k in n_q:
        for w in range(words):
            for j in range(32):
                if w * 32 + j >= k:
                    bits[at:at + k, w] |= np.uint32(1 << j)
        at += k
    tree = tree._replace(seen=_dev(bits.view(np.int32)))
    c = _cache([s + k for s, k in zip(start, n_q)], n_kv, 16, seed=n)
    _check(c, n_q, heads, masks, *_attend(c, n_q, heads, masks, tree=tree))
    _check(c, n_q, heads, masks, *_attend(c, n_q, heads, masks, tree=tree, out_dtype=BF16))


@pytest.mark.parametrize("heads,n_kv,n", [(8, 8, 1), (8, 1, 2), (8, 1, 5), (4, 2, 20), (8, 1, 64), (2, 2, 70)])
def test_long_contexts(cuda_lib, heads, n_kv, n):
    """One long sequence among short ones: the work is split, and shared out among unequal sequences."""
    lens = [20011 + n, n, 130 + n, 0, 3000 + n]
    parents = _trees([n] * 5, n)
    masks = [D.ancestors(p) for p in parents]
    c = _cache(lens, n_kv, 64, seed=5)
    q, out, lse = _attend(c, [n] * 5, heads, masks, tree=_tree(parents))
    _check(c, [n] * 5, heads, masks, q, out, lse)
    _, again, lse2 = _attend(c, [n] * 5, heads, masks, q=q, tree=_tree(parents), max_kv=20011 + n)      # another bound
    _check(c, [n] * 5, heads, masks, q, again, lse2)


@pytest.mark.parametrize("B,heads,n_kv,n", [(70, 2, 1, 3), (300, 2, 2, 1), (40, 16, 2, 9), (20, 8, 8, 30), (700, 1, 1, 20)])
def test_many_sequences(cuda_lib, B, heads, n_kv, n):
    """More sequences than SMs, lengths from nothing to a few hundred."""
    r = np.random.RandomState(B)
    n_q = [int(r.randint(0, n + 1)) for _ in range(B)]
    n_q[3] = n
    lens = [int(k + r.randint(0, 400)) if r.rand() < 0.9 else int(r.randint(0, k + 1)) for k in n_q]
    parents = _trees(n_q, B)
    masks = [D.ancestors(p) if p else np.zeros((0, 0), bool) for p in parents]
    c = _cache(lens, n_kv, 16, seed=B)
    _check(c, n_q, heads, masks, *_attend(c, n_q, heads, masks, tree=_tree(parents)))


@pytest.mark.parametrize("heads,n", [(2, 3), (8, 6), (16, 5), (16, 20)])
@pytest.mark.parametrize("page", [16, 64])
def test_pages_that_a_row_does_not_see(cuda_lib, heads, n, page):
    """Scales that are not finite on the page of the newest row: only the rows that see it may show it."""
    c = _cache([3 * page + 1, 9 * page + 1], 1, page, seed=heads + n + page)
    masks = [D.ancestors(STAR(n))] * 2
    q, out, lse = _attend(c, [n] * 2, heads, masks)
    _check(c, [n] * 2, heads, masks, q, out, lse)
    last = c.table.long()[[0, 1], [3, 9]]
    for value in (float("inf"), float("nan")):
        for t in (c.k_scale, c.v_scale):
            old = t[last].clone()
            t[last] = value
            _, got, l2 = _attend(c, [n] * 2, heads, masks, q=q)
            t[last] = old
            hold = [i for i in range(2 * n) if i % n != n - 1]
            assert bool(torch.isfinite(got[hold]).all()) and bool(torch.isfinite(l2[hold]).all())
            assert torch.allclose(got[hold], out[hold], rtol=0, atol=float(3 * 2.0 ** -11 * 127 * c.v_scale[torch.isfinite(c.v_scale)].max()))


def test_scales_far_apart(cuda_lib):
    """Contexts on pages of zero, tiny and huge value scales, and keys that make one page's scores huge."""
    for heads, n in ((2, 4), (8, 8)):
        c = _cache([600 + n, 600 + n], 1, 16, seed=9)
        t = c.table.long()
        c.v_scale[t[0, :16]] *= 2.0 ** -20
        c.k_scale[t[0, 16:32]] *= 1e-3
        c.v_scale[t[1, 3:20]] = 0
        c.k_scale[t[1, 8:9]] = 0
        c.k_scale[t[1, 22]] *= 40
        masks = [D.ancestors(p) for p in _trees([n, n], 3)]
        _check(c, [n, n], heads, masks, *_attend(c, [n, n], heads, masks))


def test_strided_rows_and_chains(cuda_lib):
    """Row strides of q and out; a chain gives what kv_attention gives, up to the weights' rounding."""
    from paper_2308_13137_gb300 import serve
    heads, n = 4, 6
    c = _cache([200, 6, 90], 2, 32, seed=4)
    wide = torch.randn(18, 3 * heads * 128, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(BF16)
    q, out = wide[:, 512:1024], torch.full((18, 2 * heads * 128), 3.0, device="cuda")
    tree = serve.draft_tree(_dev([CHAIN(n)] * 3))
    got = serve.kv_attention(c, q, heads, tree=tree, out=out[:, :512])
    want = serve.kv_attention(c, q, heads, out_dtype=F32)
    c.check()
    assert got.data_ptr() == out.data_ptr() and bool((out[:, 512:] == 3.0).all())
    masks = [D.ancestors(CHAIN(n))] * 3
    O, L, top = D.attention(c, q, heads, [(0, 6), (6, 6), (12, 6)], masks)
    assert bool(((got - want).double().view(O.shape).abs() <= 3 * 2.0 ** -11 * top[..., None]).all())


def test_bad_pages_and_lengths(cuda_lib):
    """Page ids out of range and lengths beyond the bound are reported; the other sequences are as they were."""
    from paper_2308_13137_gb300 import _lib, serve
    for heads, n in ((2, 3), (8, 9)):
        lens = [90, 200, 40]
        c = _cache(lens, 1, 16, seed=6)
        parents = _trees([n] * 3, 1)
        masks, tree = [D.ancestors(p) for p in parents], _tree(parents)
        q, out, lse = _attend(c, [n] * 3, heads, masks, tree=tree)
        c.table[1, 2] = 1 << 20
        _, lse2 = None, torch.empty_like(lse)
        got = serve.kv_attention(c, q, heads, tree=tree, lse=lse2, out_dtype=F32)
        with pytest.raises(_lib.OmqError):
            c.check()
        keep = list(range(n)) + list(range(2 * n, 3 * n))
        tol = float(3 * 2.0 ** -11 * 127 * c.v_scale[torch.isfinite(c.v_scale)].max())
        assert torch.allclose(got[keep], out[keep], rtol=0, atol=tol) and bool(torch.isfinite(got).all())
        got = serve.kv_attention(c, q, heads, tree=tree, max_kv=100, out_dtype=F32)     # sequence 1 is longer
        with pytest.raises(_lib.OmqError):
            c.check()
        assert torch.allclose(got[keep], out[keep], rtol=0, atol=tol) and bool((got[n:2 * n] == 0).all())


# ------------------------------------------------------------------------------------------------
# verification
# ------------------------------------------------------------------------------------------------

def _dists(rows, V, seed, spread=2.0, apart=0.7, dt=F32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = spread * torch.randn(rows, V, generator=g, device="cuda")
    q = torch.softmax(z + apart * torch.randn(rows, V, generator=g, device="cuda"), -1)
    return torch.softmax(z, -1).to(dt), q.to(dt)


def _draw(parents, Q, seed, chosen=False):
    """Drafted tokens: from the parent's row of Q, or its likeliest (with a repetition here and there)."""
    r = np.random.RandomState(seed)
    tokens, at = [], 0
    for p in parents:
        kids = {}
        for i, up in enumerate(p):
            if up < 0:
                tokens.append(0)
                continue
            row = Q[at + up].double()
            if chosen:
                k = kids[up] = kids.get(up, -1) + 1
                top = torch.topk(row, min(len(row), k + 1)).indices
                tokens.append(int(top[-1 if r.rand() < 0.9 else 0]))
            else:
                c = (row / row.sum()).cumsum(0)
                tokens.append(min(int((c <= r.rand()).sum()), len(row) - 1))
        at += len(p)
    return tokens


def _verify(parents, tokens, P, Q, u, steps=None, **kw):
    """Runs the operator and the 64-bit walk and compares them exactly."""
    from paper_2308_13137_gb300 import serve
    tree = _tree(parents)
    status = torch.zeros(1, dtype=I32, device="cuda")
    got = serve.verify_drafts(tree, _dev(tokens), P, u, draft_probs=Q, steps=steps, status=status, **kw)
    steps, at, num = got.path.shape[1], 0, u.double().tolist()
    for b, p in enumerate(parents):
        if not p:
            assert int(got.count[b]) == 0 and bool((got.path[b] == -1).all()) and bool((got.tokens[b] == -1).all())
            continue
        rows = slice(at, at + len(p))
        at += len(p)
        path, out = D.verify(p, tokens[rows], P[rows], None if Q is None else Q[rows], num[rows], steps)
        assert int(got.count[b]) == len(path)
        assert got.path[b].tolist() == path + [-1] * (steps - len(path)), b
        assert got.tokens[b].tolist() == out + [-1] * (steps - len(out)), b
    return got, status


def _uniform(n, seed):
    return torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("V", [1, 2, 5, 127, 128, 129, 1000, 4096, 4097, 8192, 32000, 50001])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_verify(cuda_lib, V, drawn, dt):
    n_q = [1, 2, 13, 0, 40, 9, 26]
    parents = _trees(n_q, V)
    P, Q = _dists(sum(n_q), V, V + 1, dt=dt)
    for seed in range(4):
        tokens = _draw(parents, Q, seed, chosen=not drawn)
        _, st = _verify(parents, tokens, P, Q if drawn else None, _uniform(sum(n_q), seed))
        assert int(st) == 0


@pytest.mark.parametrize("drawn", [True, False])
def test_many_rejections(cuda_lib, drawn):
    """Wide nodes whose children mostly fail: distributions far apart, numbers near one."""
    parents = [STAR(200), [-1] + [0] * 30 + [5] * 30 + [40] * 10, CHAIN(20)] * 4
    n = sum(len(p) for p in parents)
    P, Q = _dists(n, 3000, 5, spread=1.0, apart=3.0)
    for seed, lo in ((0, 0.9), (1, 0.0), (2, 0.999)):
        _verify(parents, _draw(parents, Q, seed, chosen=not drawn), P, Q if drawn else None, lo + (1 - lo) * _uniform(n, seed))


def test_a_thousand_children(cuda_lib):
    parents = [STAR(1024), CHAIN(1024)]
    P, Q = _dists(2048, 600, 6, spread=1.0, apart=3.0)
    tokens = _draw(parents, Q, 1)
    u = 0.97 + 0.03 * _uniform(2048, 2)
    _verify(parents, tokens, P, Q, u, steps=40)
    _verify(parents, tokens, P, None, u, steps=40)
    _verify(parents, tokens, Q, Q, u * 0.9, steps=1024)             # the same distribution: the whole chain is accepted


def test_steps(cuda_lib):
    """The path ends at its last column; what it has there is not tested further, and the new token comes from its row."""
    parents = [CHAIN(9), D.random_tree(30, np.random.RandomState(1)), [-1]]
    P, Q = _dists(40, 500, 3, apart=0.05)
    tokens = _draw(parents, Q, 3)
    for steps in (1, 2, 3, 8, 9, 12):
        for q in (Q, None):
            got, st = _verify(parents, tokens, P, q, _uniform(40, steps) * 0.5, steps=steps)
            assert int(st) == 0 and int(got.count.max()) <= steps


def test_verify_rows_of_any_stride(cuda_lib):
    """Rows within wider ones, an odd vocabulary, a base that is not aligned to a vector, P and Q of unequal stride."""
    parents = _trees([12, 12], 8)
    for V, dt in ((777, F32), (6001, F32), (6001, BF16), (8200, BF16)):
        P, Q = _dists(24, V, V, dt=dt)
        wide = torch.full((24, V + 37), float("nan"), dtype=dt, device="cuda")
        wide[:, 5:5 + V] = P
        other = torch.full((24, 2 * V + 3), float("nan"), dtype=dt, device="cuda")
        other[:, V:2 * V] = Q
        tokens = _draw(parents, Q, 2)
        for seed in range(3):
            u = _uniform(24, seed)
            a, _ = _verify(parents, tokens, wide[:, 5:5 + V], other[:, V:2 * V], u)
            b, _ = _verify(parents, tokens, P, Q, u)
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_verify_at_the_borders(cuda_lib):
    """Numbers of zero and one below one, equal distributions, tokens that the target or the draft cannot give, weight on
    one token only, and the sum's border hit exactly."""
    V = 8
    eye = torch.eye(V, device="cuda")
    half = torch.zeros(1, V, device="cuda")
    half[0, 2] = half[0, 5] = 0.5
    parents = [[-1, 0, 0]]
    last = 1 - 2.0 ** -24
    for P, Q, tokens, u, path, out in (
            (half, half, [0, 2, 5], [0.0, last, 0.5], [0, 1], [2, 2]),          # equal: accepted at any number; then half again
            (half, half, [0, 2, 5], [0.5, last, 0.5], [0, 1], [2, 5]),          # running sum 0.5 does not pass 0.5: the next
            (half, eye[3:4], [0, 3, 5], [0.0, 0.0, 0.0], [0, 2], [5, 2]),       # 0 < 0 is false; then q(5) = 0 < the rest
            (half, None, [0, 2, 5], [0.0, 0.5, 0.3], [0, 2], [5, 2]),           # 0.5 < 0.5 is false; 0.3 0.5 < 0.5
            (half, None, [0, 2, 2], [0.0, 0.5, 0.0], [0], [5]),                 # the same token again weighs nothing
            (half, None, [0, 1, 7], [last, 0.0, 0.0], [0], [5]),                # what the target cannot give
            (eye[4:5], None, [0, 4, 4], [0.3, last, 0.0], [0, 1], [4, 4]),
            (eye[4:5], eye[1:2], [0, 1, 1], [last, 0.0, 0.0], [0], [4])):
        Pr = P.expand(3, V).contiguous()
        Qr = Q.expand(3, V).contiguous() if Q is not None else None
        got, _ = _verify(parents, tokens, Pr, Qr, torch.tensor(u, device="cuda"))
        assert got.path[0, :len(path)].tolist() == path and got.tokens[0, :len(out)].tolist() == out


def test_verify_odd_numbers(cuda_lib):
    """NaN, infinite and negative probabilities count as zero or one, numbers outside [0, 1) as the nearest; a row without
    weight is reported and gives token 0."""
    from paper_2308_13137_gb300 import serve
    parents = _trees([10, 10, 10], 4)
    P, Q = _dists(30, 300, 4)
    tokens = _draw(parents, Q, 1)
    P[3, 10:40] = float("nan")
    P[::4, 77] = -1.0
    Q[::3, 5:9] = float("nan")
    u = _uniform(30, 1)
    u[0], u[4], u[11], u[20] = 1.0, float("nan"), -3.0, float("inf")
    for q in (Q, None):
        _, st = _verify(parents, tokens, P, q, u)
        assert int(st) == 0
    one = torch.zeros(2, 50, device="cuda")
    one[0, 7] = float("inf")                                       # counts as one
    st = torch.zeros(1, dtype=I32, device="cuda")
    tree = serve.draft_tree(_dev([[-1], [-1]]))
    got = serve.verify_drafts(tree, _dev([0, 0]), one, torch.full((2,), 0.9, device="cuda"), status=st)
    assert got.tokens.tolist() == [[7], [0]] and int(st) == 1


def test_verify_bad_nodes(cuda_lib):
    """Parents and tokens out of range are reported; such rows are nobody's children, the others count."""
    from paper_2308_13137_gb300 import serve
    P, Q = _dists(6, 40, 2, apart=0.01)
    st = torch.zeros(1, dtype=I32, device="cuda")
    good = ([-1, 0, 1, 2, 0, 0], [0, 3, 4, 5, 6, 7])
    for parent, token in (([-1, 0, 1, 9, 0, 0], good[1]), (good[0], [0, 3, 40, 5, 6, 7]), (good[0], [0, 3, 4, -1, 6, 7]),
                          ([-1, 0, 1, 3, 0, 0], good[1]), ([0, 0, 1, 2, 0, 0], good[1])):
        st.zero_()
        tree = serve.DraftTree(_dev(parent), _dev(parent), _dev(parent).view(-1, 1), _cu([6]), 6)
        u = torch.zeros(6, device="cuda")                          # every child that can be is accepted
        got = serve.verify_drafts(tree, _dev(token), P, u, status=st)
        fixed = [p if 0 <= p < i and 0 <= token[i] < 40 else -1 for i, p in enumerate(parent)]
        path, out = D.verify(fixed, token, P, None, [0.0] * 6, 6)
        assert int(st) == 1 and got.path[0, :len(path)].tolist() == path and got.tokens[0, :len(out)].tolist() == out
    # sequences whose bounds are out of range: nothing accepted, the others as ever
    st.zero_()
    tree = serve.DraftTree(_dev([-1, 0, 1, -1, 0, 1]), None, None, _dev([0, 3, 2, 6]), 4)
    got = serve.verify_drafts(tree, _dev(good[1]), P, torch.zeros(6, device="cuda"), status=st)
    assert int(st) == 1 and got.count.tolist()[1] == 0 and got.path[1].tolist() == [-1] * 4
    assert int(got.count[0]) == len(D.verify([-1, 0, 1], [0, 3, 4], P[:3], None, [0.0] * 3, 4)[0])


@pytest.mark.parametrize("drawn", [True, False])
def test_what_comes_out_is_distributed_as_the_target(cuda_lib, drawn):
    """60000 sequences of one distribution each over 6 tokens, three drafts at the root and two below the first: the first
    emitted token has the target's frequencies, and the second, where the first draft was accepted, those of its row.  A
    count of n draws strays by sqrt(n p (1 - p)); five of these are allowed."""
    from paper_2308_13137_gb300 import serve
    B, V, n = 60000, 6, 6
    parent = [-1, 0, 0, 0, 1, 1]
    P1, Q1 = _dists(n, V, 11, spread=1.0, apart=1.0)
    g = torch.Generator(device="cuda").manual_seed(9)
    P, Q = P1.repeat(B, 1), Q1.repeat(B, 1)
    if drawn:
        up = _dev([0, 0, 0, 0, 1, 1], torch.int64)
        tok = torch.multinomial(Q1[up].repeat(B, 1), 1, generator=g)[:, 0].to(I32)
    else:
        tok = _dev([0, 4, 1, 2, 0, 5]).repeat(B)
    got = serve.verify_drafts(serve.draft_tree(_dev(parent).repeat(B).view(B, n)), tok, P, torch.rand(B * n, generator=g, device="cuda"),
                              draft_probs=Q if drawn else None, steps=3)
    for rows, p in ((got.tokens[:, 0], P1[0]), (got.tokens[:, 1][(got.count >= 2) & (got.path[:, 1] == 1)], P1[1])):
        if rows.numel() < 1000:
            continue
        count, p, m = torch.bincount(rows.long(), minlength=V).double(), p.double(), rows.numel()
        assert bool(((count - m * p).abs() <= 5 * (m * p * (1 - p)).sqrt() + 1).all())


# ------------------------------------------------------------------------------------------------
# the accepted path in the cache
# ------------------------------------------------------------------------------------------------

def _paths(n_q, seed, steps):
    r = np.random.RandomState(seed)
    out = []
    for n in n_q:
        k = int(r.randint(0, min(n, steps) + 1))
        out.append(sorted(r.choice(n, k, replace=False).tolist()))
    return out


def _path_tensors(paths, steps):
    p = np.full((len(paths), steps), -1, np.int32)
    for b, x in enumerate(paths):
        p[b, :len(x)] = x
    return _dev(p), _dev([len(x) for x in paths])


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n_kv", [1, 8])
@pytest.mark.parametrize("n", [1, 5, 40, 300])
def test_keep(cuda_lib, page, n_kv, n):
    """Codes and scales are those of the stated order of roundings, bit for bit; nothing else changes."""
    from paper_2308_13137_gb300 import serve
    r = np.random.RandomState(n)
    n_q = [n, max(1, n // 2), n, n, 0, n]
    lens = [k + int(s) for k, s in zip(n_q, [0, 1, page - 1, page, 3, r.randint(0, 200)])]
    steps = min(n, 150)
    paths = _paths(n_q, n + page, steps)
    paths[0] = list(range(min(n, steps)))                     # all in place
    a, b = _pair(lens, n_kv, page, n + page)
    for t in (a, b):
        t.k_scale[t.k_scale > 0] *= 1
    path, count = _path_tensors(paths, steps)
    tree = serve.DraftTree(torch.zeros(sum(n_q), dtype=I32, device="cuda"), None, None, _cu(n_q), max(n_q))
    serve.kv_keep(a, tree, path, count)
    a.check()
    for s, p in enumerate(paths):
        if p:
            D.keep(b, lens[s] - n_q[s], p, s)
    for x, y in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_kept_values(cuda_lib):
    """The kept tokens' values, in double: half a step of the new scale off at most, another half where a page's codes
    were rounded again."""
    from paper_2308_13137_gb300 import serve
    n_q, lens, steps = [50, 50], [61, 50], 12
    for page in (16, 64):
        c = _cache(lens, 2, page, seed=page)
        paths = [[0, 3, 17, 40, 49], [0, 1, 2, 20, 30, 31, 45]]
        old = [(REF.dequant(c, "k", b, lens[b]), REF.dequant(c, "v", b, lens[b])) for b in range(2)]
        path, count = _path_tensors(paths, steps)
        serve.kv_keep([c], serve.DraftTree(torch.zeros(100, dtype=I32, device="cuda"), None, None, None, 50), path, count)
        c.check()
        for b in range(2):
            s = lens[b] - n_q[b]
            for name, was in zip("kv", old[b]):
                now = REF.dequant(c, name, b, lens[b])
                idx = list(range(s)) + [s + p for p in paths[b]]
                top = getattr(c, name + "_scale")[c.table[b].long().clamp_min(0)][torch.arange(len(idx), device="cuda") // page].double()[..., None]
                assert bool(((now[:len(idx)] - was[idx]).abs() <= 0.5001 * top).all())


def test_keep_of_many_layers(cuda_lib):
    """One call for 131 caches equals a call for each."""
    from paper_2308_13137_gb300 import serve
    lens, n_q = [30, 45], [20, 33]
    many, single = ([_cache(lens, 2, 16, seed=i) for i in range(131)] for _ in range(2))
    path, count = _path_tensors([[0, 4, 19], [0, 5, 6, 30]], 6)
    tree = serve.DraftTree(torch.zeros(53, dtype=I32, device="cuda"), None, None, _cu(n_q), 33)
    serve.kv_keep(many, tree, path, count)
    for a, b in zip(many, single):
        serve.kv_keep(b, tree, path, count)
        a.check(), b.check()
        for x, y in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_keep_bad_paths(cuda_lib):
    """Paths that do not rise or leave the rows, counts out of range, and page ids out of range: reported, and the sequence
    (or page) is left as it was."""
    from paper_2308_13137_gb300 import serve
    lens, n_q, steps = [40, 40], [20, 20], 5
    tree = serve.DraftTree(torch.zeros(40, dtype=I32, device="cuda"), None, None, None, 20)
    for bad, n in (([0, 2, 2], 3), ([0, 5, 3], 3), ([0, 1, 20], 3), ([-1, 4], 2), ([0, 4, 5, 6, 7], 6), ([0, 4], -1)):
        a, b = _pair(lens, 2, 16, 3)
        path, count = _path_tensors([[0, 3, 9], bad], steps)
        count[1] = n
        serve.kv_keep(a, tree, path, count)
        assert int(a.status) == 1
        D.keep(b, 20, [0, 3, 9], 0)
        assert torch.equal(a.k, b.k) and torch.equal(a.v_scale.view(torch.int32), b.v_scale.view(torch.int32))
    a, b = _pair([40], 1, 16, 4)
    a.table[0, 2] = 10 ** 6                                    # tokens 32.. lie nowhere: row 15 stays away, row 3 moves
    path, count = _path_tensors([[0, 3, 15]], 3)
    serve.kv_keep(a, serve.DraftTree(torch.zeros(20, dtype=I32, device="cuda"), None, None, None, 20), path, count)
    assert int(a.status) == 1
    want = b.k.clone()
    p = b.table[0].tolist()
    want[p[1], :, 5] = b.k[p[1], :, 7]                        # token 23 to 21: page 1
    assert torch.equal(a.k, want)
