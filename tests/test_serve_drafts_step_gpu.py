"""Steps that check drafted tokens: the operators one after another, eager and captured, in a block, on two streams, over caches that
are slices of pooled tensors, and over batches of thousands of sequences."""
import numpy as np
import pytest
import torch

import _drafts_ref as D
from test_serve_block_gpu import _case, _rel
from test_serve_cache_gpu import _cache, _cu
from test_serve_drafts_gpu import CHAIN, F32, I32, _attend, _check, _dev, _path_tensors, _tree, _trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,n", [(2, 2), (8, 3), (16, 5), (32, 5)])
def test_thousands_of_sequences_mostly_without_tokens(cuda_lib, heads, n):
    """A CTA's share has more sequences without tokens in a row than it looks ahead, and sequences of one tile."""
    B = 3000
    r = np.random.RandomState(heads)
    lens = [int(r.randint(1, 200)) if i % 89 == 5 or 1000 <= i < 1020 else 0 for i in range(B)]
    n_q = [n] * B
    masks = [D.ancestors(CHAIN(n))] * B
    c = _cache(lens, 1, 16, seed=heads)
    _check(c, n_q, heads, masks, *_attend(c, n_q, heads, masks, tree=_tree([CHAIN(n)] * B)))


def _pooled(c):
    """The same cache as the middle one of three layers, and it alone."""
    from paper_2308_13137_gb300 import serve
    pools = [torch.stack([t, t, t]) for t in (c.k, c.v, c.k_scale, c.v_scale)]
    assert pools[2][1].data_ptr() % 16 != 0
    return serve.KVCache(*[p[1] for p in pools], c.table, c.kv_len), pools


def test_layers_of_one_tensor(cuda_lib):
    """Scales of a layer start at any fp32 boundary of the tensor that holds all layers'."""
    from paper_2308_13137_gb300 import serve
    for heads, n in ((2, 4), (8, 8)):
        a = _cache([40, 25], 1, 16, seed=heads)
        b, pools = _pooled(a)
        parents = _trees([n, n], 5)
        tree = _tree(parents)
        x = torch.randn(2 * n, (heads + 2) * 128, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
        rope = serve.rope_table(64)
        path, count = _path_tensors([[0, 2, 3], [0, 3]], 4)
        out = []
        for c in (a, b):
            q = serve.kv_append(c, x, rope, heads, tree=tree)
            o = serve.kv_attention(c, q, heads, tree=tree)
            serve.kv_keep([c], tree, path, count)
            c.check()
            out.append((q, o, c.k.clone(), c.v.clone(), c.k_scale.view(I32).clone(), c.v_scale.view(I32).clone()))
        assert all(torch.equal(s, t) for s, t in zip(*out))
        assert all(torch.equal(p[0].view(torch.uint8), p[2].view(torch.uint8)) for p in pools)


def _step(s, caches, tree):
    from paper_2308_13137_gb300 import serve
    serve.draft_tree(s["parent"], s["cu"], s["max_q"], out=tree, status=caches[0].status)
    outs = []
    for c in caches:
        q = serve.kv_append(c, s["qkv"], s["rope"], s["heads"], tree=tree)
        outs.append(serve.kv_attention(c, q, s["heads"], tree=tree))
    got = serve.verify_drafts(tree, s["tokens"], s["probs"], s["u"], draft_probs=s["draft"], steps=5, status=caches[0].status)
    serve.kv_keep(caches, tree, got.path, got.count)
    return outs + list(got)


@pytest.mark.parametrize("heads,n_kv,n", [(4, 4, 6), (8, 1, 7), (16, 2, 40)])
def test_step_eager_and_captured(cuda_lib, heads, n_kv, n):
    """A whole step over two layers' caches, captured on a side stream and replayed over other numbers in the same buffers, gives
    the same bits as the calls one by one, in the outputs and in the caches."""
    from paper_2308_13137_gb300 import serve
    V, lens = 4567, [70 + n, n, 900]
    n_q = [n, n, 3]

    def numbers(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rows, total = sum(n_q), heads + 2 * n_kv
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        return dict(parent=_dev(sum(_trees(n_q, seed, depth=4), [])), cu=_cu(n_q), max_q=n, heads=heads,
                    qkv=rand(rows, total * 128), rope=serve.rope_table(1024), tokens=torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=I32),
                    probs=torch.softmax(3 * rand(rows, V), -1), draft=torch.softmax(3 * rand(rows, V), -1),
                    u=torch.rand(rows, generator=g, device="cuda") * 0.3)

    def fresh(seed):
        return [_cache(lens, n_kv, 16, seed=seed + i) for i in range(2)]

    def plan(s):
        rows = sum(n_q)
        return serve.DraftTree(s["parent"], torch.empty(rows, dtype=I32, device="cuda"),
                               torch.empty(rows, (n + 31) // 32, dtype=I32, device="cuda"), s["cu"], n)

    state = lambda cs: [t.clone() for c in cs for t in (c.k, c.v, c.k_scale.view(I32), c.v_scale.view(I32))]  # noqa: E731
    want = {}
    for seed in (1, 2, 3):
        s, cs = numbers(seed), fresh(10 * seed)
        want[seed] = [t.clone() for t in _step(s, cs, plan(s))] + state(cs)
        for c in cs:
            c.check()

    s, cs = numbers(1), fresh(10)
    tree = plan(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(s, cs, tree)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = _step(s, cs, tree)
    for seed in (2, 3, 2, 1):
        for k, t in numbers(seed).items():
            if torch.is_tensor(t):
                s[k].copy_(t)
        for c, f in zip(cs, fresh(10 * seed)):
            for x, y in ((c.k, f.k), (c.v, f.v), (c.k_scale, f.k_scale), (c.v_scale, f.v_scale), (c.table, f.table), (c.kv_len, f.kv_len)):
                x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for c in cs:
            c.check()
        assert all(torch.equal(x, y) for x, y in zip(outs + state(cs), want[seed]))


def test_two_streams(cuda_lib):
    """Calls on two streams at once have workspaces of their own."""
    cases = []
    for seed, (heads, n, lens) in enumerate([(8, 8, [3000, 90, 1700]), (8, 6, [2500, 2400, 40]), (2, 3, [5000, 77, 310]), (16, 20, [900, 1100, 700])]):
        parents = _trees([n] * 3, seed)
        masks = [D.ancestors(p) for p in parents]
        c = _cache(lens, 1, 32, seed=seed)
        tree = _tree(parents)
        cases.append((c, [n] * 3, heads, masks, tree) + _attend(c, [n] * 3, heads, masks, tree=tree))
    from paper_2308_13137_gb300 import serve
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[] for _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, (c, _, heads, _, tree, q, _, _) in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                got[i].append(serve.kv_attention(c, q, heads, tree=tree, out_dtype=F32))
    torch.cuda.synchronize()
    for i, case in enumerate(cases):
        case[0].check()
        assert all(torch.equal(o, case[6]) for o in got[i])


@pytest.mark.parametrize("n_heads,n_kv", [(4, 4), (8, 2), (8, 1)])
def test_trees_through_a_block(cuda_lib, n_heads, n_kv):
    """Every drafted row's output is that of its branch alone, given as a chain of new tokens, and so is the step after the accepted
    branch has been kept: up to the quantizers' noise (a page's scale depends on the rows beside the branch), which the
    block's other tests bound by 6 % of its contribution."""
    from paper_2308_13137_gb300 import serve
    sh, blk, x, _, _ = _case(n_heads, n_kv, 1, 8)
    rope = serve.rope_table(sh.T)
    start, parents = [40, 21], [[-1, 0, 0, 1, 1, 4], [-1, 0, 1, 2, 1, 0]]
    n_q = [6, 6]
    ctx = [x[:40], x[40:61]]
    new = [x[61:67], x[67:73]]

    def context():
        c = blk.cache(2, 64, page=16)
        c.kv_len.copy_(torch.tensor(start, dtype=I32))
        blk.forward(torch.cat(ctx), c, rope, cu_q=_cu(start), max_q=max(start))
        return c

    c = context()
    c.kv_len.add_(6)
    h, d = blk.forward(torch.cat(new), c, rope, tree=_tree(parents))
    c.check()
    out = (h + d).split(n_q)
    for rows in (([0, 1, 3], [0, 1, 2, 3]), ([0, 1, 4, 5], [0, 1, 4]), ([0, 2], [0, 5])):
        p = context()
        k = [len(r) for r in rows]
        p.kv_len.copy_(torch.tensor([s + m for s, m in zip(start, k)], dtype=I32))
        h, d = blk.forward(torch.cat([t[r] for t, r in zip(new, rows)]), p, rope, cu_q=_cu(k), max_q=max(k))
        for y, o, t, r in zip((h + d).split(k), out, new, rows):
            assert _rel(o[r] - t[r], y - t[r]) < 0.06
    # the branches of the second round are kept; the next token of each sequence
    c, rows = context(), ([0, 1, 4, 5], [0, 1, 4])
    c.kv_len.add_(6)
    tree = _tree(parents)
    blk.forward(torch.cat(new), c, rope, tree=tree)
    path, count = _path_tensors(rows, 6)
    serve.kv_keep(c, tree, path, count)
    c.kv_len.copy_(torch.tensor([s + len(r) + 1 for s, r in zip(start, rows)], dtype=I32))
    h, d = blk.forward(x[73:75], c, rope, max_q=1)
    c.check()
    p = context()
    k = [len(r) for r in rows]
    p.kv_len.copy_(torch.tensor([s + m for s, m in zip(start, k)], dtype=I32))
    blk.forward(torch.cat([t[r] for t, r in zip(new, rows)]), p, rope, cu_q=_cu(k), max_q=max(k))
    p.kv_len.add_(1)
    h2, d2 = blk.forward(x[73:75], p, rope, max_q=1)
    assert _rel(h + d - x[73:75], h2 + d2 - x[73:75]) < 0.06
