"""Waits of the attention of draft trees (more than 16 rows per KV head) that run out: the kernel ends by itself within its
limit, reports OMQ_ERR_TIMEOUT and leaves the context usable.  Nothing faults: a chunk of tokens is simply never handed out, or
the roles give up before what they wait for has come."""
import time

import numpy as np
import pytest
import torch

import _drafts_ref as D
from test_serve_cache_gpu import _cache
from test_serve_drafts_gpu import _tree

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32
TIMEOUT = 6


def _case(heads, n_kv, n, page):
    """A sequence of a few chunks of tokens, one that has only its tree, one without rows, and so many short ones that most CTAs
    have a few pieces of work: with the one that ends the share three chunks at least."""
    lens, n_q = [3000 + n, 200 + n, n, 50, 1025] + [20 + n] * 400, [n, n, n, 0, n] + [n] * 400
    c = _cache(lens, n_kv, page, seed=n)
    parents = [D.random_tree(k, np.random.RandomState(k)) if k else [] for k in n_q]
    tree = _tree(parents)
    q = torch.randn(sum(n_q), heads * 128, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda").to(BF16)
    return c, tree, q


class _Run:
    def __init__(self, heads, n_kv, n, page):
        from paper_2308_13137_gb300 import _lib
        self.heads = heads
        self.c, self.tree, self.q = _case(heads, n_kv, n, page)
        rows = self.q.shape[0]
        self.max_kv = 3000 + n
        self.ws = torch.empty(_lib.omq_kv_attention_tree_workspace_size(self.c.B, rows, n, self.max_kv, heads, n_kv), dtype=torch.uint8,
                              device="cuda")
        self.o = torch.empty(rows, heads * 128, device="cuda")
        self.st = torch.zeros(1, dtype=I32, device="cuda")

    def ordinary(self):
        from paper_2308_13137_gb300 import serve
        out = serve.kv_attention(self.c, self.q, self.heads, tree=self.tree, max_kv=self.max_kv, out_dtype=torch.float32)
        self.c.check()
        return out

    def __call__(self, limit, withhold):
        from paper_2308_13137_gb300 import _lib
        self.st.zero_()
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        t = self.tree
        _lib.omq_selftest_tree_wait(self.c.handle, self.q.shape[0], t.max_q, t.cu_q, t.seen, t.seen.shape[1], self.max_kv, self.heads,
                                    self.q, self.o, self.ws, limit, withhold, self.st)
        code = _lib.omq_stream_status(self.st)
        return code, time.perf_counter() - t0


# four, two and one copies of a row, a tile's tokens on one page and on several
@pytest.mark.parametrize("heads,n_kv,n,page", [(8, 1, 4, 64), (6, 1, 9, 16), (8, 1, 8, 32), (16, 2, 40, 64), (4, 1, 40, 16)])
def test_withheld_chunk(cuda_lib, heads, n_kv, n, page):
    run = _Run(heads, n_kv, n, page)
    want = run.ordinary()
    assert run(100_000_000, -1)[0] == 0 and torch.equal(run.o, want)
    for chunk in (0, 1, 2):
        code, took = run(50_000, chunk)
        assert code == TIMEOUT and took < 1.0
        assert torch.equal(run.ordinary(), want)
    run.o.zero_()
    assert run(100_000_000, -1)[0] == 0 and torch.equal(run.o, want)


@pytest.mark.parametrize("heads,n_kv,n,page", [(8, 1, 4, 64), (8, 1, 8, 32), (16, 2, 40, 64), (4, 1, 40, 16)])
def test_roles_that_give_up_anywhere(cuda_lib, heads, n_kv, n, page):
    """Limits from none at all to a few tries: the roles leave with copies and products in flight, at other places each time.
    A call either reports that or is right."""
    run = _Run(heads, n_kv, n, page)
    want = run.ordinary()
    codes = []
    for limit in (1_000, 1_400, 2_700, 4_000, 6_600, 13_000, 26_000):
        for _ in range(10):
            code, took = run(limit, -1)
            codes.append(code)
            assert code in (0, TIMEOUT) and took < 1.0
            assert code or torch.equal(run.o, want)
        assert torch.equal(run.ordinary(), want)
    assert TIMEOUT in codes[:10]                             # without a try, the first chunk is not there yet


def test_the_librarys_own_limit(cuda_lib):
    """A withheld chunk under the limit of ordinary calls: two waits one after another at most."""
    run = _Run(8, 1, 8, 32)
    want = run.ordinary()
    code, took = run(1_000_000_000, 0)
    print(f"a wait that nothing ends: {took:.3f} s")
    assert code == TIMEOUT and 0.05 < took < 2.5
    assert torch.equal(run.ordinary(), want)


def test_refusals(cuda_lib):
    from paper_2308_13137_gb300 import _lib
    run = _Run(8, 1, 8, 32)
    t, st = run.tree, run.st
    good = dict(cache=run.c.handle, total_q=run.q.shape[0], max_q=8, cu_q=t.cu_q, seen=t.seen, words=1, max_kv=run.max_kv, n_heads=8,
                Q=run.q, O=run.o, workspace=run.ws, wait_limit_ns=50_000, withhold=-1, dev_status=st)
    for bad in (dict(wait_limit_ns=10), dict(wait_limit_ns=2_000_000_000), dict(withhold=-2), dict(Q=None), dict(O=None), dict(seen=None),
                dict(words=0), dict(max_q=2), dict(workspace=None), dict(n_heads=0)):
        with pytest.raises(_lib.OmqError):
            _lib.omq_selftest_tree_wait(**dict(good, **bad))
    assert _lib.omq_stream_status(st) == 0
