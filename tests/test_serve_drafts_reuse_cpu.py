"""A DraftTree whose buffers serve again in the next step describes that step (no GPU: the call itself is a stand-in)."""
import pytest
import torch

from paper_2308_13137_gb300 import serve

I32 = torch.int32


class _Calls:
    """Takes draft_tree's arguments and reports success."""

    def draft_tree(self, parent, cu_q, max_q, depth, seen, status):
        self.got = (parent, cu_q, max_q, depth, seen)
        return 0


@pytest.fixture
def calls(monkeypatch):
    c = _Calls()
    monkeypatch.setattr(serve, "_calls", c)
    return c


def _ints(*v):
    return torch.tensor(v, dtype=I32)


def _out(parent, cu_q, max_q, rows=6):
    return serve.DraftTree(parent, torch.zeros(rows, dtype=I32), torch.zeros(rows, 1, dtype=I32), cu_q, max_q)


def test_the_next_steps_tree_in_the_same_buffers(calls):
    old = _out(_ints(-1, 0, 0, -1, 0, 1), _ints(0, 3, 6), 3)
    parent, cu = _ints(-1, 0, 1, 2, -1, 0), _ints(0, 4, 6)
    t = serve.draft_tree(parent, cu, 4, out=old)
    assert t.parent is parent and t.cu_q is cu and t.max_q == 4 and t.depth is old.depth and t.seen is old.seen
    assert calls.got == (parent, cu, 4, old.depth, old.seen)


@pytest.mark.parametrize("change", ["parent", "cu_q", "max_q", "no cu_q", "no parent"])
def test_one_of_them_is_another(calls, change):
    parent, cu = _ints(-1, 0, 0, -1, 0, 1), _ints(0, 3, 6)
    old = _out(parent, cu, 3)
    if change == "parent":
        parent = parent.clone()
    elif change == "cu_q":
        cu = _ints(0, 3, 6)
    elif change == "no cu_q":
        old = old._replace(cu_q=None)
    elif change == "no parent":
        old = old._replace(parent=None)
    max_q = 4 if change == "max_q" else 3
    t = serve.draft_tree(parent, cu, max_q, out=old)
    assert t.parent is parent and t.cu_q is cu and t.max_q == max_q and t.depth is old.depth and t.seen is old.seen


def test_rows_of_equal_number(calls):
    old = _out(_ints(-1, 0, 0, -1, 0, 1), _ints(0, 3, 6), 3)
    parent = _ints(-1, 0, 1, -1, 0, 1).view(2, 3)
    t = serve.draft_tree(parent, out=old)
    assert t.cu_q is None and t.max_q == 3 and t.parent.data_ptr() == parent.data_ptr() and t.parent.shape == (6,)
    # refilled in place: the tree is the one that was handed in
    assert serve.draft_tree(parent, out=t) is t
    again = _out(_ints(-1, 0, 0, -1, 0, 1), _ints(0, 3, 6), 3)
    assert serve.draft_tree(again.parent, again.cu_q, 3, out=again) is again
