"""Refusals of the entry points for drafted tokens: found on the host, before any launch (no GPU)."""
import ctypes
import os

import pytest

from paper_2308_13137_gb300 import _lib
from test_serve_abi import ALIGN, BAD_CACHES, FAKE, INVALID, ROWS, SHAPE, WORKSPACE, _cache

pytestmark = pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libomq.so not built")


def _tree(B=3, total=9, max_q=3, cu=None, parent=FAKE, depth=FAKE, seen=FAKE, words=1):
    return _lib.lib().omq_draft_tree(None, B, total, max_q, cu, parent, depth, seen, words, None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), SHAPE), (dict(B=70000, total=210000), SHAPE), (dict(total=8), SHAPE), (dict(max_q=0), SHAPE), (dict(total=0), SHAPE),
    (dict(max_q=1025, B=1, total=1025, words=40), SHAPE), (dict(max_q=33, B=1, total=33), SHAPE), (dict(words=0), SHAPE),
    (dict(words=2000), SHAPE), (dict(max_q=10, cu=FAKE), SHAPE), (dict(parent=None), INVALID), (dict(depth=None), INVALID),
    (dict(seen=None), INVALID), (dict(parent=FAKE + 2), ALIGN), (dict(cu=FAKE + 1), ALIGN)])
def test_tree_refusals(kw, code):
    assert _tree(**kw) == code


def _append(cache=None, total=3, max_q=1, cu=None, heads=4, depth=FAKE, X=FAKE, ld=1024, Q=FAKE, ldq=512):
    c = cache if cache is not None else _cache()
    return _lib.lib().omq_kv_append_tree(None, ctypes.byref(c), total, max_q, cu, depth, heads, X, 0, ld, FAKE, 64, None, Q, ldq,
                                         None, None, 0, None)


def _attend(cache=None, total=3, max_q=1, cu=None, seen=FAKE, words=1, max_kv=256, heads=4, Q=FAKE, ldq=512, Of=FAKE, ldo=512,
            ws=FAKE, ws_bytes=1 << 40):
    c = cache if cache is not None else _cache()
    return _lib.lib().omq_kv_attention_tree(None, ctypes.byref(c), total, max_q, cu, seen, words, max_kv, heads, Q, ldq, Of, None,
                                            ldo, None, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_cache_refusals(kw, code):
    c = _cache(**kw)
    assert _append(c) == code and _attend(c) == code
    if "n_kv" not in kw or kw["n_kv"] != 3:                    # (no heads in that call)
        assert _keep([c]) == code


@pytest.mark.parametrize("kw,code", ROWS + [(dict(depth=None), INVALID), (dict(depth=FAKE + 2), ALIGN), (dict(X=None), INVALID),
                                            (dict(ld=1016), SHAPE), (dict(ldq=516), ALIGN)])
def test_append_refusals(kw, code):
    assert _append(**kw) == code


@pytest.mark.parametrize("kw,code", ROWS + [
    (dict(seen=None), INVALID), (dict(seen=FAKE + 2), ALIGN), (dict(words=0), SHAPE), (dict(max_q=33, total=99), SHAPE),
    (dict(max_q=-5), SHAPE), (dict(Q=None), INVALID), (dict(Of=None), INVALID), (dict(max_kv=0), SHAPE), (dict(ldo=504), SHAPE),
    (dict(ldq=516), ALIGN), (dict(ws=FAKE + 8), ALIGN), (dict(max_kv=100000, ws=None, ws_bytes=0), WORKSPACE),
    (dict(max_kv=100000, ws_bytes=64), WORKSPACE)])
def test_attention_refusals(kw, code):
    assert _attend(**kw) == code


def test_attention_workspace_size():
    size = _lib.omq_kv_attention_tree_workspace_size
    assert size(1, 1, 1, 131072, 8, 8) > 0
    assert size(0, 1, 1, 64, 8, 8) == 0 and size(1, 1, 1, 64, 8, 3) == 0 and size(1, 1, 0, 64, 8, 8) == 0


def _verify(B=3, total=9, max_q=3, cu=None, parent=FAKE, tokens=FAKE, V=100, P=FAKE, Q=FAKE, dt=0, ldp=100, ldq=100, u=FAKE, steps=3,
            out=FAKE, path=FAKE, count=FAKE):
    return _lib.lib().omq_verify_drafts(None, B, total, max_q, cu, parent, tokens, V, P, Q, dt, ldp, ldq, u, steps, out, path, count,
                                        None)


@pytest.mark.parametrize("kw,code", [
    (dict(parent=None), INVALID), (dict(tokens=None), INVALID), (dict(P=None), INVALID), (dict(u=None), INVALID),
    (dict(out=None), INVALID), (dict(path=None), INVALID), (dict(count=None), INVALID), (dict(dt=2), INVALID), (dict(B=0), SHAPE),
    (dict(total=10), SHAPE), (dict(max_q=0), SHAPE), (dict(max_q=1025, B=1, total=1025), SHAPE), (dict(steps=0), SHAPE),
    (dict(steps=1025), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 20) + 1, ldp=1 << 21, ldq=1 << 21), SHAPE), (dict(ldp=99), SHAPE),
    (dict(ldq=99), SHAPE), (dict(P=FAKE + 2), ALIGN), (dict(Q=FAKE + 1, dt=1), ALIGN), (dict(u=FAKE + 2), ALIGN),
    (dict(tokens=FAKE + 2), ALIGN), (dict(count=FAKE + 1), ALIGN)])
def test_verify_refusals(kw, code):
    assert _verify(**kw) == code


def _keep(caches, total=3, max_q=1, cu=None, path=FAKE, steps=2, count=FAKE, n=None, null=False):
    held = (ctypes.c_void_p * max(1, len(caches)))(*[ctypes.addressof(c) if c is not None else None for c in caches])
    return _lib.lib().omq_kv_keep(None, None if null else held, None, len(caches) if n is None else n, total, max_q, cu, path, steps,
                                  count)


@pytest.mark.parametrize("kw,code", ROWS[:5] + [
    (dict(path=None), INVALID), (dict(count=None), INVALID), (dict(steps=0), SHAPE), (dict(steps=1025), SHAPE),
    (dict(path=FAKE + 2), ALIGN), (dict(count=FAKE + 1), ALIGN), (dict(n=0), INVALID), (dict(null=True), INVALID)])
def test_keep_refusals(kw, code):
    assert _keep([_cache()], **kw) == code


def test_keep_of_unlike_or_repeated_caches():
    a, b = _cache(), _cache(k=FAKE * 2, v=FAKE * 3)
    assert _keep([a, None]) == INVALID
    assert _keep([a, _cache(k=FAKE * 2, v=FAKE * 3, page=32)]) == SHAPE
    assert _keep([a, _cache(k=FAKE * 2, v=FAKE * 3, n_kv=4)]) == SHAPE
    assert _keep([b, a, b]) == INVALID and _keep([a, a]) == INVALID           # moved twice at once
    assert _keep([a, _cache(k=FAKE * 2)]) == INVALID                          # another's values
