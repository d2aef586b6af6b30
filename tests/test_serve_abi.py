"""Refusals of the 8-bit serving entry points: found on the host, before any launch (no GPU)."""
import ctypes
import os

import pytest

from paper_2308_13137_gb300 import _lib

pytestmark = pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libomq.so not built")
FAKE = 0x10000     # 16-byte aligned dummy address: every call below returns before touching it
INVALID, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 7


def _norm(T=4, C=512, X=FAKE, xd=0, ldx=512, R=FAKE, H=FAKE, rd=0, ldr=512, gain=FAKE, eps=1e-6, codes=FAKE, Xq=FAKE,
          h=FAKE, z=FAKE, bits=8, cfg=True):
    c = _lib.omq_qcfg(16, bits, 0, 0, 1e-5, 0, None, 0, 0)
    return _lib.lib().omq_rmsnorm_quant(None, T, C, X, xd, ldx, R, H, rd, ldr, gain, None, eps, codes, Xq, h, z,
                                        ctypes.byref(c) if cfg else None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=0), SHAPE), (dict(C=0), SHAPE), (dict(C=32776, ldx=32776, ldr=32776), SHAPE), (dict(ldx=504), SHAPE),
    (dict(ldr=8), SHAPE), (dict(C=500), ALIGN), (dict(ldx=516), ALIGN), (dict(ldr=516), ALIGN), (dict(X=FAKE + 8), ALIGN),
    (dict(gain=FAKE + 4), ALIGN), (dict(X=None), INVALID), (dict(codes=None, Xq=None), INVALID),
    (dict(bits=16, Xq=None), INVALID), (dict(h=None), INVALID), (dict(z=None), INVALID), (dict(xd=2), INVALID),
    (dict(rd=-1), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(bits=9), UNSUPPORTED),
    (dict(cfg=False), INVALID)])
def test_norm_refusals(kw, code):
    assert _norm(**kw) == code


def _gemm(M=4, N=64, K=128, A=FAKE, lda=128, ah=FAKE, az=None, B=FAKE, ldb=128, bh=FAKE, bz=None, bias=None, Cf=FAKE,
          Cb=None, ldc=64, ws=None, ws_bytes=0):
    return _lib.lib().omq_qgemm_i8(None, M, N, K, A, lda, ah, az, B, ldb, bh, bz, bias, Cf, Cb, ldc, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(M=0), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(K=65552, lda=65552, ldb=65552), SHAPE),
    (dict(lda=112), SHAPE), (dict(ldb=112), SHAPE), (dict(ldc=56), SHAPE), (dict(M=1 << 22), SHAPE),
    (dict(K=120), ALIGN), (dict(lda=136), ALIGN), (dict(ldb=136), ALIGN), (dict(N=60), ALIGN), (dict(ldc=68), ALIGN),
    (dict(A=FAKE + 8), ALIGN), (dict(bias=FAKE + 4), ALIGN), (dict(az=FAKE + 4), ALIGN), (dict(A=None), INVALID),
    (dict(B=None), INVALID), (dict(ah=None), INVALID), (dict(bh=None), INVALID), (dict(Cf=None), INVALID), (dict(ws=FAKE + 8), ALIGN),
    (dict(M=2048, N=4096, K=8192, lda=8192, ldb=8192, ldc=4096), WORKSPACE),
    (dict(M=2048, N=4096, K=8192, lda=8192, ldb=8192, ldc=4096, ws=FAKE, ws_bytes=64), WORKSPACE)])
def test_gemm_refusals(kw, code):
    assert _gemm(**kw) == code


def _cache(**kw):
    f = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, page_table=FAKE, kv_len=FAKE, n_pages=10, n_kv=2, page=64,
             max_pages=4, B=3)
    f.update(kw)
    return _lib.omq_kv_cache(*[f[n] for n, _ in _lib.omq_kv_cache._fields_])


def _append(cache=None, total=3, max_q=1, cu=None, heads=4, X=FAKE, dt=0, ld=1024, rope=FAKE, n_pos=64, Q=FAKE, ldq=512,
            K=None, V=None, ldkv=0):
    c = cache if cache is not None else _cache()
    return _lib.lib().omq_kv_append(None, ctypes.byref(c), total, max_q, cu, heads, X, dt, ld, rope, n_pos, None, Q, ldq, K,
                                    V, ldkv, None)


def _attend(cache=None, total=3, max_q=1, cu=None, max_kv=256, heads=4, Q=FAKE, ldq=512, Of=FAKE, Ob=None, ldo=512,
            ws=FAKE, ws_bytes=1 << 40):
    c = cache if cache is not None else _cache()
    return _lib.lib().omq_kv_attention(None, ctypes.byref(c), total, max_q, cu, max_kv, heads, Q, ldq, Of, Ob, ldo, None, ws,
                                       ws_bytes, None)


BAD_CACHES = [(dict(k=None), INVALID), (dict(v_scale=None), INVALID), (dict(page_table=None), INVALID),
              (dict(kv_len=None), INVALID), (dict(page=48), SHAPE), (dict(page=0), SHAPE), (dict(n_kv=0), SHAPE),
              (dict(n_kv=3), SHAPE), (dict(B=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(max_pages=0), SHAPE),
              (dict(v=FAKE + 8), ALIGN), (dict(kv_len=FAKE + 4), ALIGN)]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_cache_refusals(kw, code):
    assert _append(_cache(**kw)) == code and _attend(_cache(**kw)) == code


ROWS = [(dict(total=4), SHAPE), (dict(max_q=0), SHAPE), (dict(total=0), SHAPE), (dict(max_q=5, cu=FAKE), SHAPE),
        (dict(cu=FAKE + 4), ALIGN), (dict(heads=5), SHAPE), (dict(heads=0), SHAPE)]


@pytest.mark.parametrize("kw,code", ROWS + [
    (dict(X=None), INVALID), (dict(rope=None), INVALID), (dict(Q=None), INVALID), (dict(K=FAKE), INVALID), (dict(dt=3), INVALID),
    (dict(n_pos=0), SHAPE), (dict(ld=1016), SHAPE), (dict(ldq=504), SHAPE), (dict(K=FAKE, V=FAKE, ldkv=248), SHAPE),
    (dict(ld=1028), ALIGN), (dict(ldq=516), ALIGN), (dict(K=FAKE, V=FAKE + 8, ldkv=256), ALIGN), (dict(X=FAKE + 4), ALIGN)])
def test_append_refusals(kw, code):
    assert _append(**kw) == code


@pytest.mark.parametrize("kw,code", ROWS + [
    (dict(Q=None), INVALID), (dict(Of=None), INVALID), (dict(max_kv=0), SHAPE), (dict(ldq=504), SHAPE), (dict(ldo=504), SHAPE),
    (dict(ldq=516), ALIGN), (dict(ldo=516), ALIGN), (dict(Q=FAKE + 8), ALIGN), (dict(ws=FAKE + 8), ALIGN),
    (dict(max_kv=100000, ws=None, ws_bytes=0), WORKSPACE), (dict(max_kv=100000, ws_bytes=64), WORKSPACE)])
def test_attention_refusals(kw, code):
    assert _attend(**kw) == code


def test_gemm_workspace_size():
    size = _lib.omq_qgemm_i8_workspace_size
    assert size(1, 4096, 4096) == 0 and size(0, 8, 16) == 0 and size(512, 0, 64) == 0
    assert size(2048, 22016, 4096) >= 2048 * 4096 * 2              # the widened activation codes


def test_workspace_size():
    size = _lib.omq_kv_attention_workspace_size
    assert size(512, 512, 1, 256, 32, 32) == 0                 # enough sequences and heads: nothing is split
    assert size(1, 1, 1, 131072, 8, 8) > 8 * 128 * 4           # one long sequence: one partial result per chunk and head
    assert size(0, 1, 1, 64, 8, 8) == 0 and size(1, 1, 1, 64, 8, 3) == 0


def test_rope_table_refusals():
    f = _lib.lib().omq_rope_table
    assert f(None, 0, 10000.0, FAKE) == SHAPE and f(None, 8, 10000.0, None) == INVALID
    assert f(None, 8, 0.0, FAKE) == INVALID and f(None, 8, 10000.0, FAKE + 8) == ALIGN
