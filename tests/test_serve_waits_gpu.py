"""A wait of the integer product that runs out: the kernel ends by itself within its limit, reports
OMQ_ERR_TIMEOUT, and leaves the context usable.  Nothing faults: the first tile is simply never loaded."""
import time

import pytest
import torch

import _serve_ref as REF

pytestmark = pytest.mark.gpu
U8 = torch.uint8


def _case(M, N, K):
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    a, w = (torch.randint(0, 256, (n, K), generator=g, device="cuda", dtype=torch.int32).to(U8) for n in (M, N))
    ah, wh = torch.rand(M, generator=g, device="cuda") + 0.5, torch.rand(N, generator=g, device="cuda") + 0.5
    return a, ah, w, wh, REF.int_product(a, None, w, None).float() * ah[:, None] * wh


# one to five tiles per CTA, a ring that is filled again, clusters of one and more, every block of rows
@pytest.mark.parametrize("M,N,K", [(1, 64, 256), (3, 4096, 4096), (12, 264, 65536), (20, 5120, 1024), (32, 20000, 4096)])
def test_withheld_tile(cuda_lib, M, N, K):
    from paper_2308_13137_gb300 import _lib, serve
    a, ah, w, wh, want = _case(M, N, K)
    C, st = torch.empty(M, N, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(limit, withhold):
        st.zero_()
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        _lib.omq_selftest_qgemm_wait(M, N, K, a, ah, w, wh, C, limit, withhold, st)
        code = _lib.omq_stream_status(st)
        return code, time.perf_counter() - t0

    assert run(100_000_000, 0)[0] == 0 and torch.equal(C, want)
    code, took = run(50_000, 1)
    assert code == 6 and took < 1.0                          # OMQ_ERR_TIMEOUT
    C.zero_()
    assert run(100_000_000, 0)[0] == 0 and torch.equal(C, want)
    assert torch.equal(serve.qgemm(a, ah, None, w, wh, None), want)


def test_the_librarys_own_limit_is_a_second(cuda_lib):
    """Two waits one after another at most: for a tile, and for the copies in flight before the CTA leaves.  A
    wait is a quarter of a million tries."""
    from paper_2308_13137_gb300 import _lib
    a, ah, w, wh, want = _case(2, 128, 2048)
    C, st = torch.empty(2, 128, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    _lib.omq_selftest_qgemm_wait(2, 128, 2048, a, ah, w, wh, C, 1_000_000_000, 1, st)
    assert _lib.omq_stream_status(st) == 6
    assert time.perf_counter() - t0 < 2.5
    st.zero_()
    _lib.omq_selftest_qgemm_wait(2, 128, 2048, a, ah, w, wh, C, 1_000_000_000, 0, st)
    assert _lib.omq_stream_status(st) == 0 and torch.equal(C, want)


def test_refusals(cuda_lib):
    from paper_2308_13137_gb300 import _lib
    a, ah, w, wh, _ = _case(2, 128, 256)
    C, st = torch.empty(2, 128, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    good = dict(M=2, N=128, K=256, A=a, a_h=ah, B=w, b_h=wh, C=C, wait_limit_ns=50_000, withhold=0, dev_status=st)
    for bad in (dict(M=33), dict(M=0), dict(N=124), dict(K=250), dict(N=65544), dict(A=None), dict(C=None),
                dict(wait_limit_ns=2_000_000_000), dict(wait_limit_ns=10), dict(withhold=2)):
        with pytest.raises(_lib.OmqError):
            _lib.omq_selftest_qgemm_wait(**dict(good, **bad))
    assert _lib.omq_stream_status(st) == 0
