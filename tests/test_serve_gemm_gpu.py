"""Product of 8-bit codes (omq_qgemm_i8).  The integer sum is exact, and its conversion, the two
scalings and the bias are one fp32 rounding each, so every output is compared bit for bit."""
import pytest
import torch

import _serve_ref as REF

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _case(M, N, K, zero, seed=0, lo=0, hi=256):
    g = torch.Generator(device="cuda").manual_seed(seed + M * 7 + N * 11 + K)
    ints = lambda a, b, *s: torch.randint(a, b, s, generator=g, device="cuda")  # noqa: E731
    a, w = ints(lo, hi, M, K).to(torch.uint8), ints(lo, hi, N, K).to(torch.uint8)
    ah = torch.rand(M, generator=g, device="cuda") * 0.1 + 0.01
    wh = torch.rand(N, generator=g, device="cuda") * 0.01 + 0.001
    az = ints(-40, 300, M).to(torch.int32) if zero else None
    wz = ints(-40, 300, N).to(torch.int32) if zero else None
    return a, ah, az, w, wh, wz, torch.randn(N, generator=g, device="cuda")


def _want(a, ah, az, w, wh, wz, bias):
    y = REF.int_product(a, az, w, wz).float() * ah[:, None] * wh[None, :]
    return y if bias is None else y + bias


SIZES = [(1, 8, 16), (1, 4096, 4096), (2, 264, 48), (3, 20000, 160), (11, 19472, 528), (5, 136, 1040), (8, 1024, 2048), (16, 520, 4112), (17, 4096, 11008),
         (33, 1000, 1024), (2, 5120, 1536), (18, 5120, 13824), (5, 2560, 4096), (64, 256, 512), (65, 2056, 1008), (127, 264, 2064), (128, 4096, 1024), (129, 512, 4096),
         (200, 1288, 208), (256, 256, 64), (300, 4104, 2064), (511, 1032, 1040), (1024, 2048, 512), (700, 6152, 1168),
         (40, 12296, 4112), (2000, 264, 128), (513, 4104, 4096), (90, 20008, 2064)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("zero", [False, True])
def test_exact(cuda_lib, M, N, K, zero):
    from paper_2308_13137_gb300 import serve
    *ops, bias = _case(M, N, K, zero)
    got = serve.qgemm(*ops, bias=bias)
    assert torch.equal(got, _want(*ops, bias))
    assert torch.equal(serve.qgemm(*ops, out_dtype=BF16), _want(*ops, None).to(BF16))


@pytest.mark.parametrize("M", [17, 23, 24, 25, 33, 41, 48, 49, 65, 72, 73])
@pytest.mark.parametrize("N,K", [(520, 2064), (4104, 1040)])
def test_rows_around_the_blocks(cuda_lib, M, N, K):
    """Blocks of 24 and 32 rows, full and with a few rows in the last."""
    from paper_2308_13137_gb300 import serve
    *ops, bias = _case(M, N, K, True)
    assert torch.equal(serve.qgemm(*ops, bias=bias), _want(*ops, bias))


@pytest.mark.parametrize("M", [1, 12, 40, 100, 300])
@pytest.mark.parametrize("K", [1024, 8192, 65536])
def test_extreme_codes(cuda_lib, M, K):
    """All codes at 0 or 255: the largest sums that the operands can make."""
    from paper_2308_13137_gb300 import serve
    a, ah, _, w, wh, _, bias = _case(M, 264, K, False, lo=0, hi=1)
    w[::2] = 255
    a[1::3] = 255
    a[:, ::2] = 0
    for zs in ((None, None), (torch.full((M,), 255, dtype=torch.int32, device="cuda"), None),
               (torch.full((M,), -70000, dtype=torch.int32, device="cuda"),
                torch.full((264,), 90001, dtype=torch.int32, device="cuda"))):
        ops = (a, ah, zs[0], w, wh, zs[1])
        assert torch.equal(serve.qgemm(*ops, bias=bias), _want(*ops, bias))


@pytest.mark.parametrize("M,N,K", [(260, 4104, 1024), (260, 4104, 8192), (300, 2056, 65536), (1100, 4096, 1040)])
def test_extreme_codes_of_many_rows(cuda_lib, M, N, K):
    """The same on the tensor-core form, with and without a split of K."""
    from paper_2308_13137_gb300 import serve
    a, ah, _, w, wh, _, bias = _case(M, N, K, False, lo=0, hi=1)
    w[::2] = 255
    a[1::3] = 255
    az = torch.full((M,), 255, dtype=torch.int32, device="cuda")
    az[7::9] = -70000
    wz = torch.full((N,), 3, dtype=torch.int32, device="cuda")
    wz[5::300] = 90001
    for zs in ((None, None), (az, None), (None, wz), (az, wz)):
        ops = (a, ah, zs[0], w, wh, zs[1])
        assert torch.equal(serve.qgemm(*ops, bias=bias), _want(*ops, bias))


@pytest.mark.parametrize("M", [3, 24, 90, 260])
def test_one_sided_zero_points_and_strides(cuda_lib, M):
    from paper_2308_13137_gb300 import serve
    a, ah, az, w, wh, wz, bias = _case(M, 520, 1040, True)
    for ops in ((a, ah, az, w, wh, None), (a, ah, None, w, wh, wz)):
        assert torch.equal(serve.qgemm(*ops), _want(*ops, None))
    wide_a, wide_w = torch.full((M, 1104), 3, dtype=torch.uint8, device="cuda"), torch.full((520, 1072), 5, dtype=torch.uint8, device="cuda")
    wide_a[:, 32:1072], wide_w[:, 16:1056] = a, w
    out = torch.full((M, 544), 7.0, device="cuda")
    got = serve.qgemm(wide_a[:, 32:1072], ah, az, wide_w[:, 16:1056], wh, wz, bias=bias, out=out[:, 8:528])
    assert torch.equal(got, _want(a, ah, az, w, wh, wz, bias))
    assert bool((out[:, :8] == 7).all()) and bool((out[:, 528:] == 7).all())


@pytest.mark.parametrize("M", [1, 20, 120, 400])
def test_both_outputs_repeat_and_side_stream(cuda_lib, M):
    from paper_2308_13137_gb300 import _lib, serve
    a, ah, az, w, wh, wz, bias = _case(M, 776, 2064, True)
    f, h = torch.empty(M, 776, device="cuda"), torch.empty(M, 776, dtype=BF16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    need = _lib.omq_qgemm_i8_workspace_size(M, 776, 2064)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    torch.cuda.synchronize()
    _lib.omq_qgemm_i8(M, 776, 2064, a, 2064, ah, az, w, 2064, wh, wz, bias, f, h, 776, ws, status, stream=s)
    s.synchronize()
    want = _want(a, ah, az, w, wh, wz, bias)
    assert torch.equal(f, want) and torch.equal(h, want.to(BF16)) and int(status) == 0
    for _ in range(3):
        assert torch.equal(serve.qgemm(a, ah, az, w, wh, wz, bias=bias), want)


def test_codes_of_the_calibration_quantizers(cuda_lib):
    """The codes, steps and zero points of omq_act_quant_per_token and omq_lwc_fakequant_fwd run as they
    are: the product equals the fp64 product of the values they stand for."""
    from paper_2308_13137_gb300 import _lib, serve
    T, Ci, Co = 37, 512, 264
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda dt, *s: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
    x = torch.randn(T, Ci, generator=g, device="cuda")
    x[5] += 40                                                   # a row far from zero: z well outside 0..255
    W = (torch.randn(Co, Ci, generator=g, device="cuda") * 0.02).to(BF16)
    cfg = _lib.make_cfg(8, 8, 0, 0)
    xq, xc, xh, xz, i0, i1 = new(BF16, T, Ci), new(torch.uint8, T, Ci), new(F32, T), *(new(torch.int32, T) for _ in range(3))
    _lib.omq_act_quant_per_token(T, Ci, x, None, None, xq, xc, xh, xz, i0, i1, cfg)
    gl, bl = torch.full((Co, 1), 4.0, device="cuda"), torch.full((Co, 1), 4.0, device="cuda")
    wc, wh, wz, j0, j1 = new(torch.uint8, Co, Ci), new(F32, Co), *(new(torch.int32, Co) for _ in range(3))
    _lib.omq_lwc_fakequant_fwd(Co, Ci, W, None, None, gl, bl, None, wc, wh, wz, j0, j1, None, None, None, cfg)
    y = serve.qgemm(xc, xh, xz, wc, wh, wz)
    xv = (xc.double() - xz.double()[:, None]) * xh.double()[:, None]
    wv = (wc.double() - wz.double()[:, None]) * wh.double()[:, None]
    want = xv @ wv.t()
    assert int(xz[5]) < -255
    assert bool(((y.double() - want).abs() <= 2.0 ** -22 * want.abs()).all())   # three roundings
