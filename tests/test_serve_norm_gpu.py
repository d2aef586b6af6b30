"""Residual addition + RMSNorm + per-token quantizer (omq_rmsnorm_quant) against float64."""
import pytest
import torch

import _parity as PY
import _serve_ref as REF

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
# single-precision roundings between the inputs and y: the sum of squares (at most 32 sequential
# products per thread, then two five-step trees: its relative error halves under the root), the
# root and quotient, the addition, two products and the bias
ULPS = 32.0


def _case(T, C, xd, rd, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + T * 131 + C)
    x = (torch.randn(T, C, generator=g, device="cuda") * 2).to(xd)
    r = None if rd is None else torch.randn(T, C, generator=g, device="cuda").to(rd)
    gain = torch.exp(0.3 * torch.randn(C, generator=g, device="cuda"))
    bias = 0.1 * torch.randn(C, generator=g, device="cuda")
    return x, r, gain, bias


def _check(name, out, x, r, gain, bias, bits, eps=1e-6):
    Q = 2 ** bits - 1
    t, y = REF.norm_rows(x, r, gain, bias, eps)
    g64 = gain.double() if gain is not None else torch.ones((), dtype=torch.float64, device=x.device)
    b64 = bias.double() if bias is not None else torch.zeros((), dtype=torch.float64, device=x.device)
    mag = (t / (t.square().mean(1, keepdim=True) + eps).sqrt() * g64).abs() + b64.abs()
    hi, lo = y.amax(1), y.amin(1)
    h = ((hi - lo) / Q).clamp_min(float(torch.tensor(1e-5)))
    tol = (ULPS * 2.0 ** -24) * 2 * mag.amax(1) / Q + 1e-7 * h
    assert bool(((out.h.double() - h).abs() <= tol).all())
    u = torch.where(h > 1e-5, Q * lo / (hi - lo).clamp_min(1e-300), lo / h)
    PY.check_zero_points(name, u.cpu(), out.z.cpu(), band_rel=ULPS * 2.0 ** -24 * 4 * 2)
    quot = (y / out.h.double()[:, None]).cpu()
    band = (ULPS * 2.0 ** -24 * mag / out.h.double()[:, None]).cpu()
    PY.check_codes(name, quot, out.codes.cpu(), out.z.cpu(), bits, band)
    if out.values is not None:
        want = ((out.codes.float() - out.z.float()[:, None]) * out.h[:, None]).to(BF16)
        assert torch.equal(out.values, want)
    if out.residual is not None:
        s = x.float() + r.float() if r is not None else x.float()
        assert torch.equal(out.residual, s.to(out.residual.dtype))


@pytest.mark.parametrize("T,C", [(1, 8), (1, 4096), (3, 136), (5, 8200), (7, 16392), (2, 28672), (300, 512), (2, 32768)])
@pytest.mark.parametrize("xd,rd", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, None)])
def test_norm_quant(cuda_lib, T, C, xd, rd):
    from paper_2308_13137_gb300 import serve
    x, r, gain, bias = _case(T, C, xd, rd)
    out = serve.rmsnorm_quant(x, r, gain, bias, values=True)
    _check(f"norm {T}x{C}", out, x, r, gain, bias, 8)


@pytest.mark.parametrize("bits", [2, 4, 6])
def test_fewer_bits_and_no_affine(cuda_lib, bits):
    from paper_2308_13137_gb300 import serve
    x, r, gain, _ = _case(33, 1024, F32, F32, seed=bits)
    _check(f"norm bits {bits}", serve.rmsnorm_quant(x, r, None, None, bits=bits, values=True), x, r, None, None, bits)
    _check(f"norm gain only {bits}", serve.rmsnorm_quant(x, r, gain, None, bits=bits), x, r, gain, None, bits)


def test_quantizer_off(cuda_lib):
    """abits = 16: the bf16 rounding of y alone."""
    from paper_2308_13137_gb300 import serve
    x, r, gain, bias = _case(9, 264, BF16, F32)
    out = serve.rmsnorm_quant(x, r, gain, bias, bits=16)
    _, y = REF.norm_rows(x, r, gain, bias, 1e-6)
    assert out.codes is None and bool(((out.values.double() - y).abs() <= 2.0 ** -8 * y.abs() + 1e-5).all())


def test_strides_and_in_place(cuda_lib):
    """Strided rows (a slice of a wider buffer) and the residual stream updated in place."""
    from paper_2308_13137_gb300 import serve
    x, r, gain, bias = _case(21, 520, F32, F32)
    wide_x, wide_r = torch.full((21, 1040), 9.0, device="cuda"), torch.full((21, 528), 7.0, device="cuda")
    wide_x[:, 8:528], wide_r[:, :520] = x, r
    xs, rs = wide_x[:, 8:528], wide_r[:, :520]
    ref = serve.rmsnorm_quant(x, r, gain, bias, values=True)
    new = lambda dt, *s: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
    out = serve.QuantRows(new(torch.uint8, 21, 520), new(F32, 21), new(torch.int32, 21), new(BF16, 21, 520), rs)
    serve.rmsnorm_quant(xs, rs, gain, bias, out=out)
    for a, b in zip(ref, out):
        assert torch.equal(a, b)
    assert bool((wide_r[:, 520:] == 7).all()) and bool((wide_x[:, :8] == 9).all())


def test_constant_zero_and_non_finite_rows(cuda_lib):
    from paper_2308_13137_gb300 import serve
    x, r, gain, bias = _case(6, 512, F32, None)
    x[1] = 0
    x[2, 17] = float("inf")
    x[3, 400] = float("nan")
    x[4, 0] = -float("inf")
    out = serve.rmsnorm_quant(x, None, gain, None, values=True)
    ok = [0, 1, 5]
    part = serve.QuantRows(out.codes[ok], out.h[ok], out.z[ok], out.values[ok])
    _check("norm rows beside non-finite ones", part, x[ok], None, gain, None, 8)
    assert float(out.h[1]) == pytest.approx(1e-5) and bool((out.values[1] == 0).all())
    for i in (2, 3, 4):
        assert bool(out.h[i].isnan()) and bool(out.values[i].isnan().all()) and int(out.codes[i].max()) == 0


def test_side_stream_and_repeat(cuda_lib):
    from paper_2308_13137_gb300 import serve
    x, r, gain, bias = _case(64, 4096, BF16, F32)
    a = serve.rmsnorm_quant(x, r, gain, bias, values=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = serve.rmsnorm_quant(x, r, gain, bias, values=True)
    s.synchronize()
    for u, v in zip(a, b):
        assert torch.equal(u, v)


def test_rows_far_from_zero(cuda_lib):
    """Rows whose values lie many steps from zero: a bias of up to 2^24 steps, beyond what the short form of
    the rounding covers, and a constant row (h floored, z large)."""
    from paper_2308_13137_gb300 import serve
    x, r, _, _ = _case(6, 512, F32, None)
    for bias in (3e3, 2e5, 1e6):
        b = torch.full((512,), bias, device="cuda")
        out = serve.rmsnorm_quant(x, r, None, b, values=True)
        _check(f"norm bias {bias:g}", out, x, r, None, b, 8)
    b = torch.full((512,), 300.0, device="cuda")
    z = torch.zeros_like(x)
    out = serve.rmsnorm_quant(z, None, None, b, values=True)
    assert bool((out.h == 1e-5).all())
    _check("norm constant row", out, z, None, None, b, 8)


def test_non_finite_bias(cuda_lib):
    from paper_2308_13137_gb300 import serve
    x, _, gain, bias = _case(3, 512, F32, None)
    for v in (float("nan"), float("inf"), -float("inf")):
        bias[77] = v
        out = serve.rmsnorm_quant(x, None, gain, bias, values=True)
        assert bool(out.h.isnan().all()) and bool(out.values.isnan().all()) and int(out.codes.max()) == 0


@pytest.mark.parametrize("C,ld", [(8, 16), (1032, 1040), (4096, 4096), (6144, 6152)])
@pytest.mark.parametrize("xd", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rd", [None, torch.float32, torch.bfloat16])
def test_many_rows_equal_few_at_a_time(cuda_lib, C, ld, xd, rd):
    """The form for many rows gives what 500 rows at a time give, bit for bit."""
    from paper_2308_13137_gb300 import serve
    g = torch.Generator(device="cuda").manual_seed(C)
    T = 2000
    x = torch.randn(T, ld, generator=g, device="cuda").to(xd)[:, :C]
    r = None if rd is None else torch.randn(T, ld, generator=g, device="cuda").to(rd)[:, :C]
    gain, bias = torch.randn(C, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda")
    whole = serve.rmsnorm_quant(x, r=r, gain=gain, bias=bias)
    for i in range(0, T, 500):
        part = serve.rmsnorm_quant(x[i:i + 500], r=None if r is None else r[i:i + 500], gain=gain, bias=bias)
        for w, p in zip(whole, part):
            if torch.is_tensor(p):
                assert torch.equal(w[i:i + 500], p)
