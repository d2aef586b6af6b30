"""8-bit paged cache: the write of new tokens (omq_kv_append) and attention over it (omq_kv_attention)
against float64."""
import math

import pytest
import torch

import _serve_ref as REF

pytestmark = pytest.mark.gpu
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64


def _cache(lens, n_kv, page, seed=0, fill=True, spare=2):
    """A cache whose pages lie in random order; unused pages hold codes 255 and NaN scales."""
    from paper_2308_13137_gb300 import serve
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + spare
    table = torch.full((len(lens), max(1, max(need) + 1)), -7, dtype=torch.int32)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (n_pages, n_kv, page, 128)
    used = torch.zeros(n_pages, dtype=torch.bool)
    used[order[:at]] = True

    def codes():
        c = (torch.randn(shape, generator=g, device="cuda") * 35 + 128).round().clamp(1, 255).to(torch.uint8)
        c[~used.cuda()] = 255
        for b, n in enumerate(lens):                       # slots beyond the last token
            if n % page:
                c[table[b, need[b] - 1], :, n % page:] = 255
        return c

    def scales(spread):
        s = torch.exp(spread * torch.randn(n_pages, n_kv, generator=g, device="cuda")) / 30
        s[~used.cuda()] = float("nan")
        return s

    return serve.KVCache(codes(), codes(), scales(0.3), scales(1.0), table.cuda(),
                         torch.tensor(lens, dtype=torch.int32, device="cuda"))


def _cu(n):
    return torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device="cuda")


def _attend(cache, n_q, heads, seed=1, q=None, **kw):
    from paper_2308_13137_gb300 import serve
    total = sum(n_q)
    if q is None:
        g = torch.Generator(device="cuda").manual_seed(seed)
        q = (torch.randn(total, heads * 128, generator=g, device="cuda") * 1.5).to(BF16)
    lse = torch.empty(total, heads, device="cuda")
    out = serve.kv_attention(cache, q, heads, cu_q=_cu(n_q), max_q=max(n_q), lse=lse, out_dtype=F32, **kw)
    cache.check()
    return q, out, lse


def _check(cache, n_q, heads, q, out, lse):
    """Weights are rounded to fp16 (2^-11 relative each), everything else to fp32, so an output is within
    2^-11 of the largest |v| the row sees; half as much again covers the fp32 parts."""
    cu = _cu(n_q).tolist()
    O, L, top = REF.attention(cache, q, heads, [(cu[b], n) for b, n in enumerate(n_q)])
    got = out.double().view(O.shape)
    assert bool(((got - O).abs() <= 1.5 * 2.0 ** -11 * top[..., None]).all()), float(((got - O).abs() / top[..., None].clamp_min(1e-30)).max())
    empty = torch.isinf(L)
    assert torch.equal(torch.isinf(lse), empty) and bool((got[empty] == 0).all())
    assert bool(((lse.double() - L)[~empty].abs() <= 1e-4).all())


LAYOUTS = [(1, 1), (4, 4), (8, 1), (6, 2), (14, 2), (16, 2)]


@pytest.mark.parametrize("heads,n_kv", LAYOUTS)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_decode(cuda_lib, heads, n_kv, page):
    """One new token per sequence at lengths of zero, one, around a page and a tile, and several pages."""
    lens = [1, 0, 2, 15, 16, 17, page - 1, page, page + 1, 3 * page + 5, 700]
    c = _cache(lens, n_kv, page, seed=heads * 100 + page)
    n_q = [1] * len(lens)
    _check(c, n_q, heads, *_attend(c, n_q, heads))


@pytest.mark.parametrize("heads,n_kv", LAYOUTS)
@pytest.mark.parametrize("n_q", [[2, 5, 1, 3], [8, 8, 8, 8], [16, 0, 1, 9], [40, 7, 70, 33]])
def test_several_new_tokens(cuda_lib, heads, n_kv, n_q):
    """Ragged rows, sequences shorter than their rows (their first rows see nothing), none at all."""
    lens = [max(n_q[0], 300), max(0, n_q[1] - 3), 70, 45]
    c = _cache(lens, n_kv, 32, seed=heads + sum(n_q))
    _check(c, n_q, heads, *_attend(c, n_q, heads))


@pytest.mark.parametrize("heads,n_kv,n_q", [(8, 8, 1), (8, 1, 1), (8, 1, 3), (4, 2, 20)])
def test_long_context_is_split(cuda_lib, heads, n_kv, n_q):
    lens = [9001, 130, 0]
    c = _cache(lens, n_kv, 64, seed=5)
    _check(c, [n_q] * 3, heads, *_attend(c, [n_q] * 3, heads))


def test_scales_of_very_different_size(cuda_lib):
    """A row whose weight lies on pages with a V scale 2^-20 of the others', and pages with zero scales."""
    c = _cache([512, 512], 2, 16, seed=9)
    tab = c.table.long()
    c.v_scale[tab[0, :16]] *= 2.0 ** -20
    c.k_scale[tab[0, 16:32]] *= 1e-3
    c.v_scale[tab[1, 3:6]] = 0
    c.k_scale[tab[1, 8:9]] = 0
    q, out, lse = _attend(c, [1, 1], 4)
    _check(c, [1, 1], 4, q, out, lse)
    # all of a sequence's values zero: the rows are zero and the sum still counts
    c.v_scale[tab[1, :32]] = 0
    q, out, lse = _attend(c, [1, 1], 4)
    assert bool((out[1] == 0).all()) and bool(torch.isfinite(lse[1]).all())
    # keys far from the others in scale: the whole weight on a small-valued page
    c2 = _cache([64], 1, 16, seed=10)
    t2 = c2.table.long()
    c2.v_scale[t2[0, 0]] *= 2.0 ** -12
    c2.k_scale[t2[0, 1:4]] *= 1e-6
    c2.k[t2[0, 0]] = 255
    q = torch.full((1, 128), 30.0, device="cuda").to(BF16)
    q, out, lse = _attend(c2, [1], 1, q=q)
    O, _, _ = REF.attention(c2, q, 1, [(0, 1)])
    top = (c2.v[t2[0, 0]].double() - 128).abs().max() * c2.v_scale[t2[0, 0]].double().max()
    assert bool(((out.double().view_as(O) - O).abs() <= 1.5 * 2.0 ** -11 * top).all())


@pytest.mark.parametrize("heads,n_q", [(2, 3), (4, 4), (8, 3), (16, 3), (16, 7)])
@pytest.mark.parametrize("page", [16, 64])
def test_a_page_that_a_row_does_not_see(cuda_lib, heads, n_q, page):
    """The newest token lies alone on its page, whose scales are not finite: only its own rows may show it."""
    c = _cache([3 * page + 1, 9 * page + 1], 1, page, seed=heads + n_q + page)
    q, out, lse = _attend(c, [n_q] * 2, heads)
    _check(c, [n_q] * 2, heads, q, out, lse)
    O, _, top = REF.attention(c, q, heads, [(0, n_q), (n_q, n_q)])
    last = c.table.long()[[0, 1], [3, 9]]
    old = [i for i in range(2 * n_q) if i % n_q != n_q - 1]
    for which in ("k_scale", "v_scale"):
        for bad in (float("inf"), float("nan")):
            keep = getattr(c, which).clone()
            getattr(c, which)[last] = bad
            _, out, lse2 = _attend(c, [n_q] * 2, heads, q=q)
            err = (out.double().view(O.shape) - O).abs()[old]
            assert bool((err <= 1.5 * 2.0 ** -11 * top[old][..., None]).all())
            assert bool(((lse2 - lse).abs()[old] <= 2e-4).all())
            getattr(c, which).copy_(keep)


def test_queries_of_extreme_size(cuda_lib):
    c = _cache([100, 100, 100, 100], 1, 16, seed=2)
    c.k_scale *= 1e-30
    q = torch.randn(4, 256, device="cuda")
    q *= torch.tensor([1e30, 1e-30, 0.0, 1e36], device="cuda")[:, None]
    c.k_scale[c.table.long()[3, :7]] *= 1e-6
    q, out, lse = _attend(c, [1] * 4, 2, q=q.to(BF16))
    _check(c, [1] * 4, 2, q, out, lse)


def test_strides_types_and_repeat(cuda_lib):
    from paper_2308_13137_gb300 import serve
    lens, heads = [333, 80, 2500], 8
    c = _cache(lens, 2, 64, seed=3)
    q, ref, lse = _attend(c, [1, 1, 1], heads)
    wide = torch.zeros(3, heads * 128 + 64, dtype=BF16, device="cuda")
    wide[:, 8:8 + heads * 128] = q
    out = torch.full((3, heads * 128 + 32), 5.0, dtype=BF16, device="cuda")
    got = serve.kv_attention(c, wide[:, 8:8 + heads * 128], heads, out=out[:, 16:16 + heads * 128])
    assert torch.equal(got, ref.to(BF16))
    assert bool((out[:, :16] == 5).all()) and bool((out[:, 16 + heads * 128:] == 5).all())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = serve.kv_attention(c, q, heads, out_dtype=F32)
    s.synchronize()
    assert torch.equal(again, ref)


def test_offsets_beyond_32_bits(cuda_lib):
    """Pages more than 4 GB into the pool."""
    from paper_2308_13137_gb300 import serve
    n_pages, G, page = 33000, 8, 128
    new = lambda dt, *s: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
    k, v = new(torch.uint8, n_pages, G, page, 128), new(torch.uint8, n_pages, G, page, 128)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2, 32769]], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    for p in table[0].tolist():
        for t in (k, v):
            t[p] = torch.randint(1, 256, t[p].shape, generator=g, device="cuda").to(torch.uint8)
    c = serve.KVCache(k, v, torch.full((n_pages, G), 0.02, device="cuda"), torch.full((n_pages, G), 0.02, device="cuda"),
                      table, torch.tensor([500], dtype=torch.int32, device="cuda"))
    _check(c, [1], 16, *_attend(c, [1], 16))
    # and a write there: the 500th token lies in page 32769
    qkv = torch.randn(1, (16 + 2 * G) * 128, generator=g, device="cuda")
    serve.kv_append(c, qkv, serve.rope_table(512), 16)
    c.check()
    want = qkv.view(-1, 128)[16 + G:]
    got = (v[32769, :, 499 - 384].float() - 128) * c.v_scale[32769][:, None]
    assert bool(((got - want).abs() <= 0.5001 * c.v_scale[32769][:, None]).all())


def test_page_ids_and_lengths_are_checked(cuda_lib):
    """Out-of-range table entries and lengths set the status word and are not followed."""
    from paper_2308_13137_gb300 import _lib, serve
    rope = serve.rope_table(64)
    for what in ("page", "negative page", "length", "negative length", "rows"):
        c = _cache([40, 40], 2, 16, seed=4)
        if what == "page":
            c.table[1, 1] = c.k.shape[0]
        elif what == "negative page":
            c.table[1, 0] = -1
        elif what == "length":
            c.kv_len[1] = 4000
        elif what == "negative length":
            c.kv_len[1] = -5
        cu = _cu([1, 1])
        if what == "rows":
            cu[2] = 9
        k0, v0 = c.k.clone(), c.v.clone()
        q = torch.randn(2, 4 * 128, device="cuda").to(BF16)
        serve.kv_attention(c, q, 4, cu_q=cu, max_q=1, max_kv=64)
        with pytest.raises(_lib.OmqError):
            c.check()
        c.check()                                        # reported once
        if what in ("length", "negative length", "rows"):
            serve.kv_append(c, torch.randn(2, 8 * 128, device="cuda"), rope, 4, cu_q=cu, max_q=1)
            with pytest.raises(_lib.OmqError):
                c.check()
            p = c.table[1].long().clamp(0, c.k.shape[0] - 1)
            assert torch.equal(c.k[p], k0[p]) and torch.equal(c.v[p], v0[p])


# ------------------------------------------------------------------------------------------------
# the write
# ------------------------------------------------------------------------------------------------

def _append_ref(c, before, qkv, rope, heads, n_q, sa):
    """float64: q, and per sequence the (page, head) scales and the values before rounding."""
    G, page = c.n_kv, c.page
    x = qkv.double().view(-1, heads + 2 * G, 128)
    lens, row, q_all, writes = c.kv_len.tolist(), 0, [], []
    for b, n in enumerate(n_q):
        pos = torch.arange(lens[b] - n, lens[b], device="cuda")
        t = x[row:row + n]
        row += n
        s = sa.double().view(G, 128) if sa is not None else torch.ones(G, 128, dtype=F64, device="cuda")
        q = REF.turned(t[:, :heads], rope, pos).view(n, G, heads // G, 128) / s[:, None]
        q_all.append(q.reshape(n, heads * 128))
        writes.append((pos, REF.turned(t[:, heads:heads + G], rope, pos) * s, t[:, heads + G:]))
    return torch.cat(q_all), writes


@pytest.mark.parametrize("heads,n_kv", LAYOUTS)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append(cuda_lib, heads, n_kv, page, dtype):
    from paper_2308_13137_gb300 import serve
    n_q = [1, 1, 5, 0, page + 3, 2 * page, 1]
    lens = [1, page + 1, page + 2, 40, page + 3, 2 * page + 7, 3 * page]
    c = _cache(lens, n_kv, page, seed=heads + page)
    g = torch.Generator(device="cuda").manual_seed(7)
    qkv = (torch.randn(sum(n_q), (heads + 2 * n_kv) * 128, generator=g, device="cuda") * 3).to(dtype)
    sa = torch.exp(0.3 * torch.randn(n_kv * 128, generator=g, device="cuda"))
    rope = serve.rope_table(max(lens))
    b4 = {n: getattr(c, n).clone() for n in ("k", "v", "k_scale", "v_scale")}
    ko, vo = (torch.empty(sum(n_q), n_kv * 128, dtype=BF16, device="cuda") for _ in range(2))
    q = serve.kv_append(c, qkv, rope, heads, cu_q=_cu(n_q), max_q=max(n_q), sa=sa, k_out=ko, v_out=vo)
    c.check()
    q64, writes = _append_ref(c, b4, qkv, rope, heads, n_q, sa)
    # q: four fp32 roundings of sums of two products (an absolute band), then bf16
    mag = qkv.float().abs().max() * 2 / sa.min()
    assert bool(((q.double() - q64).abs() <= 2.0 ** -8 * q64.abs() + 4 * 2.0 ** -24 * mag).all())
    touched = set()
    row = 0
    for b, (pos, k64, v64) in enumerate(writes):
        for name, val, outv in (("k", k64, ko), ("v", v64, vo)):
            for p in sorted(set((pos // page).tolist())):
                pid = int(c.table[b, p])
                touched.add(pid)
                here = (pos // page) == p
                kept = max(0, int(pos[0]) - p * page)
                old = b4[name + "_scale"][pid].double() if kept else torch.zeros(n_kv, dtype=F64, device="cuda")
                big = val[here].abs().amax((0, 2))
                scale = getattr(c, name + "_scale")[pid].double()
                want = torch.maximum(old, big / 127)
                band = 4 * 2.0 ** -24 * val[here].abs().amax() * 2
                assert bool(((scale - want).abs() <= 2.0 ** -22 * want + band / 127).all())
                # new codes: the nearest integers of value / scale, up to the band of the fp32 value
                slots = (pos[here] - p * page)
                quot = val[here] / scale[None, :, None]
                code = getattr(c, name)[pid][:, slots].permute(1, 0, 2).double() - 128
                err = (code - quot).abs()
                assert bool((err <= 0.5 + 1e-5 + band / scale[None, :, None]).all()) and float(code.abs().max()) <= 127
                got = outv[row:row + len(pos)][here].view(-1, n_kv, 128)
                assert torch.equal(got, (code.float() * scale.float()[None, :, None]).to(BF16))
                # older codes: rounded again where the scale grew, untouched elsewhere
                if kept:
                    o = b4[name][pid][:, :kept].double() - 128
                    n = getattr(c, name)[pid][:, :kept].double() - 128
                    r = torch.where(scale > old, old / scale, torch.ones_like(old))[:, None, None]
                    assert bool(((n - o * r).abs() <= 0.5 + 1e-5).all())
                    same = (scale == old)[:, None, None].expand_as(o)
                    assert torch.equal(n[same], o[same])
                # slots after the last token keep their bytes
                end = int(slots[-1]) + 1
                assert torch.equal(getattr(c, name)[pid][:, end:], b4[name][pid][:, end:])
        row += len(pos)
    rest = torch.tensor([i for i in range(c.k.shape[0]) if i not in touched], device="cuda")
    for n in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(c, n)[rest].nan_to_num(-1), b4[n][rest].nan_to_num(-1)) if n.endswith("scale") else \
            torch.equal(getattr(c, n)[rest], b4[n][rest])


def test_append_without_scale_strided_and_zero_rows(cuda_lib):
    from paper_2308_13137_gb300 import serve
    heads, G = 4, 2
    c = _cache([1, 18], G, 16, seed=1)
    wide = torch.zeros(2, (heads + 2 * G) * 128 + 16, device="cuda")
    wide[1, 8:8 + (heads + 2 * G) * 128] = torch.randn((heads + 2 * G) * 128, device="cuda")
    qo = torch.full((2, heads * 128 + 8), 3.0, dtype=BF16, device="cuda")
    rope = serve.rope_table(32)
    serve.kv_append(c, wide[:, 8:8 + (heads + 2 * G) * 128], rope, heads, q_out=qo[:, :heads * 128])
    c.check()
    p0 = int(c.table[0, 0])
    assert bool((c.k[p0, :, 0] == 128).all()) and bool((c.k_scale[p0] == 0).all())      # a zero token: zero scale
    assert bool((qo[:, heads * 128:] == 3).all()) and bool((qo[0, :heads * 128] == 0).all())
    want = REF.turned(wide[1:, 8:8 + heads * 128].double().view(1, heads, 128), rope, torch.tensor([17], device="cuda"))
    assert bool(((qo[1, :heads * 128].double() - want.view(-1)).abs() <= 2.0 ** -8 * want.view(-1).abs() + 1e-5).all())


def test_rope_table(cuda_lib):
    from paper_2308_13137_gb300 import serve
    t = serve.rope_table(70000).double()
    ang = torch.arange(70000, dtype=F64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, 128, 2, dtype=F64, device="cuda") / 128)
    assert float((t[..., 0] - ang.cos()).abs().max()) < 3e-7 and float((t[..., 1] - ang.sin()).abs().max()) < 3e-7


def test_written_one_by_one_then_read(cuda_lib):
    """Tokens appended one at a time and attended to: the cache holds each within its page's rounding."""
    from paper_2308_13137_gb300 import serve
    heads, G, page, n = 4, 2, 16, 40
    c = serve.KVCache.empty(8, G, page, 1, 4)
    c.table.copy_(torch.tensor([[5, 2, 7, 0]], dtype=torch.int32))
    rope = serve.rope_table(64)
    g = torch.Generator(device="cuda").manual_seed(2)
    qkv = torch.randn(n, (heads + 2 * G) * 128, generator=g, device="cuda")
    for i in range(n):
        c.kv_len.fill_(i + 1)
        q = serve.kv_append(c, qkv[i:i + 1], rope, heads)
        out = serve.kv_attention(c, q, heads, out_dtype=F32)
    c.check()
    v = REF.dequant(c, "v", 0, n)
    want = qkv.double().view(n, -1, 128)[:, heads + G:]
    # half a step when written, and half a step more at each of the later growths of its page's scale
    grown = 16
    for p in range(3):
        rows = slice(p * page, min(n, (p + 1) * page))
        step = c.v_scale[c.table.long()[0, p]].double()[None, :, None]
        assert bool(((v[rows] - want[rows]).abs() <= step * (0.5 + 0.5 * grown)).all())
        assert float(((v[rows] - want[rows]) / step).square().mean().sqrt()) < 1.0
    O, _, top = REF.attention(c, q, heads, [(0, 1)])
    assert bool(((out.double().view_as(O) - O).abs() <= 1.5 * 2.0 ** -11 * top[..., None]).all())
    assert math.isfinite(float(out.sum()))
