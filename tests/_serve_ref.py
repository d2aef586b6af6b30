"""Plain float64 forms of the 8-bit serving operators, for the tests."""
import math

import torch

F64 = torch.float64
HD = 128


def norm_rows(x, r, gain, bias, eps):
    t = x.double() + (r.double() if r is not None else 0)
    y = t / (t.square().mean(1, keepdim=True) + eps).sqrt()
    if gain is not None:
        y = y * gain.double()
    return t, y + (bias.double() if bias is not None else 0)


def int_product(a, za, w, zw):
    """Exact integer sums (float64 holds them: below 2^53)."""
    za = 128 if za is None else za.double()[:, None]
    zw = 128 if zw is None else zw.double()[:, None]
    return (a.double() - za) @ (w.double() - zw).t()


def turned(x, rope, pos):
    """Rotate-half pairs (i, i + 64) of x [n, heads, 128] at pos [n]."""
    cs = rope.double()[pos][:, None]
    a, b = x[..., :64], x[..., 64:]
    return torch.cat([a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]], -1)


def pages_of(cache, b, length):
    n = -(-length // cache.page)
    return cache.table[b, :n].long()


def dequant(cache, name, b, length):
    """Values [length, n_kv, 128] of one sequence."""
    p = pages_of(cache, b, length)
    v = (getattr(cache, name)[p].double() - 128) * getattr(cache, name + "_scale")[p].double()[..., None, None]
    return v.permute(0, 2, 1, 3).reshape(-1, cache.n_kv, HD)[:length]


def attention(cache, q, n_heads, rows):
    """rows: per sequence (first row, number of rows).  Returns O, lse (base 2) and, per (row, head), the
    largest |v| that the row sees."""
    G = cache.n_kv
    rep = n_heads // G
    O = torch.zeros(q.shape[0], n_heads, HD, dtype=F64, device=q.device)
    lse = torch.full((q.shape[0], n_heads), -math.inf, dtype=F64, device=q.device)
    top = torch.zeros(q.shape[0], n_heads, dtype=F64, device=q.device)
    kv = cache.kv_len.tolist()
    for b, (r0, n) in enumerate(rows):
        L = kv[b]
        if L == 0 or n == 0:
            continue
        k, v = dequant(cache, "k", b, L), dequant(cache, "v", b, L)
        k, v = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
        for i in range(n):
            seen = L - n + i + 1
            if seen <= 0:
                continue
            s = torch.einsum("hd,lhd->hl", q[r0 + i].double().view(n_heads, HD), k[:seen]) / math.sqrt(HD)
            lse[r0 + i] = torch.logsumexp(s, 1) / math.log(2)
            O[r0 + i] = torch.einsum("hl,lhd->hd", torch.softmax(s, 1), v[:seen])
            top[r0 + i] = v[:seen].abs().amax((0, 2))
    return O, lse, top
