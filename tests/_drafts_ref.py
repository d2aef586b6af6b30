"""Plain forms of the operators that check drafted tokens, in float64 (and the kept codes in their stated order of
fp32 roundings), for the tests."""
import math

import numpy as np
import torch

import _serve_ref as REF

F64 = torch.float64


def random_tree(n, r, depth=6, width=4):
    """Parents of n nodes in an order that is not level by level."""
    parent, d, kids = [-1], [0], [0]
    while len(parent) < n:
        ok = [i for i in range(len(parent)) if d[i] < depth and kids[i] < width] or [len(parent) - 1]
        p = int(ok[r.randint(len(ok))])
        kids[p] += 1
        parent.append(p)
        d.append(d[p] + 1)
        kids.append(0)
    return parent[:n]


def ancestors(parent):
    """[n, n] truth values: j is i or above it."""
    m = np.zeros((len(parent), len(parent)), bool)
    for i, p in enumerate(parent):
        if p >= 0:
            m[i] = m[p]
        m[i, i] = True
    return m


def words_of(m, words):
    """Truth values [n, k] as int32 words [n, words]."""
    full = np.zeros((m.shape[0], words * 32), bool)
    full[:, :m.shape[1]] = m
    return np.packbits(full.reshape(len(m), words, 32), axis=-1, bitorder="little").view(np.int32).reshape(len(m), words)


def attention(cache, q, n_heads, rows, masks):
    """masks: per sequence [n, n] truth values over its newest tokens.  O, lse (base 2) and, per (row, head), the largest
    |v| that the row sees."""
    G, rep = cache.n_kv, n_heads // cache.n_kv
    O = torch.zeros(q.shape[0], n_heads, 128, dtype=F64, device=q.device)
    lse = torch.full((q.shape[0], n_heads), -math.inf, dtype=F64, device=q.device)
    top = torch.zeros(q.shape[0], n_heads, dtype=F64, device=q.device)
    kv = cache.kv_len.tolist()
    for b, (r0, n) in enumerate(rows):
        L = kv[b]
        if L == 0 or n == 0:
            continue
        seen = torch.zeros(n, L, dtype=torch.bool, device=q.device)
        start = L - n
        m = torch.as_tensor(masks[b], device=q.device)
        seen[:, :max(0, start)] = True
        seen[:, max(0, start):] = m[:, max(0, -start):]
        k, v = REF.dequant(cache, "k", b, L), REF.dequant(cache, "v", b, L)
        for g in range(G):
            h = slice(g * rep, (g + 1) * rep)
            s = torch.einsum("nrd,ld->nrl", q[r0:r0 + n].double().view(n, n_heads, 128)[:, h], k[:, g]) / math.sqrt(128)
            s = s.masked_fill(~seen[:, None], -math.inf)
            some = seen.any(1)
            lse[r0:r0 + n, h] = torch.logsumexp(s, -1) / math.log(2)
            p = torch.softmax(s, -1).masked_fill(~seen[:, None], 0)
            vg = v[:, g]
            o = torch.zeros(n, rep, 128, dtype=F64, device=q.device)
            for i in range(n):
                if some[i]:
                    o[i] = p[i][:, seen[i]] @ vg[seen[i]]
                    top[r0 + i, h] = vg[seen[i]].abs().max()
            O[r0:r0 + n, h] = o
    return O, lse, top


def clean(p):
    p = p.double()
    return torch.where(torch.isnan(p), torch.zeros_like(p), p).clamp(0, 1)


def verify(parent, tokens, P, Q, u, steps):
    """One sequence: (path, emitted tokens), by the residual distribution itself, normalised after every rejection."""
    V = P.shape[1]
    num = [min(max(0.0 if math.isnan(x) else x, 0.0), 0.99999994) for x in u]
    node, path, out = 0, [0], []
    while True:
        p = clean(P[node])
        r, q = p, (clean(Q[node]) if Q is not None else None)
        nxt = None
        if len(path) < steps:
            for i in range(node + 1, len(parent)):
                if parent[i] != node or not 0 <= tokens[i] < V:
                    continue
                x = tokens[i]
                if num[i] * (float(q[x]) if q is not None else 1.0) < float(r[x]):
                    nxt = i
                    break
                if q is not None:
                    r = (r - q).clamp_min(0)
                    r = r / r.sum() if float(r.sum()) > 0 else r
                else:
                    left = 1.0 - float(r[x])
                    r = r.clone()
                    r[x] = 0
                    r = r / left if left > 0 else r
        if nxt is not None:
            out.append(tokens[nxt])
            path.append(nxt)
            node = nxt
            continue
        if float(r.sum()) == 0:
            r = p
        c = r.cumsum(0)
        over = torch.nonzero(c > num[0] * c[-1])
        out.append(int(over[0]) if len(over) else 0)
        return path, out


def keep(cache, start, path, b):
    """One sequence's accepted rows moved, in the order of fp32 roundings that omq_kv_keep states.  Changes the cache."""
    P, table = cache.page, cache.table[b].tolist()
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        old_codes, old_scale = codes.clone(), scale.clone()
        by_page = {}
        for j, p in enumerate(path):
            by_page.setdefault((start + j) // P, []).append((start + j, start + p))
        for pg, moves in by_page.items():
            if all(to == fro for to, fro in moves):
                continue
            d = table[pg]
            before = old_scale[d]
            want = torch.zeros_like(before)
            for to, fro in moves:
                if fro // P != pg:
                    s = table[fro // P]
                    top = (old_codes[s, :, fro % P].float() - 128).abs().amax(-1)
                    want = torch.maximum(want, (top * old_scale[s]) / torch.full_like(before, 127.0))
            after = torch.maximum(before, want)
            grown = (after > before)[:, None, None]
            again = torch.round((old_codes[d].float() - 128) * (before / after)[:, None, None]).clamp(-127, 127) + 128
            new = torch.where(grown, again, old_codes[d].float())
            for to, fro in moves:
                if to == fro:
                    continue
                s = table[fro // P]
                r = torch.where(after > 0, old_scale[s] / after, torch.zeros_like(after))
                new[:, to % P] = torch.round((old_codes[s, :, fro % P].float() - 128) * r[:, None]).clamp(-127, 127) + 128
            codes[d] = new.to(torch.uint8)
            scale[d] = after
