"""The operators that check drafted tokens over the 8-bit cache, over the sizes that they meet.

* ``tree``    parents of drafted tokens to depths and to the bits of what each sees (``draft_tree``).
* ``append``  the cache write of the drafted rows at their depths' positions (``kv_append`` with a tree).
* ``attend``  attention of every drafted row over the context and its own ancestors (``kv_attention`` with
              a tree).
* ``verify``  the walk through the tree: drafted tokens against the target's probabilities, from given random
              numbers, and the new token (``verify_drafts``).
* ``keep``    the accepted path to the front of the drafted tokens, in every layer's cache (``kv_keep``).

``run`` computes an operator in elementary torch operations (``own`` false) or through the package's
entry points (``own`` true), from the same prepared state.  Heads are those of the LLaMA-7B (32) and LLaMA-2-70B
(64 query, 8 KV) blocks of this repository, trees of one token to a thousand, vocabularies generic.
"""
import math

import numpy as np
import torch

own = False

HD = 128                       # head dimension
THETA = 10000.0
I32, F32, F64, BF16 = torch.int32, torch.float32, torch.float64, torch.bfloat16


def listed():
    return [
        # the tree of one sequence, made anew at every step: latency
        dict(name="tree_1x26", op="tree", B=1, nq=26, ragged=False, depth=5),
        # a large batch of wide trees
        dict(name="tree_384x509", op="tree", B=384, nq=509, ragged=True, depth=9),
        # one sequence of the 7B block
        dict(name="append_1x26", op="append", B=1, nq=26, ragged=False, depth=5, heads=32, kv=32, kv_max=2048, page=64,
             x="f32"),
        # a serving batch at 70B heads, trees of unequal size
        dict(name="append_64_ragged", op="append", B=64, nq=61, ragged=True, depth=7, heads=64, kv=8, kv_max=4099, page=32,
             x="f32"),
        # one sequence of the 7B block, a few drafts: latency
        dict(name="attend_1x9", op="attend", B=1, nq=9, ragged=False, depth=4, heads=32, kv=32, kv_max=2048, page=64),
        # a serving batch at 70B heads, small trees, ragged contexts, a sequence that has only its tree
        dict(name="attend_64x13_ragged", op="attend", B=64, nq=13, ragged=True, depth=5, heads=64, kv=8, kv_max=4099, page=32,
             fresh=True),
        # wide trees at 70B heads: 512 rows on every KV head
        dict(name="attend_16x64", op="attend", B=16, nq=64, ragged=False, depth=8, heads=64, kv=8, kv_max=8192, page=64),
        # very long contexts at 70B heads, short chains: the cache read is everything
        dict(name="attend_4x4_131072", op="attend", B=4, nq=4, ragged=False, depth=4, heads=64, kv=8, kv_max=131072, page=64),
        # one sequence's tree of drawn tokens
        dict(name="verify_1x26", op="verify", B=1, nq=26, ragged=False, depth=5, V=32000, p="f32", drawn=True),
        # a serving batch, a large vocabulary
        dict(name="verify_64x15_ragged", op="verify", B=64, nq=15, ragged=True, depth=6, V=128256, p="f32", drawn=True),
        # one sequence, every layer of the 7B model
        dict(name="keep_1x26", op="keep", B=1, nq=26, ragged=False, depth=5, kv=32, kv_max=500, page=64, layers=32),
        # a serving batch at 70B heads, as many layers as lie on one GPU of a few
        dict(name="keep_64_ragged", op="keep", B=64, nq=61, ragged=True, depth=7, kv=8, kv_max=300, page=32, layers=40),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "append", "attend", "attend", "verify", "verify", "keep"])
    depth = rng.randint(1, 12)
    if op == "tree":
        nq = _log(rng, 16, 1024)                        # (smaller ones have hardly any trees but one)
        return dict(op=op, B=min(_log(rng, 1, 384), max(1, 384 * 509 // nq)), nq=nq, ragged=rng.random() < 0.5,
                    depth=_log(rng, 3, max(3, min(nq // 3, 200))))
    if op == "verify":
        V = _log(rng, 500, 160000)
        nq = _log(rng, 1, 64)
        B = min(_log(rng, 1, 64), max(1, 64 * 15 * 128256 // (nq * V)))
        return dict(op=op, B=B, nq=nq, ragged=rng.random() < 0.5, depth=depth, V=V, p=rng.choice(["f32", "f32", "bf16"]),
                    drawn=rng.random() < 0.6)
    kv = rng.choice([1, 2, 4, 8, 32, 40])
    heads = kv * (rng.choice([1, 2, 3, 4, 7, 8]) if kv <= 8 else 1)
    page = rng.choice([16, 32, 64, 128])
    nq = _log(rng, 1, 128)
    if op == "append":
        B = min(_log(rng, 1, 64), max(1, 64 * 61 * 80 // (nq * (heads + 2 * kv))))
        top = max(nq + 1, min(_log(rng, 64, 4096), 64 * 4099 * 8 // (B * kv)))
        return dict(op=op, B=B, nq=nq, ragged=rng.random() < 0.5, depth=depth, heads=heads, kv=kv, kv_max=top, page=page,
                    x=rng.choice(["f32", "bf16"]))
    if op == "keep":
        layers = rng.choice([1, 1, 4, 32, 70])
        B = min(_log(rng, 1, 64), max(1, 64 * 8 * 40 // (kv * layers)))
        return dict(op=op, B=B, nq=nq, ragged=rng.random() < 0.5, depth=depth, kv=kv, kv_max=nq + rng.randint(0, 200), page=page,
                    layers=layers)
    B = _log(rng, 1, 96)
    rows = nq * heads // kv
    most = min(4 * 131072 * 8 // (B * kv), 16 * 8192 * 8 * 512 // (B * kv * max(16, rows)))
    top = max(nq, _log(rng, 16, min(131072, max(64, most))))
    return dict(op=op, B=B, nq=nq, ragged=rng.random() < 0.5, depth=depth, heads=heads, kv=kv, kv_max=top, page=page,
                fresh=rng.random() < 0.3)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

_DT = {"f32": F32, "bf16": BF16}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _dev(a, dt=None):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dt)


def _lengths(c, seed):
    """Tokens in the cache (the drafted ones among them) and drafted rows of every sequence.  The case alone
    gives the lengths, so that every seed has the same shapes; the seed gives their order."""
    B, nq, top = c["B"], c["nq"], c.get("kv_max", c["nq"])
    r = np.random.RandomState(B * 7 + nq * 1009 + top)
    q = r.randint(1, nq + 1, B) if c["ragged"] else np.full(B, nq)
    q[0] = nq
    kv = np.maximum(r.randint(max(1, top // 4), top + 1, B), q)
    kv[0] = max(top, nq)
    if c.get("fresh") and B > 1:
        kv[1] = q[1]                                    # no context: its first row sees only itself
    order = np.random.RandomState(int(seed) % (1 << 31)).permutation(B)
    return kv[order].astype(np.int32), q[order].astype(np.int32)


def _tree(n, depth, r):
    """Parents of n nodes, level by level: a root, then every level's nodes under random nodes of the level
    before, mostly under its first ones (the likelier drafts)."""
    parent, level, at = [-1], [0], 1
    left = min(depth, n - 1)
    while at < n:
        width = n - at if left <= 1 else max(1, min(n - at - (left - 1), int(round((n - at) / left * r.uniform(0.5, 1.5)))))
        pick = np.sort((np.array(level)[(r.rand(width) ** 2 * len(level)).astype(int)]))
        parent += pick.tolist()
        level = list(range(at, at + width))
        at += width
        left -= 1
    return np.array(parent, np.int32)


def _plan(c, q, seed):
    """The trees of a step, packed: parents, depths and the ancestor bits, as the package lays them out."""
    r = np.random.RandomState((int(seed) + 11) % (1 << 31))
    first = np.cumsum(q) - q
    parent = np.concatenate([_tree(int(n), c["depth"], r) for n in q])
    depth, bits = np.full(len(parent), -1, np.int32), np.zeros((len(parent), (int(q.max()) + 31) // 32), np.uint32)
    base, at = np.repeat(first, q), np.arange(len(parent)) - np.repeat(first, q)
    rows = np.arange(len(parent))                       # every row's walk to its root, all rows together
    while len(rows):
        bits[rows, at // 32] |= np.left_shift(np.uint32(1), (at % 32).astype(np.uint32))
        depth[rows] += 1
        at = parent[base[rows] + at]
        rows, at = rows[at >= 0], at[at >= 0]
    return parent, depth, bits.view(np.int32)


def _pool(c, g, kv, seed, layers=1):
    """Page pools of 8-bit caches: codes of bell-shaped values, scales that differ by page and head."""
    page, need = c["page"], [max(1, -(-int(n) // c["page"])) for n in kv]
    n_pages = sum(need) + 3
    order = np.random.RandomState((int(seed) + 5) % (1 << 31)).permutation(n_pages)
    table = np.full((len(kv), max(need)), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (layers, n_pages, c["kv"], page, HD)

    def codes():
        out = torch.empty(shape, dtype=torch.uint8, device="cuda")
        for part in out.view(-1, *shape[2:]).split(4096):           # bounded scratch for the large pools
            part.copy_((_randn(g, *part.shape) * 30 + 128).round_().clamp_(1, 255))
        return out

    s = dict(table=_dev(table), kv_len=_dev(kv))
    s["pools"] = dict(k=codes(), v=codes(), k_scale=torch.exp(0.3 * _randn(g, layers, n_pages, c["kv"])) / 30,
                      v_scale=torch.exp(0.5 * _randn(g, layers, n_pages, c["kv"])) / 30)
    s["layers"] = [{k: t[i] for k, t in s["pools"].items()} for i in range(layers)]
    return s


def _rope(n):
    ang = torch.arange(n, dtype=F64, device="cuda")[:, None] * \
        THETA ** (-torch.arange(0, HD, 2, dtype=F64, device="cuda") / HD)
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()      # [n, 64, 2]


def _accepted(parent, steps, r, room):
    """A path from the root as a verification leaves it: mostly a few nodes.  Its nodes lie behind the places
    that they move to (or on them), and those in one page, so that the move can be repeated."""
    steps = min(steps, room)
    for _ in range(64):
        path = [0]
        while len(path) < steps and r.rand() < 0.75:
            kids = np.flatnonzero(parent == path[-1])
            if len(kids) == 0:
                break
            path.append(int(kids[min(len(kids) - 1, r.geometric(0.5) - 1)]))
        if all(p == j or p >= len(path) for j, p in enumerate(path)):
            return path
    return [0]


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    kv, q = _lengths(c, seed)
    cu = np.concatenate([[0], np.cumsum(q)]).astype(np.int32)
    s = dict(case=c, total=int(q.sum()), max_q=int(q.max()), max_kv=max(1, int(kv.max())), cu=_dev(cu), q_len=_dev(q))
    parent, depth, seen = _plan(c, q, seed)
    s["parent"], s["depth"], s["seen"] = _dev(parent), _dev(depth), _dev(seen)
    s["steps"] = int(depth.max()) + 1
    s["seq"] = _dev(np.repeat(np.arange(len(q)), q))                              # row -> sequence
    s["at"] = _dev(np.concatenate([np.arange(n) for n in q]))                     # row -> its place in it
    total = s["total"]
    new = lambda dt, *shape: torch.empty(*shape, dtype=dt, device="cuda")  # noqa: E731
    if c["op"] == "tree":
        s["out"] = dict(depth=new(I32, total), seen=new(I32, total, seen.shape[1]))
    elif c["op"] == "verify":
        _drafts(s, c, g, q, parent)
        B = len(q)
        s["out"] = dict(tokens=new(I32, B, s["steps"]), path=new(I32, B, s["steps"]), count=new(I32, B))
    elif c["op"] == "keep":
        s.update(_pool(c, g, kv, seed, c["layers"]))
        r = np.random.RandomState((int(seed) + 23) % (1 << 31))
        path, count = np.full((len(q), s["steps"]), -1, np.int32), np.zeros(len(q), np.int32)
        for b in range(len(q)):
            p = _accepted(parent[cu[b]:cu[b + 1]], s["steps"], r, c["page"] - int(kv[b] - q[b]) % c["page"])
            path[b, :len(p)], count[b] = p, len(p)
        s["path"], s["count"] = _dev(path), _dev(count)
    else:
        s.update(_pool(c, g, kv, seed))
        if c["op"] == "append":
            s["qkv"] = _randn(g, total, (c["heads"] + 2 * c["kv"]) * HD).to(_DT[c["x"]])
            s["rope"] = _rope(s["max_kv"])
            s["sa"] = torch.exp(0.1 * _randn(g, c["kv"] * HD))
            s["out"] = dict(q=new(BF16, total, c["heads"] * HD), k_new=new(BF16, total, c["kv"] * HD),
                            v_new=new(BF16, total, c["kv"] * HD))
        else:
            s["q"] = _randn(g, total, c["heads"] * HD).to(BF16)
            s["out"] = dict(o=new(BF16, total, c["heads"] * HD), lse=new(F32, total, c["heads"]))
    return s


def _drafts(s, c, g, q, parent):
    """Target and draft distributions of every row (bell-shaped scores a few units wide, the draft's near the
    target's), and the drafted tokens: drawn from the draft's distribution at the parent, or its most likely ones."""
    total, V = s["total"], c["V"]
    up = parent.astype(np.int64) + np.repeat(np.cumsum(q) - q, q)            # row of the parent (roots: themselves)
    up = np.where(parent < 0, np.arange(total), up)
    rank = np.zeros(total, np.int64)                                         # among its siblings
    for i in range(1, total):
        if parent[i] >= 0 and up[i] == up[i - 1] and parent[i - 1] >= 0:
            rank[i] = rank[i - 1] + 1
    s["probs"], s["q"] = torch.empty(total, V, dtype=_DT[c["p"]], device="cuda"), None
    draft = torch.empty(total, V, dtype=_DT[c["p"]], device="cuda")
    for i in range(0, total, 64):
        z = 2.5 * _randn(g, min(64, total - i), V)
        s["probs"][i:i + 64] = torch.softmax(z, -1)
        draft[i:i + 64] = torch.softmax(z + 0.7 * _randn(g, *z.shape), -1)
    up, tokens = _dev(up), torch.empty(total, dtype=I32, device="cuda")
    if c["drawn"]:
        s["q"] = draft
        at = torch.rand(total, generator=g, device="cuda", dtype=F64)
        for i in range(0, total, 64):
            cum = draft[up[i:i + 64]].double().cumsum(-1)
            tokens[i:i + 64] = (cum > at[i:i + 64, None] * cum[:, -1:]).to(torch.uint8).argmax(-1).to(I32)
    else:
        rank = _dev(rank)
        wide = min(V, int(rank.max()) + 1)
        for i in range(0, total, 64):
            top = draft[up[i:i + 64]].float().topk(wide, -1).indices
            tokens[i:i + 64] = top.gather(1, rank[i:i + 64, None].clamp_max(wide - 1))[:, 0].to(I32)
    s["tokens"] = tokens
    s["u"] = torch.rand(total, generator=g, device="cuda")


# ------------------------------------------------------------------------------------------------
# the package's entry points
# ------------------------------------------------------------------------------------------------

def _handles(s):
    """The plan and the cache handles, made once as a serving loop makes them."""
    from paper_2308_13137_gb300 import serve
    if "tree" not in s:
        s["tree"] = serve.DraftTree(s["parent"], s["depth"], s["seen"], s["cu"], s["max_q"])
        s["caches"] = [serve.KVCache(y["k"], y["v"], y["k_scale"], y["v_scale"], s["table"], s["kv_len"])
                       for y in s.get("layers", ())]
    return serve, s["tree"], s["caches"]


def _own_tree(s):
    from paper_2308_13137_gb300 import serve
    o = s["out"]
    serve.draft_tree(s["parent"], s["cu"], s["max_q"], out=serve.DraftTree(s["parent"], o["depth"], o["seen"], s["cu"], s["max_q"]))
    return o


def _own_append(s):
    serve, tree, (cache,) = _handles(s)
    o = s["out"]
    serve.kv_append(cache, s["qkv"], s["rope"], s["case"]["heads"], tree=tree, sa=s["sa"], q_out=o["q"], k_out=o["k_new"],
                    v_out=o["v_new"])
    return dict(o, **s["layers"][0])


def _own_attend(s):
    serve, tree, (cache,) = _handles(s)
    o = s["out"]
    serve.kv_attention(cache, s["q"], s["case"]["heads"], tree=tree, max_kv=s["max_kv"], out=o["o"], lse=o["lse"])
    return o


def _own_verify(s):
    serve, tree, _ = _handles(s)
    o = s["out"]
    serve.verify_drafts(tree, s["tokens"], s["probs"], s["u"], draft_probs=s["q"], out=serve.Verified(**o))
    return o


def _own_keep(s):
    serve, tree, caches = _handles(s)
    serve.kv_keep(caches, tree, s["path"], s["count"])
    return s["pools"]


# ------------------------------------------------------------------------------------------------
# plain forms, 32 bits (64 where a comparison decides)
# ------------------------------------------------------------------------------------------------

def _parent_rows(s):
    """Row of every row's parent, -1 at a root."""
    first = (s["cu"][:-1])[s["seq"]].long()
    return torch.where(s["parent"] < 0, torch.full_like(first, -1), first + s["parent"].long())


def _plain_tree(s):
    """Every node takes its parent's bits, one level of the tree after another."""
    words = s["out"]["seen"].shape[1]
    at, up = s["at"].long(), _parent_rows(s)
    hop, root = up.clamp_min(0), up < 0
    mine = torch.zeros(s["total"], words, dtype=torch.int64, device="cuda")
    mine.scatter_(1, (at // 32)[:, None], (torch.ones_like(at) << (at % 32))[:, None])
    seen, depth = mine.clone(), torch.zeros_like(at)
    for _ in range(s["steps"] - 1):
        seen = mine | torch.where(root[:, None], torch.zeros_like(mine), seen[hop])
        depth = torch.where(root, torch.zeros_like(at), depth[hop] + 1)
    return dict(depth=depth.to(I32), seen=seen.to(I32))


def _plain_append(s):
    c = s["case"]
    H, G, page = c["heads"], c["kv"], c["page"]
    x = s["qkv"].float().view(s["total"], H + 2 * G, HD)
    start = (s["kv_len"] - s["q_len"])[s["seq"]].long()
    slot = start + s["at"]
    cs = s["rope"][start + s["depth"].long()]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]

    def turn(t):
        a, b = t[..., :64], t[..., 64:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    sa = s["sa"].view(G, HD)
    q = turn(x[:, :H]).view(-1, G, H // G, HD) / sa[:, None]
    k, v = turn(x[:, H:H + G]) * sa, x[:, H + G:]
    page_at = s["table"][s["seq"], slot // page].long()
    # the pages that this call writes, and the tokens that each held before it (none in one it starts)
    pages, where = torch.unique(page_at, return_inverse=True)
    kept = torch.zeros_like(pages)
    kept[where] = (start - slot // page * page).clamp(0, page)
    out = dict(q=q.reshape(s["total"], -1).to(BF16))
    y = s["layers"][0]
    top = torch.full((), 127.0, device="cuda")          # a tensor: division by a number multiplies by its reciprocal
    for name, val in (("k", k), ("v", v)):
        codes, scale = y[name], y[name + "_scale"]
        held = codes[pages]
        big = torch.zeros(len(pages), G, device="cuda")
        big.index_reduce_(0, where, val.abs().amax(-1), "amax")
        before = torch.where((kept > 0)[:, None], scale[pages], torch.zeros_like(big))
        after = torch.maximum(before, big / top)
        # tokens already in a page whose scale grows are rounded again to the new scale
        grown = (after > before)[:, :, None, None] & (torch.arange(page, device="cuda") < kept[:, None])[:, None, :, None]
        again = torch.round((held.float() - 128) * (before / after)[..., None, None]) + 128
        held = torch.where(grown, again, held.float()).to(torch.uint8)
        sc = after[where][..., None]
        new = torch.where(sc > 0, torch.round(val / sc), torch.zeros_like(val)).clamp(-127, 127)
        held[where, :, slot % page] = (new + 128).to(torch.uint8)
        codes[pages], scale[pages] = held, after
        out[name + "_new"] = (new * sc).reshape(s["total"], -1).to(BF16)
    return dict(out, **y)


def _plain_attend(s):
    """Over the gathered, dequantised pages; softmax base 2 as the package's lse."""
    c, y = s["case"], s["layers"][0]
    G, R = c["kv"], c["heads"] // c["kv"]
    B, n, L = c["B"], s["max_q"], s["table"].shape[1] * c["page"]
    tab = s["table"].clamp_min(0).long()

    def gather(name):
        t = (y[name][tab].float() - 128) * y[name + "_scale"][tab][..., None, None]          # [B, pages, G, page, HD]
        return t.permute(0, 2, 1, 3, 4).reshape(B, G, L, HD)

    q = torch.zeros(B, n, c["heads"] * HD, device="cuda")
    q[s["seq"], s["at"]] = s["q"].float()
    q = q.view(B, n, G, R, HD).permute(0, 2, 1, 3, 4).reshape(B, G, -1, HD)                  # [B, G, n R, HD]
    sc = (q @ gather("k").transpose(-1, -2)) * (math.log2(math.e) / math.sqrt(HD))
    bits = torch.zeros(B, n, s["seen"].shape[1], dtype=I32, device="cuda")
    bits[s["seq"], s["at"]] = s["seen"]
    start = (s["kv_len"] - s["q_len"]).long()
    node = torch.arange(L, device="cuda") - start[:, None]                                   # [B, L] place in the tree
    inside = (node >= 0) & (node < s["q_len"][:, None])
    at = node.clamp(0, n - 1)
    word = bits.gather(2, (at // 32)[:, None].expand(B, n, L))
    seen = ((word >> (at % 32)[:, None]) & 1).bool() & inside[:, None]
    seen |= (torch.arange(L, device="cuda") < start[:, None])[:, None]
    sc = torch.where(seen.repeat_interleave(R, 1)[:, None], sc, torch.full_like(sc, -math.inf))
    m = sc.amax(-1, keepdim=True)
    p = torch.exp2(sc - torch.where(m > -math.inf, m, torch.zeros_like(m)))
    l = p.sum(-1, keepdim=True)
    o = (p @ gather("v")) / torch.where(l > 0, l, torch.ones_like(l))
    lse = m + torch.log2(l)

    def rows(t, w):
        t = t.view(B, G, -1, R, w).permute(0, 2, 1, 3, 4).reshape(B, -1, G * R * w)
        return t[s["seq"], s["at"]]

    return dict(o=rows(o, HD).to(BF16), lse=rows(lse, 1))


def _plain_verify(s):
    """All sequences together, one drafted row after another in row order (children lie behind their parents):
    a sequence that has come to the row's parent tests it.  p - a q holds the residual of the rejected ones."""
    B = s["case"]["B"]
    first, n_rows = s["cu"][:-1].long(), s["q_len"].long()
    P, Q = s["probs"], s["q"]
    seqs = torch.arange(B, device="cuda")
    cur, count = torch.zeros(B, dtype=torch.int64, device="cuda"), torch.ones(B, dtype=torch.int64, device="cuda")
    a, T = torch.zeros(B, dtype=F64, device="cuda"), torch.ones(B, dtype=F64, device="cuda")
    steps = s["steps"]
    path = torch.full((B, steps + 1), -1, dtype=torch.int64, device="cuda")
    tokens = path.clone()
    path[:, 0] = 0
    weight = P[first].double()                           # [B, V]: what the new token would be drawn from here
    base = weight
    q_here = Q[first].double() if Q is not None else None
    for i in range(1, s["max_q"]):
        row = (first + i).clamp_max(s["total"] - 1)
        here = (i < n_rows) & (s["parent"][row].long() == cur)
        x = s["tokens"][row].long()
        u = s["u"][row].double()
        rx = weight[seqs, x]
        qx = q_here[seqs, x] if Q is not None else torch.ones_like(rx)
        ok = here & (u * T * qx < rx)
        no = here & ~ok
        # the accepted move on
        cur = torch.where(ok, torch.full_like(cur, i), cur)
        path[seqs, torch.where(ok, count, torch.full_like(count, steps))] = i
        tokens[seqs, torch.where(ok, count - 1, torch.full_like(count, steps))] = x
        count = count + ok.long()
        # the rejected take the drafted part out
        if Q is not None:
            a = torch.where(no, a + T, torch.where(ok, torch.zeros_like(a), a))
            base = torch.where(ok[:, None], P[row].double(), base)
            q_here = torch.where(ok[:, None], Q[row].double(), q_here)
            weight = torch.where((no | ok)[:, None], (base - a[:, None] * q_here).clamp_min(0), weight)
            T = torch.where(no, weight.sum(-1), T)
        else:
            T = torch.where(no, T - rx, T)
            weight = weight.scatter(1, x[:, None], torch.where(no, torch.zeros_like(rx), rx)[:, None])
            weight = torch.where(ok[:, None], P[row].double(), weight)
        T = torch.where(ok, torch.ones_like(T), T)
    cum = weight.cumsum(-1)
    new = (cum > s["u"][first].double()[:, None] * cum[:, -1:]).to(torch.uint8).argmax(-1)
    tokens[seqs, count - 1] = new
    path, tokens = path[:, :steps], tokens[:, :steps]
    past = torch.arange(steps, device="cuda") >= count[:, None]
    return dict(tokens=tokens.masked_fill(past, -1).to(I32), path=path.masked_fill(past, -1).to(I32), count=count.to(I32))


def _plain_keep(s):
    c = s["case"]
    page, G = c["page"], c["kv"]
    steps = s["steps"]
    start = (s["kv_len"] - s["q_len"]).long()
    to = start[:, None] + torch.arange(steps, device="cuda")
    fro = start[:, None] + s["path"].long()
    live = torch.arange(steps, device="cuda") < s["count"][:, None]
    seq = torch.arange(c["B"], device="cuda")[:, None].expand_as(to)[live]
    to, fro = to[live], fro[live]
    to_page, from_page = s["table"][seq, to // page].long(), s["table"][seq, fro // page].long()
    pages, where = torch.unique(to_page, return_inverse=True)
    top = torch.full((), 127.0, device="cuda")
    for y in s["layers"]:
        for name in ("k", "v"):
            codes, scale = y[name], y[name + "_scale"]
            moved = codes[from_page, :, fro % page].float() - 128                            # [n, G, HD]
            sf, before = scale[from_page], scale[pages]
            big = torch.zeros(len(pages), G, device="cuda")
            mag = torch.where((from_page != to_page)[:, None], moved.abs().amax(-1) * sf, torch.zeros_like(sf))
            big.index_reduce_(0, where, mag, "amax")
            after = torch.maximum(before, big / top)
            held = codes[pages].float() - 128
            ratio = torch.where(after > before, before / after, torch.ones_like(after))
            held = torch.round(held * ratio[..., None, None]).clamp(-127, 127)
            here = after[where]
            r = torch.where(here > 0, sf / here, torch.zeros_like(sf))
            moved = torch.round(moved * r[..., None]).clamp(-127, 127)
            held[where, :, to % page] = moved
            codes[pages], scale[pages] = (held + 128).to(torch.uint8), after
    return s["pools"]


def run(state):
    op = state["case"]["op"]
    if own:
        return {"tree": _own_tree, "append": _own_append, "attend": _own_attend, "verify": _own_verify, "keep": _own_keep}[op](state)
    return {"tree": _plain_tree, "append": _plain_append, "attend": _plain_attend, "verify": _plain_verify,
            "keep": _plain_keep}[op](state)


# ------------------------------------------------------------------------------------------------
# 64 bits, from the definitions
# ------------------------------------------------------------------------------------------------

def exact(case, seed):
    by = {"tree": _exact_tree, "append": _exact_append, "attend": _exact_attend, "verify": _exact_verify, "keep": _exact_keep}
    return by[case["op"]](prepare(case, seed))


def _ancestors(parent):
    """[n, n] truth values: j is i or lies above it."""
    n = len(parent)
    m = np.eye(n, dtype=bool)
    for i in range(n):
        j = int(parent[i])
        while j >= 0:
            m[i, j] = True
            j = int(parent[j])
    return m


def _exact_tree(s):
    """Every node's ancestors by their definition, as truth values of all pairs; powers of the parent relation."""
    q, parent, words = s["q_len"].cpu().numpy(), s["parent"].long(), s["out"]["seen"].shape[1]
    depth, seen, row = [], [], 0
    for n in q:
        n = int(n)
        p = parent[row:row + n]
        row += n
        m = torch.eye(n, dtype=F64, device="cuda")
        m[torch.arange(n, device="cuda")[p >= 0], p[p >= 0]] = 1
        for _ in range(max(1, (s["steps"] - 1).bit_length())):                     # (I + N)^(2^k)
            m = (m @ m > 0).double()
        depth.append(m.sum(1) - 1)
        wide = torch.zeros(n, words * 32, dtype=torch.int64, device="cuda")
        wide[:, :n] = m.long()
        seen.append((wide.view(n, words, 32) << torch.arange(32, device="cuda")).sum(-1))
    return dict(depth=torch.cat(depth).to(I32), seen=torch.cat(seen).to(I32))


def _exact_append(s):
    c, y = s["case"], s["layers"][0]
    H, G = c["heads"], c["kv"]
    kv, q_len, depth = s["kv_len"].cpu().numpy(), s["q_len"].cpu().numpy(), s["depth"].long()
    x = s["qkv"].double().view(-1, H + 2 * G, HD)
    rope, sa = s["rope"].double(), s["sa"].double().view(G, HD)
    k_scale, v_scale = y["k_scale"].double().clone(), y["v_scale"].double().clone()
    q_all, k_all, v_all = [], [], []
    table, row = s["table"].cpu().numpy(), 0
    for b in range(len(kv)):
        n = int(q_len[b])
        t, pos = x[row:row + n], depth[row:row + n]
        row += n
        start = int(kv[b]) - n
        turn = torch.complex(rope[start + pos, :, 0], rope[start + pos, :, 1])[:, None]
        z = torch.complex(t[..., :64], t[..., 64:])[:, :H + G] * turn
        qk = torch.cat([z.real, z.imag], -1)
        q_all.append((qk[:, :H].reshape(-1, G, H // G, HD) / sa[:, None]).reshape(-1, H * HD))
        for new, scale, out in ((qk[:, H:] * sa, k_scale, k_all), (t[:, H + G:], v_scale, v_all)):
            vals = torch.empty_like(new)
            p = start // c["page"]
            while p * c["page"] < int(kv[b]):
                lo, hi = max(start, p * c["page"]) - start, min(int(kv[b]), (p + 1) * c["page"]) - start
                before = scale[table[b, p]] if p * c["page"] < start else torch.zeros_like(scale[0])
                st = torch.maximum(before, new[lo:hi].abs().amax((0, 2)) / 127)
                scale[table[b, p]] = st
                vals[lo:hi] = torch.round(new[lo:hi] / st[:, None]).clamp(-127, 127) * st[:, None]
                p += 1
            out.append(vals.reshape(-1, G * HD))
    return dict(q=torch.cat(q_all), k_new=torch.cat(k_all), v_new=torch.cat(v_all), k=None, v=None, k_scale=k_scale,
                v_scale=v_scale)


def _exact_attend(s):
    """One sequence and KV head at a time, over its own pages."""
    c, y = s["case"], s["layers"][0]
    G, R = c["kv"], c["heads"] // c["kv"]
    kv, q_len, table, parent = s["kv_len"].cpu().numpy(), s["q_len"].cpu().numpy(), s["table"].long(), s["parent"].cpu().numpy()
    o = torch.zeros(s["total"], c["heads"], HD, dtype=F64, device="cuda")
    lse = torch.full((s["total"], c["heads"]), -math.inf, dtype=F64, device="cuda")
    row = 0
    for b in range(len(kv)):
        n, L = int(q_len[b]), int(kv[b])
        rows = slice(row, row + n)
        pages = table[b, :-(-L // c["page"])]
        hidden = torch.zeros(n, L, dtype=torch.bool, device="cuda")
        hidden[:, L - n:] = ~_dev(_ancestors(parent[row:row + n]))
        row += n
        for g in range(G):
            k, v = ((y[m][pages, g].double() - 128) * y[m + "_scale"][pages, g].double()[:, None, None] for m in ("k", "v"))
            k, v = k.reshape(-1, HD)[:L], v.reshape(-1, HD)[:L]
            heads = slice(g * R, (g + 1) * R)
            q = s["q"][rows].double().view(n, -1, HD)[:, heads]
            t = torch.einsum("nrd,ld->nrl", q, k) / math.sqrt(HD)
            t.masked_fill_(hidden[:, None], -math.inf)
            lse[rows, heads] = torch.logsumexp(t, -1) / math.log(2.0)
            o[rows, heads] = torch.einsum("nrl,ld->nrd", torch.softmax(t, -1), v)
    return dict(o=o.view(s["total"], -1), lse=lse)


def _exact_verify(s):
    """One sequence at a time: the residual distribution itself, normalised after every rejection."""
    cu, parent = s["cu"].cpu().numpy(), s["parent"].cpu().numpy()
    tok, u = s["tokens"].cpu().numpy(), s["u"].double().cpu().numpy()
    B = len(cu) - 1
    tokens, path = (np.full((B, s["steps"]), -1, np.int32) for _ in range(2))
    count = np.zeros(B, np.int32)
    for b in range(B):
        lo, hi = int(cu[b]), int(cu[b + 1])
        par, node, at, out = parent[lo:hi], 0, [0], []
        while True:
            r = s["probs"][lo + node].double()
            q = s["q"][lo + node].double() if s["q"] is not None else None
            for i in np.flatnonzero(par == node):
                x = int(tok[lo + i])
                if u[lo + i] * (float(q[x]) if q is not None else 1.0) < float(r[x]):
                    node = int(i)
                    at.append(node)
                    out.append(x)
                    break
                if q is not None:
                    r = (r - q).clamp_min(0)
                    r = r / r.sum()
                else:
                    left = 1.0 - float(r[x])
                    r[x] = 0
                    r = r / left
            else:
                cum = r.cumsum(0)
                out.append(int((cum > u[lo] * cum[-1]).to(torch.uint8).argmax()))
                break
        path[b, :len(at)], tokens[b, :len(out)], count[b] = at, out, len(at)
    return dict(tokens=_dev(tokens), path=_dev(path), count=_dev(count))


def _exact_keep(s):
    """The scales in 64 bits (codes are whole numbers under them)."""
    c = s["case"]
    kv, q_len, table = s["kv_len"].cpu().numpy(), s["q_len"].cpu().numpy(), s["table"].cpu().numpy()
    path, count = s["path"].cpu().numpy(), s["count"].cpu().numpy()
    by_page = {}                                       # page -> (page that it came from, slot there) of what moves in
    for b in range(len(kv)):
        start = int(kv[b] - q_len[b])
        for j in range(int(count[b])):
            at, fro = start + j, start + int(path[b, j])
            if at // c["page"] != fro // c["page"]:
                by_page.setdefault(int(table[b, at // c["page"]]), []).append((int(table[b, fro // c["page"]]), fro % c["page"]))
    new = dict(k=None, v=None)
    for name in ("k", "v"):
        old = s["pools"][name + "_scale"].double()
        sc = old.clone()
        for p, moves in by_page.items():
            src, slot = (torch.tensor(t, device="cuda") for t in zip(*moves))
            top = (s["pools"][name][:, src, :, slot].double() - 128).abs().amax(-1)          # [moves, layers, G]
            top = top * old[:, src].transpose(0, 1)
            sc[:, p] = torch.maximum(sc[:, p], top.amax(0) / 127)
        new[name + "_scale"] = sc
    return {k: new[k] for k in s["pools"]}


# ------------------------------------------------------------------------------------------------

def work(case):
    """Each input once, each output once; products as two operations each."""
    c = case
    size = {"f32": 4, "bf16": 2}
    kv, q = _lengths(c, 1)
    rows = int(q.sum())
    if c["op"] == "tree":
        words = (int(q.max()) + 31) // 32
        return dict(bytes=rows * (8 + 4 * words) + 4 * c["B"], flops=rows * words)
    if c["op"] == "verify":
        # the distribution of the last node of every path, the draft's there where tokens were drawn
        n = c["B"] * c["V"]
        return dict(bytes=n * size[c["p"]] * (2 if c["drawn"] else 1) + rows * 12, flops=2 * n)
    if c["op"] == "keep":
        moved = c["B"] * c["kv"] * c["layers"] * 2 * HD * min(3, c["depth"])
        return dict(bytes=2 * moved, flops=moved)
    if c["op"] == "append":
        wide = (c["heads"] + 2 * c["kv"]) * HD
        touched = sum(-(-int(a) // c["page"]) - (int(a) - int(n)) // c["page"] for a, n in zip(kv, q))
        # in: the rows; out: q, k and v in bf16 and the codes, and the scales of the pages touched
        return dict(bytes=rows * (wide * (size[c["x"]] + 2) + 2 * c["kv"] * HD) + touched * c["kv"] * 16, flops=8 * rows * wide)
    # every row sees the context and, of its tree, its ancestors (few)
    pairs = sum(int(n) * (int(a) - int(n) + min(int(n), c["depth"])) for a, n in zip(kv, q))
    cache = 2 * int(kv.sum()) * c["kv"] * HD
    return dict(bytes=cache + rows * c["heads"] * (HD * 4 + 4), flops=4 * pairs * c["heads"] * HD)
