"""The operators that serve a calibrated block in 8 bits, over the sizes that they meet.

* ``norm``    residual addition, RMSNorm with the folded gain and bias, and the per-token 8-bit MinMax
              quantizer that feeds the next product (``omq_rmsnorm_quant``).
* ``gemm``    the product of 8-bit activation and weight codes with a step and zero point per token
              and per output channel (``omq_qgemm_i8``).
* ``append``  rotary positions and the [Q, K] scale on new q, k, v rows, and the write of k and v into
              the pages of an 8-bit cache with one scale per page and head (``omq_kv_append``).
* ``attend``  attention of the newest tokens of every sequence over that cache (``omq_kv_attention``).

``run`` computes an operator in elementary torch operations (``own`` false) or through the package's
entry points (``own`` true), from the same prepared state.  Sizes: the LLaMA-7B (hidden 4096, 32
heads, FFN 11008), LLaMA-13B (5120, 40 heads, 13824) and LLaMA-2-70B (8192, 64 query and 8 KV heads,
28672) blocks of this repository, at serving batch sizes and context lengths, and generic odd ones.
"""
import math

import numpy as np
import torch

own = False

HD = 128                       # head dimension
RMS_EPS = 1e-6
H_EPS = 1e-5                   # floor of the quantizer's step
THETA = 10000.0


def listed():
    return [
        # one decoded token of the 7B block: latency
        dict(name="norm_1x4096_decode", op="norm", T=1, C=4096, x="f32", r="f32", res=True, bits=8),
        # a ragged batch of prompts at the 13B FFN width, bf16 linear outputs without a residual
        dict(name="norm_777x13824_bf16", op="norm", T=777, C=13824, x="bf16", r="f32", res=False, bits=8),
        # a long prefill at the 70B width: bf16 linear output added to the fp32 residual stream
        dict(name="norm_8192x8192_prefill", op="norm", T=8192, C=8192, x="bf16", r="f32", res=True, bits=8),
        # q|k|v of the 7B block for one token: the weight read is everything
        dict(name="gemm_1x12288x4096", op="gemm", M=1, N=12288, K=4096, out="f32", zero=True, bias=True),
        # the 13B down projection for a small decode batch, odd row count
        dict(name="gemm_17x5120x13824", op="gemm", M=17, N=5120, K=13824, out="f32", zero=True, bias=False),
        # a ragged chunk of prompt tokens through the 7B down projection, symmetric codes
        dict(name="gemm_509x4096x11008", op="gemm", M=509, N=4096, K=11008, out="f32", zero=False, bias=False),
        # gate|up of the 7B block for a 2048-token prompt
        dict(name="gemm_2048x22016x4096", op="gemm", M=2048, N=22016, K=4096, out="bf16", zero=True, bias=True),
        # one new token of each of 64 sequences, 70B heads
        dict(name="append_64seq_gqa8", op="append", B=64, nq=1, ragged_q=False, heads=64, kv=8, kv_max=4096, page=64,
             x="f32"),
        # a 2048-token prompt of the 7B block written into an empty cache
        dict(name="append_2048_prompt", op="append", B=1, nq=2048, ragged_q=False, heads=32, kv=32, kv_max=2048, page=64,
             x="f32"),
        # one sequence of the 7B block: short context, latency
        dict(name="attend_1seq_2048", op="attend", B=1, nq=1, ragged_q=False, heads=32, kv=32, kv_max=2048, page=64,
             empty=False),
        # a serving batch at 70B heads, ragged contexts, up to five tokens to verify each, one sequence empty
        dict(name="attend_64seq_ragged_verify", op="attend", B=64, nq=5, ragged_q=True, heads=64, kv=8, kv_max=4099,
             page=32, empty=True),
        # four very long contexts at 70B heads: the cache read is everything
        dict(name="attend_4seq_131072", op="attend", B=4, nq=1, ragged_q=False, heads=64, kv=8, kv_max=131072, page=64,
             empty=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "gemm", "append", "attend"])
    if op == "norm":
        C = 8 * _log(rng, 16, 3584)                     # 128 .. 28672
        T = min(_log(rng, 1, 8192), 8192 * 8192 // C)
        return dict(op=op, T=T, C=C, x=rng.choice(["f32", "bf16"]), r=rng.choice(["f32", "bf16"]),
                    res=rng.random() < 0.7, bits=8)
    if op == "gemm":
        N, K = 8 * _log(rng, 32, 2752), 16 * _log(rng, 16, 864)      # 256 .. 22016, 256 .. 13824
        M = min(_log(rng, 1, 4096), max(1, 2048 * 22016 * 4096 // (N * K)))
        return dict(op=op, M=M, N=N, K=K, out=rng.choice(["f32", "bf16"]), zero=rng.random() < 0.7,
                    bias=rng.random() < 0.5)
    kv = rng.choice([1, 2, 4, 8, 32, 40])
    heads = kv * (rng.choice([1, 2, 3, 4, 7, 8]) if kv <= 8 else 1)
    page = rng.choice([16, 32, 64, 128])
    if op == "append":
        if rng.random() < 0.5:                          # decode and verify
            B, nq = _log(rng, 1, 128), rng.choice([1, 1, 1, 2, 5, 8])
            kv_max = max(nq + 1, min(_log(rng, 64, 4096), 64 * 4096 * 8 // (B * kv)))
        else:                                           # chunks of prompts
            B = rng.randint(1, 4)
            nq = _log(rng, 16, max(17, 2048 * 96 // (B * (heads + 2 * kv))))
            kv_max = nq + rng.choice([0, 1, rng.randint(1, 1000)])
        return dict(op=op, B=B, nq=nq, ragged_q=rng.random() < 0.5, heads=heads, kv=kv, kv_max=kv_max, page=page,
                    x=rng.choice(["f32", "bf16"]))
    nq = rng.choice([1, 1, 1, 2, 3, 5, 8, 16])
    B = _log(rng, 1, 96)
    kv_max = max(nq, _log(rng, 16, min(131072, max(64, 4 * 131072 * 8 // (B * kv * (1 + nq * heads // kv // 16))))))
    return dict(op=op, B=B, nq=nq, ragged_q=nq > 1 and rng.random() < 0.5, heads=heads, kv=kv, kv_max=kv_max, page=page,
                empty=rng.random() < 0.3)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _lengths(c, seed):
    """Host-side lengths of every sequence: (tokens in the cache with the new ones, new tokens).  The case
    alone gives the lengths, so that every seed has the same shapes; the seed gives their order."""
    B, nq, top = c["B"], c["nq"], c["kv_max"]
    r = np.random.RandomState(B * 7 + nq * 1009 + top)
    q = r.randint(1, nq + 1, B) if c["ragged_q"] else np.full(B, nq)
    q[0] = nq
    kv = np.maximum(r.randint(max(1, top // 4), top + 1, B), q)
    kv[0] = top
    if c.get("empty") and B > 1:
        kv[1] = 0                                       # nothing to attend to: every row of it is empty
    order = np.random.RandomState(int(seed) % (1 << 31)).permutation(B)
    return kv[order].astype(np.int32), q[order].astype(np.int32)


def _pool(c, g, kv, seed):
    """Page pool of an 8-bit cache: codes of bell-shaped values, scales that differ by page and head."""
    page, need = c["page"], [max(1, -(-int(n) // c["page"])) for n in kv]
    n_pages = sum(need) + 3
    order = np.random.RandomState((int(seed) + 5) % (1 << 31)).permutation(n_pages)
    table = np.full((len(kv), max(need)), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (n_pages, c["kv"], page, HD)

    def codes():
        out = torch.empty(shape, dtype=torch.uint8, device="cuda")
        for i in range(0, n_pages, 4096):               # bounded scratch for the large pools
            part = out[i:i + 4096]
            part.copy_((_randn(g, *part.shape) * 30 + 128).round_().clamp_(1, 255))
        return out

    s = dict(k=codes(), v=codes())
    s["k_scale"] = torch.exp(0.3 * _randn(g, n_pages, c["kv"])) / 30
    s["v_scale"] = torch.exp(0.5 * _randn(g, n_pages, c["kv"])) / 30
    s["table"] = torch.from_numpy(table).cuda()
    s["kv_len"] = torch.from_numpy(kv).cuda()
    return s


def _rope(n):
    ang = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * \
        THETA ** (-torch.arange(0, HD, 2, dtype=torch.float64, device="cuda") / HD)
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()      # [n, 64, 2]


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = dict(case=c)
    if c["op"] == "norm":
        T, C = c["T"], c["C"]
        hot = (torch.rand(C, generator=g, device="cuda") < 0.01).float() * 15 + 1     # outlier channels
        s["x"] = (_randn(g, T, C) * hot).to(_DT[c["x"]])
        s["r"] = (_randn(g, T, C) * hot).to(_DT[c["r"]]) if c["res"] else None
        s["gain"] = torch.exp(0.1 * _randn(g, C)) / hot.sqrt()
        s["bias"] = 0.05 * _randn(g, C)
    elif c["op"] == "gemm":
        M, N, K = c["M"], c["N"], c["K"]

        def codes(rows):
            out = torch.empty(rows, K, dtype=torch.uint8, device="cuda")
            for i in range(0, rows, 4096):
                part = out[i:i + 4096]
                part.copy_((_randn(g, *part.shape) * 30 + 128).round_().clamp_(0, 255))
            return out

        def zeros(n):
            if not c["zero"]:
                return None
            return torch.randint(100, 157, (n,), generator=g, device="cuda", dtype=torch.int32)

        s["a"], s["a_h"], s["a_z"] = codes(M), torch.exp(0.3 * _randn(g, M)) * 0.03, zeros(M)
        s["w"], s["w_h"], s["w_z"] = codes(N), torch.exp(0.3 * _randn(g, N)) * 6e-4, zeros(N)
        s["bias"] = _randn(g, N) if c["bias"] else None
    else:
        kv, q = _lengths(c, seed)
        s.update(_pool(c, g, kv, seed))
        total = int(q.sum())
        cu = np.concatenate([[0], np.cumsum(q)]).astype(np.int32)
        s["cu"] = torch.from_numpy(cu).cuda()
        s["total"], s["max_q"], s["max_kv"] = total, int(q.max()), max(1, int(kv.max()))
        s["seq"] = torch.from_numpy(np.repeat(np.arange(len(q)), q)).cuda()           # row -> sequence
        s["at"] = torch.from_numpy(np.concatenate([np.arange(n) for n in q])).cuda()  # row -> its place in it
        s["q_len"] = torch.from_numpy(q).cuda()
        if c["op"] == "append":
            s["qkv"] = _randn(g, total, (c["heads"] + 2 * c["kv"]) * HD).to(_DT[c["x"]])
            s["rope"] = _rope(s["max_kv"])
            s["sa"] = torch.exp(0.1 * _randn(g, c["kv"] * HD))
        else:
            s["q"] = _randn(g, total, c["heads"] * HD).to(torch.bfloat16)
    _buffers(s)
    return s


def _buffers(s):
    """Output buffers that a serving loop keeps between steps."""
    c = s["case"]
    new = lambda dt, *shape: torch.empty(*shape, dtype=dt, device="cuda")  # noqa: E731
    f32, bf16 = torch.float32, torch.bfloat16
    if c["op"] == "norm":
        s["out"] = dict(codes=new(torch.uint8, c["T"], c["C"]), h=new(f32, c["T"]), z=new(torch.int32, c["T"]),
                        values=new(bf16, c["T"], c["C"]), residual=torch.empty_like(s["r"]) if c["res"] else None)
    elif c["op"] == "gemm":
        s["out"] = new(_DT[c["out"]], c["M"], c["N"])
    elif c["op"] == "append":
        s["out"] = dict(q=new(bf16, s["total"], c["heads"] * HD), k_new=new(bf16, s["total"], c["kv"] * HD),
                        v_new=new(bf16, s["total"], c["kv"] * HD))
    else:
        s["out"] = dict(o=new(bf16, s["total"], c["heads"] * HD), lse=new(f32, s["total"], c["heads"]))


# ------------------------------------------------------------------------------------------------
# the package's entry points
# ------------------------------------------------------------------------------------------------

def _own_norm(s):
    from paper_2308_13137_gb300 import serve
    o = s["out"]
    serve.rmsnorm_quant(s["x"], s["r"], s["gain"], s["bias"], bits=s["case"]["bits"], rms_eps=RMS_EPS, h_eps=H_EPS,
                        out=serve.QuantRows(**o))
    got = dict(values=o["values"], h=o["h"])            # the values that the 8-bit codes stand for
    if o["residual"] is not None:
        got["residual"] = o["residual"]
    return got


def _own_gemm(s):
    from paper_2308_13137_gb300 import serve
    return serve.qgemm(s["a"], s["a_h"], s["a_z"], s["w"], s["w_h"], s["w_z"], bias=s["bias"], out=s["out"])


def _cache(s):
    """The handle of the cache, made once as a serving loop makes it."""
    from paper_2308_13137_gb300 import serve
    if "cache" not in s:
        s["cache"] = serve.KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], s["kv_len"])
    return s["cache"]


def _own_append(s):
    from paper_2308_13137_gb300 import serve
    o = s["out"]
    serve.kv_append(_cache(s), s["qkv"], s["rope"], s["case"]["heads"], cu_q=s["cu"], max_q=s["max_q"], sa=s["sa"],
                    q_out=o["q"], k_out=o["k_new"], v_out=o["v_new"])
    return dict(o, k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"])


def _own_attend(s):
    from paper_2308_13137_gb300 import serve
    o = s["out"]
    serve.kv_attention(_cache(s), s["q"], s["case"]["heads"], cu_q=s["cu"], max_q=s["max_q"], max_kv=s["max_kv"],
                       out=o["o"], lse=o["lse"])
    return o


# ------------------------------------------------------------------------------------------------
# plain forms, 32 bits
# ------------------------------------------------------------------------------------------------

def _plain_norm(s):
    c = s["case"]
    Q = float(2 ** c["bits"] - 1)
    x = s["x"].float() + s["r"].float() if c["res"] else s["x"].float()
    y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + RMS_EPS) * s["gain"] + s["bias"]
    hi, lo = y.amax(-1, keepdim=True), y.amin(-1, keepdim=True)
    h = ((hi - lo) / Q).clamp_min(H_EPS)
    z = -torch.round(torch.where((hi - lo) / Q >= H_EPS, Q * lo / (hi - lo), lo / h))
    q = (torch.round(y / h) + z).clamp(0, Q)
    out = dict(values=((q - z) * h).to(torch.bfloat16), h=h[:, 0])
    if c["res"]:
        out["residual"] = x.to(s["r"].dtype)
    return out


def _plain_gemm(s):
    a = s["a"].float() - (128.0 if s["a_z"] is None else s["a_z"].float()[:, None])
    w = s["w"].float() - (128.0 if s["w_z"] is None else s["w_z"].float()[:, None])
    y = (a @ w.t()) * s["a_h"][:, None] * s["w_h"][None, :]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(_DT[s["case"]["out"]])


def _plain_append(s):
    c = s["case"]
    H, G, page = c["heads"], c["kv"], c["page"]
    x = s["qkv"].float().view(s["total"], H + 2 * G, HD)
    pos = (s["kv_len"] - s["q_len"])[s["seq"]].long() + s["at"]
    cs = s["rope"][pos]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]

    def turn(t):
        a, b = t[..., :64], t[..., 64:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    sa = s["sa"].view(G, HD)
    q = turn(x[:, :H]).view(-1, G, H // G, HD) / sa[:, None]
    k, v = turn(x[:, H:H + G]) * sa, x[:, H + G:]
    page_at = s["table"][s["seq"], pos // page].long()                      # row -> page of the pool
    # the pages that this call writes, and the tokens that each held before it (none in one it starts)
    pages, where = torch.unique(page_at, return_inverse=True)
    kept = torch.zeros_like(pages)
    kept[where] = ((s["kv_len"] - s["q_len"])[s["seq"]].long() - pos // page * page).clamp(0, page)
    out = dict(q=q.reshape(s["total"], -1).to(torch.bfloat16))
    for_one = torch.full((), 127.0, device="cuda")      # a tensor: division by a number multiplies by its reciprocal
    out.update(_plain_write(s, "k", k, pages, where, pos % page, kept, for_one))
    out.update(_plain_write(s, "v", v, pages, where, pos % page, kept, for_one))
    return out


def _plain_write(s, name, val, pages, where, slot, kept, top):
    codes, scale = s[name], s[name + "_scale"]
    held, page = codes[pages], codes.shape[2]
    big = torch.zeros(len(pages), codes.shape[1], device="cuda")
    big.index_reduce_(0, where, val.abs().amax(-1), "amax")
    before = torch.where((kept > 0)[:, None], scale[pages], torch.zeros_like(big))
    after = torch.maximum(before, big / top)
    # tokens already in a page whose scale grows are rounded again to the new scale
    grown = (after > before)[:, :, None, None] & (torch.arange(page, device="cuda") < kept[:, None])[:, None, :, None]
    again = torch.round((held.float() - 128) * (before / after)[..., None, None]) + 128
    held = torch.where(grown, again, held.float()).to(torch.uint8)
    sc = after[where][..., None]
    c = torch.where(sc > 0, torch.round(val / sc), torch.zeros_like(val)).clamp(-127, 127)
    held[where, :, slot] = (c + 128).to(torch.uint8)
    codes[pages], scale[pages] = held, after
    return {name: codes, name + "_scale": scale, name + "_new": (c * sc).reshape(len(where), -1).to(torch.bfloat16)}


def _attend(s, dt):
    """Attention over the gathered, dequantised pages in the type dt; softmax base 2 as the package's lse."""
    c = s["case"]
    G, R = c["kv"], c["heads"] // c["kv"]
    B, L = c["B"], s["table"].shape[1] * c["page"]
    tab = s["table"].clamp_min(0).long()

    def gather(name):
        t = (s[name][tab].to(dt) - 128) * s[name + "_scale"][tab].to(dt)[..., None, None]   # [B, n, G, page, HD]
        return t.permute(0, 2, 1, 3, 4).reshape(B, G, L, HD)

    q = torch.zeros(B, s["max_q"], c["heads"] * HD, dtype=dt, device="cuda")
    q[s["seq"], s["at"]] = s["q"].to(dt)
    q = q.view(B, -1, G, R, HD).permute(0, 2, 1, 3, 4).reshape(B, G, -1, HD)            # [B, G, nq R, HD]
    sc = (q @ gather("k").transpose(-1, -2)) * (math.log2(math.e) / math.sqrt(HD))
    last = (s["kv_len"] - s["q_len"])[:, None] + torch.arange(s["max_q"], device="cuda")  # newest visible key
    seen = torch.arange(L, device="cuda") <= last.repeat_interleave(R, 1)[..., None]
    seen &= (torch.arange(L, device="cuda") < s["kv_len"][:, None])[:, None]
    sc = torch.where(seen[:, None], sc, torch.full_like(sc, -math.inf))
    m = sc.amax(-1, keepdim=True)
    p = torch.exp2(sc - torch.where(m > -math.inf, m, torch.zeros_like(m)))
    l = p.sum(-1, keepdim=True)
    o = (p @ gather("v")) / torch.where(l > 0, l, torch.ones_like(l))
    lse = m + torch.log2(l)

    def rows(t, w):
        t = t.view(B, G, -1, R, w).permute(0, 2, 1, 3, 4).reshape(B, -1, G * R * w)
        return t[s["seq"], s["at"]]

    return rows(o, HD), rows(lse, 1)


def _plain_attend(s):
    o, lse = _attend(s, torch.float32)
    return dict(o=o.to(torch.bfloat16), lse=lse)


def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _own_norm, "gemm": _own_gemm, "append": _own_append, "attend": _own_attend}[op](state)
    return {"norm": _plain_norm, "gemm": _plain_gemm, "append": _plain_append, "attend": _plain_attend}[op](state)


# ------------------------------------------------------------------------------------------------
# 64 bits, from the definitions
# ------------------------------------------------------------------------------------------------

def exact(case, seed):
    by = {"norm": _exact_norm, "gemm": _exact_gemm, "append": _exact_append, "attend": _exact_attend}
    return by[case["op"]](prepare(case, seed))


def _exact_norm(s):
    c = s["case"]
    Q = 2 ** c["bits"] - 1
    t = s["x"].double()
    if s["r"] is not None:
        t = t + s["r"].double()
    rms = (t.pow(2).sum(1) / t.shape[1] + RMS_EPS).sqrt()
    y = t / rms[:, None] * s["gain"].double() + s["bias"].double()
    top, bottom = y.max(1).values, y.min(1).values
    step = torch.clamp((top - bottom) / Q, min=H_EPS)
    zero = torch.round(bottom / step)                     # minus the zero point
    lev = torch.round(y / step[:, None])
    lev = torch.minimum(torch.maximum(lev, zero[:, None]), zero[:, None] + Q)
    out = dict(values=lev * step[:, None], h=step)
    if s["r"] is not None:
        out["residual"] = t
    return out


def _exact_gemm(s):
    M, N = s["a"].shape[0], s["w"].shape[0]
    out = torch.empty(M, N, dtype=torch.float64, device="cuda")
    za = s["a_z"].double() if s["a_z"] is not None else torch.full((M,), 128.0, dtype=torch.float64, device="cuda")
    zw = s["w_z"].double() if s["w_z"] is not None else torch.full((N,), 128.0, dtype=torch.float64, device="cuda")
    x = (s["a"].double() - za[:, None]) * s["a_h"].double()[:, None]
    for j in range(0, N, 2048):
        w = (s["w"][j:j + 2048].double() - zw[j:j + 2048, None]) * s["w_h"][j:j + 2048].double()[:, None]
        out[:, j:j + 2048] = torch.einsum("mk,nk->mn", x, w)
    if s["bias"] is not None:
        out += s["bias"].double()
    return out


def _exact_append(s):
    c = s["case"]
    H, G = c["heads"], c["kv"]
    kv, q_len = s["kv_len"].cpu().numpy(), s["q_len"].cpu().numpy()
    x = s["qkv"].double().view(-1, H + 2 * G, HD)
    rope, sa = s["rope"].double(), s["sa"].double().view(G, HD)
    k_scale, v_scale = s["k_scale"].double().clone(), s["v_scale"].double().clone()
    q_all, k_all, v_all = [], [], []
    table, row = s["table"].cpu().numpy(), 0
    for b in range(len(kv)):
        t = x[row:row + q_len[b]]
        row += q_len[b]
        start = int(kv[b]) - int(q_len[b])
        turn = torch.complex(rope[start:start + q_len[b], :, 0], rope[start:start + q_len[b], :, 1])[:, None]
        z = torch.complex(t[..., :64], t[..., 64:])[:, :H + G] * turn
        qk = torch.cat([z.real, z.imag], -1)
        q_all.append((qk[:, :H].reshape(-1, G, H // G, HD) / sa[:, None]).reshape(-1, H * HD))
        for new, scale, out in ((qk[:, H:] * sa, k_scale, k_all), (t[:, H + G:], v_scale, v_all)):
            vals = torch.empty_like(new)
            p = start // c["page"]
            while p * c["page"] < int(kv[b]):
                a, e = max(start, p * c["page"]) - start, min(int(kv[b]), (p + 1) * c["page"]) - start
                before = scale[table[b, p]] if p * c["page"] < start else torch.zeros_like(scale[0])
                st = torch.maximum(before, new[a:e].abs().amax((0, 2)) / 127)
                scale[table[b, p]] = st
                vals[a:e] = torch.round(new[a:e] / st[:, None]).clamp(-127, 127) * st[:, None]
                p += 1
            out.append(vals.reshape(-1, G * HD))
    return dict(q=torch.cat(q_all), k_new=torch.cat(k_all), v_new=torch.cat(v_all), k=None, v=None, k_scale=k_scale,
                v_scale=v_scale)


def _exact_attend(s):
    """One sequence and KV head at a time, over its own pages."""
    c = s["case"]
    G, R = c["kv"], c["heads"] // c["kv"]
    kv, q_len, table = s["kv_len"].cpu().numpy(), s["q_len"].cpu().numpy(), s["table"].long()
    o = torch.zeros(s["total"], c["heads"], HD, dtype=torch.float64, device="cuda")
    lse = torch.full((s["total"], c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    row = 0
    for b in range(len(kv)):
        n, L = int(q_len[b]), int(kv[b])
        rows = slice(row, row + n)
        row += n
        if L == 0:
            continue
        pages = table[b, :-(-L // c["page"])]
        hidden = torch.arange(L, device="cuda") > torch.arange(L - n, L, device="cuda")[:, None]
        for g in range(G):
            k, v = ((s[m][pages, g].double() - 128) * s[m + "_scale"][pages, g].double()[:, None, None]
                    for m in ("k", "v"))
            k, v = k.reshape(-1, HD)[:L], v.reshape(-1, HD)[:L]
            heads = slice(g * R, (g + 1) * R)
            q = s["q"][rows].double().view(n, -1, HD)[:, heads]
            t = torch.einsum("nrd,ld->nrl", q, k) / math.sqrt(HD)
            t.masked_fill_(hidden[:, None], -math.inf)
            lse[rows, heads] = torch.logsumexp(t, -1) / math.log(2.0)
            o[rows, heads] = torch.einsum("nrl,ld->nrd", torch.softmax(t, -1), v)
    return dict(o=o.view(s["total"], -1), lse=lse)


# ------------------------------------------------------------------------------------------------

def work(case):
    """Each input once, each output once; products as two operations each."""
    c = case
    size = {"f32": 4, "bf16": 2}
    if c["op"] == "norm":
        n = c["T"] * c["C"]
        # in: x (and the residual); out: codes, the bf16 values they stand for, the residual sum
        per = size[c["x"]] + 3 + (2 * size[c["r"]] if c["res"] else 0)
        return dict(bytes=n * per + 8 * c["C"] + 8 * c["T"], flops=8 * n)
    if c["op"] == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        return dict(bytes=M * K + N * K + M * N * size[c["out"]] + (8 if c["zero"] else 4) * (M + N), flops=2 * M * N * K)
    kv, q = _lengths(c, 1)
    rows = int(q.sum())
    if c["op"] == "append":
        wide = (c["heads"] + 2 * c["kv"]) * HD
        touched = sum(-(-int(a) // c["page"]) - (int(a) - int(n)) // c["page"] for a, n in zip(kv, q))
        # in: the rows; out: q, k and v in bf16 and the codes, and the scales of the pages touched
        return dict(bytes=rows * (wide * (size[c["x"]] + 2) + 2 * c["kv"] * HD) + touched * c["kv"] * 16, flops=8 * rows * wide)
    cache = 2 * int(kv.sum()) * c["kv"] * HD
    pairs = sum(int(n) * int(a) - int(n) * (int(n) - 1) // 2 for a, n in zip(kv, q) if a)
    return dict(bytes=cache + rows * c["heads"] * (HD * 4 + 4), flops=4 * pairs * c["heads"] * HD)
