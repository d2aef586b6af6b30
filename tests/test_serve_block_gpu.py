"""The serving operators together: a calibrated and packed block run in 8 bits over the paged cache."""
import pytest
import torch

import oracle as O
from paper_2308_13137_gb300 import inputs as I

pytestmark = pytest.mark.gpu


def _rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


def _case(n_heads, n_kv, let, wbits, T=96):
    from paper_2308_13137_gb300.block import BlockState
    from paper_2308_13137_gb300.serve_block import ServedBlock
    sh = I.BlockShape("served", T=T, d=512, n_heads=n_heads, n_kv=n_kv, ffn=768, wbits=wbits, abits=8, group=0, let=let,
                      outlier_scale=8.0)
    W = I.make_block_weights(sh, seed=1)
    x = I.make_block_input(sh, sample=0, weight_seed=1)
    th = I.make_block_theta(sh, W, x, seed=2)
    st = BlockState(sh, W, th)
    y_fp = O.block_fp_forward(x, W, O.BlockCfg.from_shape(sh))
    return sh, ServedBlock.from_state(st), torch.from_numpy(x).cuda(), y_fp.cuda(), st


@pytest.mark.parametrize("n_heads,n_kv,let,wbits", [(4, 4, 1, 8), (8, 2, 1, 8), (4, 1, 0, 8), (4, 4, 1, 6)])
def test_prompt_against_the_block_in_double(cuda_lib, n_heads, n_kv, let, wbits):
    """The whole prompt in one call.  Against the full-precision block in float64: 8-bit weights, activations and
    cache.  Per quantized tensor the noise is a step of range / 255 uniform, 1 to 2 % of a bell-shaped tensor's
    size; about eight of them add up (6 %), on the block's contribution y - x."""
    from paper_2308_13137_gb300 import serve
    sh, blk, x, y_fp, _ = _case(n_heads, n_kv, let, wbits)
    cache, rope = blk.cache(1, sh.T, page=32), serve.rope_table(sh.T)
    cache.kv_len.fill_(sh.T)
    h, d = blk.forward(x, cache, rope)
    cache.check()
    tol = 0.06 * (1 if wbits == 8 else 4)                      # six-bit weights: four times the step
    assert _rel(h + d - x, y_fp - x.double()) < tol


def test_same_as_the_calibration_forward(cuda_lib):
    """Close to the library's own fake-quantized forward of the same settings (W8A8: it quantizes q, k and v per
    token, the cache k and v per page and head): both carry the same kind of noise."""
    from paper_2308_13137_gb300 import serve
    sh, blk, x, _, st = _case(4, 4, 1, 8)
    y = torch.empty_like(x)
    st.forward(x, y)
    cache = blk.cache(1, sh.T)
    cache.kv_len.fill_(sh.T)
    h, d = blk.forward(x, cache, serve.rope_table(sh.T))
    assert _rel(h + d - x, y - x) < 0.06


def test_token_by_token_and_in_chunks(cuda_lib):
    """Two sequences of different lengths through two blocks: one call, ragged chunks, and single tokens give the
    same outputs up to the caches' rounding (a page is rounded again where its scale grows), and the
    second block takes the first one's output through its fused residual addition."""
    from paper_2308_13137_gb300 import serve
    sh, blk, x, _, _ = _case(8, 2, 1, 8)
    rope = serve.rope_table(sh.T)
    n = [60, 36]
    rows = [x[:60], x[60:96]]

    def run(cuts):
        caches = [blk.cache(2, 64, page=16) for _ in range(2)]
        out = [[], []]
        for lo, hi in zip(cuts[:-1], cuts[1:]):
            part = [rows[b][min(lo, n[b]):min(hi, n[b])] for b in range(2)]
            k = [len(p) for p in part]
            cu = torch.tensor([0, k[0], k[0] + k[1]], dtype=torch.int32, device="cuda")
            for c in caches:
                c.kv_len.copy_(torch.tensor([min(hi, m) for m in n], dtype=torch.int32))
            h, d = blk.forward(torch.cat(part), caches[0], rope, cu_q=cu, max_q=max(k))
            h, d = blk.forward(h, caches[1], rope, delta=d, cu_q=cu, max_q=max(k))
            for b, y in enumerate((h + d).split(k)):
                out[b].append(y)
        for c in caches:
            c.check()
        return [torch.cat(o) for o in out]

    whole = run([0, 60])
    for cuts in ([0, 17, 18, 40, 60], list(range(61))):
        for a, b, r in zip(whole, run(cuts), rows):
            assert _rel(b - r, a - r) < 0.06
