"""ServedBlock's host side, without a GPU: which arguments its calls receive."""
import os
import types

import pytest
import torch

from paper_2308_13137_gb300 import _lib, serve
from paper_2308_13137_gb300.serve_block import ServedBlock

F32, U8, I32 = torch.float32, torch.uint8, torch.int32


def _block(device="cpu"):
    """A block of random packed weights, made from the dictionary that fold_pack returns."""
    sh = types.SimpleNamespace(d=256, ffn=384, n_heads=2, n_kv=1, rms_eps=1e-6)
    outs = dict(qkv=(4 * 128, 256), o=(256, 256), gu=(2 * 384, 256), d=(256, 384))
    packed = {}
    for k, (n, m) in outs.items():
        packed["codes_" + k] = torch.zeros(n, m, dtype=U8)
        packed["h_" + k], packed["z_" + k] = torch.ones(n, 1), torch.zeros(n, 1, dtype=I32)
    return ServedBlock(sh, packed, wbits=8, abits=8, device=device)


def test_every_kernel_reports_to_the_cache(monkeypatch):
    """A wait that runs out in a product or a quantizer sets the cache's status word, so that KVCache.check raises
    (the norm has no unfinished output: a row that does not arrive is read directly)."""
    status = torch.zeros(1, dtype=I32)
    cache = types.SimpleNamespace(status=status)
    seen, words = [], []

    def qgemm(a, a_h, a_z, w, w_h, w_z, bias=None, out=None, out_dtype=F32, status=None):
        seen.append(status)
        return torch.zeros(a.shape[0], w.shape[0], dtype=out_dtype)

    def norm(x, r=None, *a, **kw):
        return serve.QuantRows(torch.zeros(x.shape, dtype=U8), torch.ones(len(x)), torch.zeros(len(x), dtype=I32), None, r)

    monkeypatch.setattr(serve, "qgemm", qgemm)
    monkeypatch.setattr(serve, "rmsnorm_quant", norm)
    monkeypatch.setattr(serve, "kv_append", lambda c, qkv, rope, h, **kw: torch.zeros(len(qkv), h * 128, dtype=torch.bfloat16))
    monkeypatch.setattr(serve, "kv_attention", lambda c, q, h, **kw: torch.zeros(len(q), h * 128))
    monkeypatch.setattr(_lib, "omq_act_quant_per_token", lambda *a: words.append(a[-1].dev_status))
    _block().forward(torch.zeros(3, 256), cache, None)
    assert len(seen) == 4 and all(s is status for s in seen)
    assert words == [status.data_ptr()] * 2


def test_the_cache_lies_on_the_blocks_device(monkeypatch):
    asked = []

    def empty(n_pages, n_kv, page, B, max_pages, device="cuda"):
        asked.append(device)
        return types.SimpleNamespace(table=torch.zeros(B, max_pages, dtype=I32))

    monkeypatch.setattr(serve.KVCache, "empty", empty)
    _block("cpu").cache(2, 100)
    assert [str(d) for d in asked] == ["cpu"]


@pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libomq.so not built")
def test_the_module_of_the_calls_loads():
    """Every symbol that the compiled module needs is exported by what it links (no device is touched)."""
    bind = serve._load_bind()
    assert all(hasattr(bind, f) for f in ("rmsnorm_quant", "qgemm", "kv_append", "kv_attention"))
    with pytest.raises(TypeError):
        bind.qgemm(None)
    with pytest.raises(ValueError):
        bind.qgemm(*[None] * 9)
