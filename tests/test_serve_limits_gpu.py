"""The ends of what the serving calls take."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16, U8, I32 = torch.float32, torch.bfloat16, torch.uint8, torch.int32


def _new(dt, *s):
    return torch.zeros(*s, dtype=dt, device="cuda")


def test_empty_batch_is_refused(cuda_lib):
    """A table of no sequences is a ValueError when the cache is made, and in the calls themselves."""
    from paper_2308_13137_gb300 import _lib, serve
    c = serve.KVCache.empty(4, 2, 16, 3, 2)
    with pytest.raises(ValueError):
        serve.KVCache(c.k, c.v, c.k_scale, c.v_scale, c.table[:0], c.kv_len[:0])
    with pytest.raises(ValueError):
        serve.KVCache.empty(4, 2, 16, 0, 2)
    none = _lib.omq_kv_cache.from_buffer_copy(c.handle)
    none.B = 0
    at, bind, rope = ctypes.addressof(none), serve._load_bind(), serve.rope_table(32)
    for n in (0, 3):
        qkv, q = _new(F32, n, 8 * 128), _new(BF16, n, 4 * 128)
        for cu, most in ((None, None), (_new(I32, 1), 1)):
            with pytest.raises(ValueError):
                bind.kv_append(at, qkv, rope, 4, cu, most, None, q, None, None, c.status)
            with pytest.raises(ValueError):
                bind.kv_attention(at, q, 4, cu, most, 32, q, None, c.status)
