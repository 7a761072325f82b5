"""Refusals of the 8-bit cache's calls at their edges, on the CPU."""
import ctypes

import torch

from paper_2609_25405_amd import _abi as A
from paper_2609_25405_amd import _abi_ops as O
from paper_2609_25405_amd import ops


def test_caches_of_a_step_share_no_pool_and_no_scale():
    """Neither like with like nor keys with values, in whole or in part."""
    from paper_2609_25405_amd import runtime as R
    from workload import Batch, DecodeRow, EmbChunk, draw_tokens, make_weights, tiny_config
    cfg = tiny_config("bf16")
    m = R.DeviceModel(cfg, make_weights(cfg, 1), device="cpu")
    shape = ops.HeadShape(4, 4, 64)
    kv, other = (ops.DeviceKV8(shape, 2, 40, 6, 4, device="cpu") for _ in range(2))
    both = Batch([EmbChunk(0, 0, 5, True)], [DecodeRow(1, 9)], draw_tokens(1, 0, 6, cfg.vocab))
    buf, out = torch.zeros(4096, dtype=torch.uint8), torch.zeros(6, max(cfg.vocab, cfg.d_model))
    at = -(-buf.data_ptr() // 256) * 256

    def call(g, e=None):
        p, e = R.PackedBatch(both), e or kv.struct()
        return O.load().orthrus_step_kv8(m.handle, m.handle, ctypes.byref(p.c), ctypes.byref(e), ctypes.byref(g), out.data_ptr(),
                                         out.data_ptr(), out.data_ptr(), out.data_ptr(), at, 2048, None)

    def changed(c, **kw):
        s = c.struct()
        for k, v in kw.items():
            setattr(s, k, v)
        return s

    pool, scales = kv.k.numel(), kv.k_scale.numel() * 4
    assert call(other.struct()) == A.ORTHRUS_ECAPACITY                # (all in order but the workspace's size)
    for kw in (dict(k_cache=kv.v.data_ptr()), dict(v_cache=kv.k.data_ptr()), dict(k_scale=kv.v_scale.data_ptr()),
               dict(v_scale=kv.k_scale.data_ptr()), dict(k_cache=kv.v.data_ptr() + pool - 16), dict(v_cache=kv.k.data_ptr() - pool + 16),
               dict(k_cache=kv.k.data_ptr() + 4096), dict(v_scale=kv.v_scale.data_ptr() + scales - 4)):
        assert call(changed(other, **kw)) == A.ORTHRUS_EINVAL, kw
    # one cache whose own pools are one
    for kw in (dict(v_cache=kv.k.data_ptr()), dict(k_scale=kv.v_scale.data_ptr())):
        one = changed(kv, **kw)
        assert call(one, one) == A.ORTHRUS_EINVAL, kw
    # side by side in one allocation they may stand
    big = torch.zeros(4 * pool + 16, dtype=torch.uint8)
    a = -(-big.data_ptr() // 16) * 16
    e, g = changed(kv, k_cache=a, v_cache=a + 2 * pool), changed(other, k_cache=a + pool, v_cache=a + 3 * pool)
    assert call(g, e) == A.ORTHRUS_ECAPACITY
