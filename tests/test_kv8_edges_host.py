"""Refusals of the 8-bit cache's calls at their edges, on the CPU."""
import ctypes
import re

import numpy as np
import pytest
import torch

from paper_2609_25405_amd import _abi as A
from paper_2609_25405_amd import _abi_ops as O
from paper_2609_25405_amd import ops


def code_of(rc):
    return pytest.raises(A.OrthrusError, match=re.escape(f"({rc})"))


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


@pytest.mark.parametrize("segs", [[(-2 ** 63, 0, 1)], [(2 ** 32, 0, 1)], [(0, -2 ** 31 - 1, 1)], [(0.5, 0, 1)],
                                  np.array([[2 ** 64 - 2 ** 32, 0, 1]], np.uint64)])
def test_segments_that_are_no_32_bit_integers_are_refused(segs):
    shape = ops.HeadShape(8, 4, 128)
    kv, rows = ops.DeviceKV8(shape, 1, 8, 4, 8, device="cpu"), ops.RaggedRows(shape, 64, 4, 128, device="cpu")
    with code_of(A.ORTHRUS_EINVAL):
        rows.items(kv, segs)


def test_segments_of_any_integer_type():
    shape = ops.HeadShape(8, 4, 128)
    kv, rows = ops.DeviceKV8(shape, 1, 8, 4, 8, device="cpu"), ops.RaggedRows(shape, 64, 4, 128, device="cpu")
    want = rows.items(kv, [(1, 3, 2)])
    for dt in (np.int32, np.int64, np.uint8, np.uint64):
        got = rows.items(kv, np.array([[1, 3, 2]], dt))
        assert got[0] == want[0] and (got[1] == want[1]).all()
    assert rows.items(kv, [])[0] == [0, 0, 0, 0]
