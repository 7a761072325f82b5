"""Calls on the 8-bit cache at its edges (bounds in kv8_common.py)."""
import numpy as np
import pytest
import torch

from oracle import kv8 as D
from paper_2609_25405_amd import _abi as A
from paper_2609_25405_amd import _abi_ops as O
from paper_2609_25405_amd import ops
from tests.kv8_common import PAGE, Both, host, tensor

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu(request):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(f"\n[case] {request.node.name}", flush=True)


def value_at(b, seq, pos, head, dim):
    """The code of one value, as a view of one byte."""
    page, slot = int(b.table[seq][pos // PAGE]), pos % PAGE
    return b.kv.v.view(torch.uint8)[b.layer, page, head, slot // 4, dim % 16, dim // 16, slot % 4:slot % 4 + 1]


@pytest.mark.parametrize("seg", [(0, 300, 4), (0, 9000, 3), (0, 500, 90), (0, 9000, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_value_that_is_not_a_number_in_the_prefix_changes_its_dim_alone(seg, dtype):
    """Every row sees it: no sum is taken another way, so all other dims are the same bits."""
    shape = ops.HeadShape(4, 2, 64, dtype=dtype)
    _, off, n = seg
    b = Both(shape, 1, 600, seed=71)
    b.fill({0: off + n})
    q = tensor(b.rng.normal(size=(n, 256)), dtype)
    rows, out, bad = b.rows([seg]), *(torch.empty(n, 256, device="cuda", dtype=shape.torch_dtype) for _ in range(2))
    ops.kv8_attend(rows, b.kv, 0, q, out)
    value_at(b, 0, 37, 1, 21).fill_(0x7f)
    ops.kv8_attend(rows, b.kv, 0, q, bad)
    o, w = out.view(n, 4, 64), bad.view(n, 4, 64)
    assert o.isfinite().all() and w[:, 2:, 21].isnan().all()
    w[:, 2:, 21] = o[:, 2:, 21]
    assert torch.equal(o, w)


@pytest.mark.parametrize("seg", [(0, 50, 4), (0, 9000, 3), (0, 40, 90), (0, 4000, 150)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [False, True])
def test_attention_in_place(seg, dtype, prefix):
    """out may be q itself, also where sums are taken again because a later row's value is not a number."""
    shape = ops.HeadShape(4, 2, 64, dtype=dtype)
    _, off, n = seg
    b = Both(shape, 1, 600, seed=73)
    b.fill({0: off + n})
    value_at(b, 0, off + n - 2, 0, 3).fill_(0xff)
    if prefix:
        value_at(b, 0, 5, 0, 40).fill_(0x7f)
    q = tensor(b.rng.normal(size=(n, 256)), dtype)
    rows, out = b.rows([seg]), torch.empty(n, 256, device="cuda", dtype=shape.torch_dtype)
    ops.kv8_attend(rows, b.kv, 0, q, out)
    if not prefix:
        b.adopt()
        b.ref.val[1] = np.nan_to_num(b.ref.val[1], nan=0.0)
        b.check_attend([seg], q, out, some=set(range(n - 2)))
        assert out.view(n, 4, 64)[n - 2:, :2, 3].isnan().all()
    ops.kv8_attend(rows, b.kv, 0, q, q)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(q.view(bits), out.view(bits))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot", [32, 128])
def test_append_in_place(dtype, rot):
    """The rotated queries may take the place of the rows' own."""
    shape = ops.HeadShape(14, 2, 128, dtype=dtype, rot_dims=rot)
    segs = [(0, 3, 40), (1, 0, 1), (2, 30, 5)]
    x = tensor(np.random.default_rng(8).normal(size=(46, 18 * 128)), dtype)
    outs = []
    for place in (False, True):
        b = Both(shape, 3, 4, seed=77)
        b.fill({0: 3, 2: 30})
        y = x.clone()
        q = y[:, :14 * 128] if place else torch.empty(46, 14 * 128, device="cuda", dtype=shape.torch_dtype)
        ops.kv8_append(b.rows(segs), b.kv, 0, y, q)
        assert torch.equal(y[:, 14 * 128:], x[:, 14 * 128:])
        outs.append([q.clone(), b.kv.k.view(torch.uint8).clone(), b.kv.v.view(torch.uint8).clone(), b.kv.k_scale.clone()])
    assert all(torch.equal(a.nan_to_num(7.0), c.nan_to_num(7.0)) for a, c in zip(*outs))


@pytest.mark.parametrize("heads", [(16, 2, 64), (16, 1, 128)])
@pytest.mark.parametrize("rows", [1, 40])
def test_equal_values_come_out_whole(heads, rows):
    """Rows whose values are all 1 give 1: the sum that divides is that of the weights as they were multiplied.  The scores
    of 64 keys are above the others' by less than 2^8, so that their weights may stay above one, and all round alike."""
    shape = ops.HeadShape(*heads)
    nq, _, hd = heads
    b = Both(shape, rows, 40, seed=83)
    k, v = b.kv.k.view(torch.uint8), b.kv.v.view(torch.uint8)
    b.kv.k_scale.fill_(1.0)
    b.kv.v_scale.fill_(1.0)
    v.fill_(0x38)                                                       # 1
    q = torch.zeros(rows, nq, hd, device="cuda")
    q[..., 0] = tensor(b.rng.uniform(3.0, 5.4, size=(rows, nq)))        # times log2(e): below 8
    plan = b.rows([(s, 575, 1) for s in range(rows)])
    for first in (256, 512):                                            # (the second or third 64 keys of one wave of four or eight)
        k.zero_()
        for s in range(rows):
            for p in range(first, first + 64, PAGE):
                k[0, int(b.table[s][p // PAGE]), :, :, 0] = 0x38
        out = torch.empty(rows, nq * hd, device="cuda", dtype=torch.bfloat16)
        ops.kv8_attend(plan, b.kv, 0, q.view(rows, nq * hd).bfloat16(), out, scale=1.0)
        assert (out == 1.0).all(), (first, float(out.float().min()), float(out.float().max()))


def test_each_call_of_another_plans_replay_changes_nothing():
    """Append, read-back and attention captured apart: after the workspace got another plan, each leaves pages, scales and
    outputs as they are and says so."""
    shape = ops.HeadShape(8, 2, 128)
    b = Both(shape, 3, 8, seed=89)
    segs = [(0, 0, 50), (1, 33, 1), (2, 64, 6)]
    b.fill({s: o for s, o, _ in segs if o})
    T = 57
    x, q = tensor(b.rng.normal(size=(T, 1536)), "bf16"), torch.zeros(T, 1024, device="cuda", dtype=torch.bfloat16)
    out, ko, vo = torch.zeros_like(q), *(torch.zeros(T, 256, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    rows = b.rows(segs)
    calls = [lambda: ops.kv8_append(rows, b.kv, 0, x, q), lambda: ops.kv8_attend(rows, b.kv, 0, q, out),
             lambda: ops.kv8_read(rows, b.kv, 0, ko, vo)]
    graphs = []
    for c in calls:
        c()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c()
        graphs.append(g)
    for g in graphs:
        g.replay()
    assert rows.device_error() == 0
    rows.plan(b.kv, [(2, 10, 3), (1, 0, 1)])
    x.neg_()
    held = [b.kv.k, b.kv.v, b.kv.k_scale, b.kv.v_scale, q, ko, vo, out]
    for g in graphs:
        for t in (q, ko, vo, out):
            t.fill_(3.0)
        was = [t.contiguous().view(torch.uint8).clone() for t in held]
        g.replay()
        assert rows.device_error() == O.ORTHRUS_DEVERR_STALE
        assert all(torch.equal(t.contiguous().view(torch.uint8), w) for t, w in zip(held, was))


def test_keys_and_values_past_four_gigabytes():
    """Pages behind 4 GiB of each pool: keys and values are held there, read back and attended to, and the pages before are
    as they were."""
    shape = ops.HeadShape(8, 8, 128)
    n_pages = 2 ** 32 // (8 * 2048) + 5
    kv = ops.DeviceKV8(shape, 1, n_pages, 1, 2)
    kv.set_block_table(np.array([[n_pages - 1, n_pages - 2]]))
    x = host(tensor(np.random.default_rng(3).normal(size=(20, 24, 128)), "bf16"))
    rows = ops.RaggedRows(shape, 20, 1, 20)
    rows.plan(kv, [(0, 0, 20)])
    q, o, ko, vo = (torch.empty(20, 1024, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    ops.kv8_append(rows, kv, 0, tensor(x.reshape(20, -1), "bf16"), q)
    ops.kv8_read(rows, kv, 0, ko, vo)
    ops.kv8_attend(rows, kv, 0, q, o)
    assert rows.device_error() == 0
    freq = 10000.0 ** (-2.0 * np.arange(64) / 128)
    turned = np.stack([D.turn(x[t, 8:16], t, freq) for t in range(20)])
    scale = host(kv.k_scale[0, [n_pages - 1] * 16 + [n_pages - 2] * 4])[..., None]
    length = np.sqrt(np.sum(turned * turned, -1, keepdims=True))
    k, v = host(ko).reshape(20, 8, 128), host(vo).reshape(20, 8, 128)
    assert (np.abs(k - turned) <= np.maximum(2.0 ** -4 * np.abs(turned), 2.0 ** -10 * scale) + 2.0 ** -18 * length).all()
    vs = host(kv.v_scale[0, [n_pages - 1] * 16 + [n_pages - 2] * 4])[..., None]
    np.testing.assert_array_equal(v, D.e4m3(x[:, 16:] / vs) * vs)
    qs, got = host(q).reshape(20, 8, 128), host(o).reshape(20, 8, 128)
    for t in range(20):
        for h in range(8):
            s = k[:t + 1, h] @ qs[t, h] * 128 ** -0.5
            p = np.exp(s - s.max())
            p /= p.sum()
            size = float(np.max(np.abs(k[:t + 1, h]) @ np.abs(qs[t, h]))) * 128 ** -0.5
            want, mag = p @ v[:t + 1, h], p @ np.abs(v[:t + 1, h])
            tol = mag * (2.0 ** -8 + 2.0 ** -16 + 2 * size * 2.0 ** -19) + np.abs(want) * 2.0 ** -8 + 1e-30
            assert (np.abs(got[t, h] - want) <= tol).all(), (t, h)
    for pool in (kv.k, kv.v):
        c = pool.view(torch.uint8)[0, :n_pages - 2].view(-1)
        assert not any(c[i:i + 2 ** 30].any() for i in range(0, c.numel(), 2 ** 30))


def test_scales_that_fp32_does_not_hold():
    """A scale that rounds to zero in fp32 is refused, not taken for the usual one; so is one that overflows on its
    way to base 2.  The least and the largest that pass are what they say."""
    shape = ops.HeadShape(4, 2, 64)
    b = Both(shape, 1, 8, seed=79)
    b.fill({0: 100})
    q = tensor(b.rng.normal(size=(1, 256)), "bf16")
    rows, out = b.rows([(0, 99, 1)]), torch.empty(1, 256, device="cuda", dtype=torch.bfloat16)
    for scale in (1e-46, 1e-300, 0.0, 2.4e38, 1e39):
        with pytest.raises(A.OrthrusError, match=r"\(-1\)"):
            ops.kv8_attend(rows, b.kv, 0, q, out, scale=scale)
    ops.kv8_attend(rows, b.kv, 0, q, out, scale=1e-30)
    b.check_attend([(0, 99, 1)], q, out, scale=1e-30)
    ops.kv8_attend(rows, b.kv, 0, torch.zeros_like(q), out, scale=2.3e38)
    b.check_attend([(0, 99, 1)], torch.zeros_like(q), out, scale=2.3e38)


def test_one_row_of_any_stride():
    """The stride of a tensor of one row is nobody's."""
    shape = ops.HeadShape(4, 2, 64)
    b = Both(shape, 1, 8, seed=97)
    b.fill({0: 100})
    q = tensor(b.rng.normal(size=(1, 256)), "bf16")
    odd = torch.empty(1 * 259 + 8, device="cuda", dtype=torch.bfloat16).as_strided((1, 256), (259, 1))
    odd.copy_(q)
    rows, out = b.rows([(0, 99, 1)]), torch.empty(1, 256, device="cuda", dtype=torch.bfloat16)
    ops.kv8_attend(rows, b.kv, 0, odd, out)
    b.check_attend([(0, 99, 1)], q, out)


def test_magnitudes_at_the_end_of_the_range():
    """What would round past the largest power of two that fp32 holds is held as not a number, like an infinity; all below
    keeps a finite value."""
    shape = ops.HeadShape(1, 1, 64, dtype="f32", rot_dims=0)
    b = Both(shape, 2, 1, seed=101)
    x = np.zeros((2, 3, 64))
    top = 2.0 ** 120
    x[0, 1:, :6] = [247.9 * top, -247.9 * top, 248 * top, float(np.finfo(np.float32).max), -255 * top, 225 * top]
    x[1, 1:, :2] = [224 * top, -1.0]
    x = host(tensor(x))
    rows = b.rows([(0, 0, 1), (1, 0, 1)])
    ops.kv8_append(rows, b.kv, 0, tensor(x.reshape(2, -1)), torch.empty(2, 64, device="cuda"))
    ko, vo = (torch.empty(2, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    ops.kv8_read(rows, b.kv, 0, ko, vo)
    for t in (host(ko), host(vo)):
        assert t[0, [0, 1, 5]].tolist() == [240 * top, -240 * top, 224 * top] and np.isnan(t[0, 2:5]).all()
        assert t[1, 0] == 224 * top and (t[1, 1:] == 0).all()


@pytest.mark.parametrize("seg", [(0, 200, 1), (0, 200, 3), (0, 2000, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [None, 1e30])
def test_scores_are_taken_of_values_not_of_codes(seg, dtype, scale):
    """Queries whose products with a page's codes leave the range of fp32, while those with its keys do not: the row is the
    value of its largest score."""
    shape = ops.HeadShape(4, 2, 64, dtype=dtype)
    _, off, n = seg
    b = Both(shape, 1, 130, seed=103)
    b.fill({0: off + n})
    size = 2.0 ** 120 if scale is None else 2.0 ** 10
    down = 2.0 ** -40 if scale is None else 1.0
    b.kv.k_scale.mul_(down)
    b.adopt()
    q = torch.zeros(n, 4, 64, device="cuda", dtype=shape.torch_dtype)
    q[:, :, 7] = size
    out = torch.empty(n, 256, device="cuda", dtype=shape.torch_dtype)
    ops.kv8_attend(b.rows([seg]), b.kv, 0, q.view(n, 256), out, scale=scale)
    k, v = b.ref.rows(b.table, 0, 0, off + n)
    for t in range(n):
        for h in range(4):
            s = k[:off + t + 1, h // 2, 7]
            most = s == s.max()
            want = v[:off + t + 1, h // 2][most].mean(0)
            tol = 2.0 ** (-7 if dtype == "bf16" else -22) * np.abs(v[:off + t + 1, h // 2][most]).mean(0)
            assert (np.abs(host(out[t].view(4, 64)[h]) - want) <= tol).all(), (t, h)


@pytest.mark.parametrize("seg", [(0, 150, 51), (0, 0, 130), (0, 9000, 40), (0, 500, 3), (0, 1500, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [2.0 ** 18, 2.0 ** 24, 2.0 ** 40, 2.0 ** 100])
def test_scores_of_any_size(seg, dtype, size):
    """The row of scores far apart is the value of the largest, whatever their size; several heads, of which one has ordinary
    scores."""
    shape = ops.HeadShape(4, 2, 64, dtype=dtype)
    _, off, n = seg
    b = Both(shape, 1, 600, seed=107)
    b.fill({0: off + n})
    q = torch.zeros(n, 4, 64, device="cuda", dtype=shape.torch_dtype)
    q[:, :, 7] = size
    q[:, 1, 7] = -size
    q[:, 3] = tensor(b.rng.normal(size=(n, 64)))
    out = torch.empty(n, 256, device="cuda", dtype=shape.torch_dtype)
    ops.kv8_attend(b.rows([seg]), b.kv, 0, q.view(n, 256), out)
    b.check_attend([seg], q, out, some=set(range(0, n, 13)))           # (bounds of the ordinary head)
    k, v = b.ref.rows(b.table, 0, 0, off + n)
    got = host(out.view(n, 4, 64))
    for t in range(0, n, 13):
        for h in range(3):
            s = k[:off + t + 1, h // 2, 7] * (-1 if h == 1 else 1)
            gap = s.max() - s
            if gap[gap > 0].size and gap[gap > 0].min() * size / 8 < 2000:
                continue
            most = gap == 0
            want, mag = v[:off + t + 1, h // 2][most].mean(0), np.abs(v[:off + t + 1, h // 2][most]).mean(0)
            assert (np.abs(got[t, h] - want) <= 2.0 ** (-7 if dtype == "bf16" else -20) * mag).all(), (t, h)


@pytest.mark.parametrize("seg", [(0, 1000, 90), (0, 37, 130), (0, 30, 3), (0, 2111, 2), (0, 9001, 40)])
@pytest.mark.parametrize("heads", [(4, 2, 64), (14, 2, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [False, True])
def test_rows_before_a_value_that_is_not_a_number(seg, heads, dtype, bad):
    """Their sums are taken again without it: in tiles and small items, over whole and partial steps, pieces, and past a bad
    page."""
    shape = ops.HeadShape(*heads, dtype=dtype)
    nq, nkv, hd = heads
    _, off, n = seg
    b = Both(shape, 1, 600, seed=109)
    b.fill({0: off + n})
    last = off + n - 1
    for d in range(hd):
        value_at(b, 0, last, d % nkv, d).fill_(0x7f if d % 3 else 0xff)
    skip = ()
    if bad:
        b.table[0][1], skip = -1, (-1,)
        b.kv.set_block_table(b.table)
    b.adopt()
    b.ref.val[1] = np.nan_to_num(b.ref.val[1], nan=0.0)
    q = tensor(b.rng.normal(size=(n, nq * hd)) * 2, dtype)
    rows, out = b.rows([seg]), torch.empty(n, nq * hd, device="cuda", dtype=shape.torch_dtype)
    ops.kv8_attend(rows, b.kv, 0, q, out)
    assert rows.device_error() == (A.ORTHRUS_DEVERR_PAGE if bad else 0)
    b.check_attend([seg], q, out, some=set(range(0, n - 1, 7)) | {max(n - 2, 0)}, skip=skip)
    got = out[n - 1].view(nkv, nq // nkv, hd).isnan()
    for g in range(nkv):
        assert got[g, :, g::nkv].all() and not got[g, :, 1 - g::nkv].any()
