"""Attention over the 8-bit cache against the float64 definition (bounds in kv8_common.py)."""
import numpy as np
import pytest
import torch

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


def attend(b, segs, spread=1.0, scale=None, some=None, pad=0, skip=()):
    s = b.shape
    T, width = sum(n for _, _, n in segs), s.n_q_heads * s.head_dim
    q = torch.full((T, width + pad), float("nan"), device="cuda", dtype=s.torch_dtype)
    q[:, :width] = tensor(b.rng.normal(size=(T, width)) * spread)
    out = torch.full((T + 1, width + pad), 9.0, device="cuda", dtype=s.torch_dtype)
    rows = b.rows(segs)
    ops.kv8_attend(rows, b.kv, b.layer, q[:, :width], out[:, :width], scale)
    torch.cuda.synchronize()
    assert rows.device_error() == (A.ORTHRUS_DEVERR_PAGE if skip else 0)
    assert (out[T] == 9.0).all() and (out[:, width:] == 9.0).all()
    b.worst = b.check_attend(segs, q[:, :width], out[:T, :width], scale, some, skip)
    print("worst / bound", b.worst, flush=True)
    return q[:, :width], out[:T, :width]


HEADS = {"mha64": (4, 4, 64), "group2": (4, 2, 128), "group4": (8, 2, 128), "group7": (14, 2, 64), "group16": (16, 1, 128)}


@pytest.mark.parametrize("heads", list(HEADS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_single_tokens_at_every_kind_of_length(heads, dtype):
    shape = ops.HeadShape(*HEADS[heads], dtype=dtype)
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 128, 255, 256, 257, 700]
    b = Both(shape, len(lens), 44, seed=len(heads), layers=2, layer=1)
    b.fill(dict(enumerate(lens)))
    attend(b, [(s, n - 1, 1) for s, n in enumerate(lens)], pad=8)


@pytest.mark.parametrize("heads", list(HEADS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_chunks_of_uneven_lengths_beside_single_tokens(heads, dtype):
    shape = ops.HeadShape(*HEADS[heads], dtype=dtype)
    segs = [(0, 0, 33), (1, 5, 1), (2, 60, 70), (3, 0, 2), (4, 100, 3), (5, 16, 16), (6, 299, 1), (7, 0, 150)]
    b = Both(shape, 8, 20, seed=3 + len(heads))
    b.fill({s: o + n for s, o, n in segs})
    attend(b, segs, pad=16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spread", [0.0, 8.0])
def test_flat_and_sharp_weights(dtype, spread):
    shape = ops.HeadShape(8, 2, 128, dtype=dtype)
    b = Both(shape, 2, 40, seed=17)
    b.fill({0: 600, 1: 90}, 2.0)
    attend(b, [(0, 599, 1), (1, 20, 70)], spread)
    attend(b, [(0, 590, 10)], spread, scale=0.02)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_ranges_come_in_pieces(dtype):
    """One token, few tokens and a chunk over long prefixes: pieces and their merge."""
    shape = ops.HeadShape(4, 2, 64, dtype=dtype)
    segs = [(0, 20000, 1), (1, 9000, 3), (2, 17000, 40), (3, 30, 1)]
    b = Both(shape, 4, 1300, seed=23)
    b.fill({s: o + n for s, o, n in segs})
    counts, _ = ops.RaggedRows(shape, 45, 4, 20001).items(b.kv, segs)
    assert counts[2] >= 6 and counts[1] > 2
    attend(b, segs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [False, True])
def test_tiles_of_many_pages(dtype, bad):
    """So many rows that no range is cut: a tile walks over more pages than it keeps at a time, a bad one among
    the later ones."""
    shape = ops.HeadShape(64, 8, 128, dtype=dtype)
    segs = [(0, 7411, 1030), (1, 4090, 20)]
    b = Both(shape, 2, 528, seed=61)
    b.fill({s: o + n for s, o, n in segs})
    counts, items = ops.RaggedRows(shape, 1050, 2, 8441).items(b.kv, segs)
    assert (items[counts[0]:, 6] - items[counts[0]:, 5]).max() > 8000
    skip = ()
    if bad:
        b.table[0][300], b.table[1][256], skip = b.kv.n_pages, -3, (b.kv.n_pages, -3)
        b.kv.set_block_table(b.table)
        b.ref.val = [np.concatenate([v, np.zeros((4,) + v.shape[1:])]) for v in b.ref.val]
    attend(b, segs, some={0, 1, 517, 1028, 1029, 1030, 1035, 1036, 1049}, skip=skip)


def test_many_rows_with_uneven_contexts():
    shape = ops.HeadShape(8, 2, 128)
    rng = np.random.default_rng(4)
    segs = [(s, int(n), 1) for s, n in enumerate(np.exp(rng.uniform(0, np.log(1500), 150)).astype(int))]
    b = Both(shape, 150, 100, seed=29)
    b.fill({s: o + n for s, o, n in segs})
    attend(b, segs, some=set(range(0, 150, 7)))


@pytest.mark.parametrize("segs", [[(0, 40, 1), (1, 33, 5)], [(0, 30, 40), (1, 0, 100)]])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_pages_are_skipped_and_flagged(segs, dtype):
    shape = ops.HeadShape(4, 2, 64, dtype=dtype)
    b = Both(shape, 2, 8, seed=31)
    b.fill({s: o + n for s, o, n in segs})
    b.table[0][1], b.table[1][0] = b.kv.n_pages + 7, -2
    b.kv.set_block_table(b.table)
    b.ref.val = [np.concatenate([v, np.zeros((10,) + v.shape[1:])]) for v in b.ref.val]
    attend(b, segs, skip=(b.kv.n_pages + 7, -2))


def test_a_row_without_keys_is_zero():
    shape = ops.HeadShape(4, 2, 64)
    b = Both(shape, 2, 2, seed=33)
    b.fill({0: 1, 1: 30})
    b.table[0][0] = -1
    b.kv.set_block_table(b.table)
    _, out = attend(b, [(0, 0, 1), (1, 29, 1)], skip=(-1,))
    assert (out[0] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seg", [(0, 50, 4), (0, 40, 90)])
def test_odd_values_reach_only_the_rows_that_see_them(dtype, seg):
    """A key or value that is not a number, in the middle of a segment's own tokens: earlier rows are
    as without it, later ones are not a number (a key: everywhere; a value: in its dim)."""
    shape = ops.HeadShape(4, 2, 64, dtype=dtype)
    _, off, n = seg
    b = Both(shape, 1, 10, seed=35)
    b.fill({0: off + n})
    q = tensor(b.rng.normal(size=(n, 256)), dtype)
    rows = b.rows([seg])
    for which in ("k", "v"):
        out, bad = (torch.empty(n, 256, device="cuda", dtype=shape.torch_dtype) for _ in range(2))
        ops.kv8_attend(rows, b.kv, 0, q, out)
        at = off + n // 2
        page, slot = int(b.table[0][at // PAGE]), at % PAGE
        pool = b.kv.k if which == "k" else b.kv.v
        keep = pool.view(torch.uint8).clone()
        if which == "k":
            pool.view(torch.uint8)[0, page, 1, slot, 5] = 0x7f
        else:
            pool.view(torch.uint8)[0, page, 1, slot // 4, 37 % 16, 37 // 16, slot % 4] = 0x7f
        ops.kv8_attend(rows, b.kv, 0, q, bad)
        pool.view(torch.uint8).copy_(keep)
        sees = torch.arange(n, device="cuda") >= n // 2
        o, w = out.view(n, 4, 64), bad.view(n, 4, 64)
        assert torch.equal(o[:, :2], w[:, :2])                         # the other KV head
        tol = 2.0 ** (-6 if dtype == "bf16" else -14)
        assert (o[~sees, 2:].float() - w[~sees, 2:].float()).abs().max() <= tol * o.float().abs().max()
        if which == "k":
            assert w[sees, 2:].isnan().all()
        else:
            assert w[sees, 2:, 37].isnan().all()
            assert not w[sees, 2:, :37].isnan().any() and not w[sees, 2:, 38:].isnan().any()
    assert rows.device_error() == 0


@pytest.mark.parametrize("seg", [(0, 300, 1), (0, 9000, 1), (0, 50, 4), (0, 9000, 3), (0, 40, 90), (0, 9000, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_row_of_scores_that_are_all_minus_infinity_is_not_a_number(seg, dtype):
    """No weights can be taken of such scores, in one piece or several; a row without keys is zero beside it.  Rows of
    other heads are as without it, and so is a row for which some keys only have such scores."""
    shape = ops.HeadShape(4, 2, 64, dtype=dtype)
    _, off, n = seg
    b = Both(shape, 2, 600, seed=36)
    b.fill({0: off + n, 1: 30})
    k = b.kv.k.view(torch.uint8)
    k[..., 5] = 0xb8                                                    # dim 5 of every key: -1 times the scale
    b.kv.k_scale.copy_(torch.where(b.kv.k_scale > 0, 2.0 ** 5, b.kv.k_scale))
    b.table[1][0] = -1
    b.kv.set_block_table(b.table)
    segs = [seg, (1, 9, 1)]
    q = tensor(b.rng.normal(size=(n + 1, 256)), dtype)
    rows, out, bad = b.rows(segs), *(torch.full((n + 1, 256), 5.0, device="cuda", dtype=shape.torch_dtype) for _ in range(2))
    ops.kv8_attend(rows, b.kv, 0, q, out)
    # a finite query whose scores overflow: -2^127 * 2^5 / sqrt(64)
    q2 = q.clone()
    q2.view(n + 1, 4, 64)[:n, 1] = 0
    q2.view(n + 1, 4, 64)[:n, 1, 5] = 2.0 ** 127
    ops.kv8_attend(rows, b.kv, 0, q2, bad)
    torch.cuda.synchronize()
    assert rows.device_error() == A.ORTHRUS_DEVERR_PAGE
    o, w = out.view(n + 1, 4, 64), bad.view(n + 1, 4, 64)
    assert w[:n, 1].isnan().all() and (w[n] == 0).all() and (o[n] == 0).all()
    for h in (0, 2, 3):
        assert torch.equal(o[:n, h], w[:n, h]) and o[:n, h].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_appended_tokens_are_seen_and_chunking_does_not_matter(dtype):
    """A prompt appended and attended at once, in chunks, and token by token."""
    shape = ops.HeadShape(4, 2, 64, dtype=dtype, interleaved=True)
    n = 75
    rng = np.random.default_rng(6)
    x = tensor(rng.normal(size=(n, 8 * 64)), dtype)
    x[:, 4 * 64:] = x[:, 4 * 64:] / x[:, 4 * 64:].float().abs().amax()      # one scale from the first token on ...
    x[0, 4 * 64:] = 1.0
    outs = []
    for cuts in ([75], [20, 1, 54], [1] * 75):
        b = Both(shape, 1, 6, seed=41)
        out = torch.empty(n, 256, device="cuda", dtype=shape.torch_dtype)
        at = 0
        for c in cuts:
            q = torch.empty(c, 256, device="cuda", dtype=shape.torch_dtype)
            rows = b.rows([(0, at, c)])
            ops.kv8_append(rows, b.kv, 0, x[at:at + c], q)
            ops.kv8_attend(rows, b.kv, 0, q, out[at:at + c])
            b.adopt()
            b.check_attend([(0, at, c)], q, out[at:at + c])
            at += c
        outs.append(host(out))
    # pages may have another scale on the way, a power of two that only tiny values see
    for o in outs[1:]:
        assert np.abs(o - outs[0]).max() <= 2.0 ** (-6 if dtype == "bf16" else -9) * np.abs(outs[0]).max()


def test_results_do_not_depend_on_the_other_rows_or_the_run():
    shape = ops.HeadShape(8, 2, 128)
    b = Both(shape, 6, 40, seed=43)
    segs = [(s, 100 * s + 3, 1) for s in range(6)]
    b.fill({s: o + n for s, o, n in segs})
    q, out = attend(b, segs)
    rows, again = b.rows(segs), torch.empty_like(out)
    for _ in range(3):
        ops.kv8_attend(rows, b.kv, 0, q, again)
        assert torch.equal(again, out)


def test_captured_calls_replay_their_plan_and_notice_another():
    """Append, read-back and attention in one graph, replayed with new inputs between eager calls; after the
    workspace got another plan, a replay changes nothing and says so."""
    shape = ops.HeadShape(8, 2, 128)
    b = Both(shape, 4, 20, seed=47)
    segs = [(0, 0, 50), (1, 33, 1), (2, 200, 2), (3, 64, 30)]
    b.fill({s: o for s, o, _ in segs if o})
    T = 83
    x, q = torch.zeros(T, 1536, device="cuda", dtype=torch.bfloat16), torch.empty(T, 1024, device="cuda", dtype=torch.bfloat16)
    out, ko, vo = torch.empty_like(q), *(torch.empty(T, 256, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    rows, eager = b.rows(segs), b.rows(segs)

    def call(r, q, out, ko, vo):
        ops.kv8_append(r, b.kv, 0, x, q)
        ops.kv8_attend(r, b.kv, 0, q, out)
        ops.kv8_read(r, b.kv, 0, ko, vo)

    call(rows, q, out, ko, vo)
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        with pytest.raises(A.OrthrusError):
            rows.plan(b.kv, segs)
        call(rows, q, out, ko, vo)
    for i in range(4):
        x.copy_(tensor(b.rng.normal(size=(T, 1536))))
        want = [torch.empty_like(t) for t in (q, out, ko, vo)]
        g.replay()
        got = [t.clone() for t in (q, out, ko, vo)]
        call(eager, *want)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want)), i
    assert rows.device_error() == 0
    rows.plan(b.kv, [(0, 0, 1)])
    out.fill_(4.0)
    g.replay()
    assert (out == 4.0).all() and rows.device_error() == O.ORTHRUS_DEVERR_STALE
    ops.kv8_attend(rows, b.kv, 0, q, out)
    assert rows.device_error() == 0 and not (out[0] == 4.0).all() and (out[1:] == 4.0).all()


def test_calls_follow_the_stream_they_are_given():
    shape = ops.HeadShape(4, 2, 64)
    b = Both(shape, 2, 8, seed=51)
    segs = [(0, 90, 1), (1, 20, 30)]
    b.fill({s: o + n for s, o, n in segs})
    q = tensor(b.rng.normal(size=(31, 256)), "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rows = ops.RaggedRows(shape, 31, 2, 91)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        rows.plan(b.kv, segs)
        out = torch.zeros(31, 256, device="cuda", dtype=torch.bfloat16)
        ops.kv8_attend(rows, b.kv, 0, q, out)
    side.synchronize()
    b.check_attend(segs, q, out)
    out2 = torch.zeros_like(out)
    torch.cuda.synchronize()
    ops.kv8_attend(rows, b.kv, 0, q, out2, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(out, out2)


def test_plans_follow_each_other_without_waiting():
    """Many plans of one handle, each used at once: the upload of one never overtakes the calls of another."""
    shape = ops.HeadShape(4, 2, 64)
    b = Both(shape, 40, 10, seed=53)
    b.fill({s: 3 * s + 5 for s in range(40)})
    q = tensor(b.rng.normal(size=(8, 256)), "bf16")
    rows = ops.RaggedRows(shape, 8, 8, 160)
    outs = []
    for s in range(32):
        rows.plan(b.kv, [(s + i, 3 * (s + i) + 4, 1) for i in range(8)])
        outs.append(torch.empty(8, 256, device="cuda", dtype=torch.bfloat16))
        ops.kv8_attend(rows, b.kv, 0, q, outs[-1])
    torch.cuda.synchronize()
    for s in range(0, 32, 5):
        b.check_attend([(s + i, 3 * (s + i) + 4, 1) for i in range(8)], q, outs[s])
    rows.plan(b.kv, [])
    ops.kv8_attend(rows, b.kv, 0, q[:0], outs[0][:0])


def test_arguments_that_are_refused():
    shape = ops.HeadShape(4, 2, 64)
    b = Both(shape, 2, 4, seed=55)
    rows = b.rows([(1, 30, 2)])
    q, out = (torch.zeros(2, 256, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    bad = [lambda: ops.kv8_attend(rows, b.kv, 1, q, out), lambda: ops.kv8_attend(rows, b.kv, -1, q, out),
           lambda: ops.kv8_attend(rows, b.kv, 0, q[:1], out), lambda: ops.kv8_attend(rows, b.kv, 0, q.float(), out),
           lambda: ops.kv8_attend(rows, b.kv, 0, q, out, scale=float("inf")), lambda: ops.kv8_attend(rows, b.kv, 0, q, out, scale=-1.0),
           lambda: ops.kv8_attend(rows, b.kv, 0, torch.zeros(2, 260, device="cuda", dtype=torch.bfloat16)[:, :256], out),
           lambda: ops.kv8_attend(rows, b.kv, 0, torch.zeros(2, 264, device="cuda", dtype=torch.bfloat16)[:, 4:260], out),
           lambda: ops.kv8_attend(rows, b.kv, 0, q.cpu(), out), lambda: ops.kv8_attend(rows, b.kv, 0, q.t(), out),
           lambda: ops.kv8_append(rows, b.kv, 0, q, out), lambda: ops.kv8_read(rows, b.kv, 0, out, out)]
    for i, call in enumerate(bad):
        with pytest.raises(A.OrthrusError, match=r"\(-1\)"):
            call()
    small = ops.DeviceKV8(shape, 1, 4, 1, 4)
    with pytest.raises(A.OrthrusError, match=r"\(-4\)"):
        ops.kv8_attend(rows, small, 0, q, out)                 # a cache without sequence 1
    fp = ops.HeadShape(4, 2, 64, dtype="f32")
    r2 = ops.RaggedRows(fp, 2, 1, 32)
    r2.plan(b.kv, [(1, 30, 2)])
    with pytest.raises(A.OrthrusError):
        ops.kv8_append(r2, b.kv, 0, torch.zeros(2, 512, device="cuda", dtype=torch.bfloat16), torch.zeros(2, 256, device="cuda"))
    torch.cuda.synchronize()
    assert rows.device_error() == 0
