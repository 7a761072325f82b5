"""The 8-bit cache's operators and token scores on the CPU: headers and bindings, refusals, the
attention work lists, and the float64 definitions they are compared with elsewhere."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from oracle import kv8 as D
from paper_2609_25405_amd import _abi as A
from paper_2609_25405_amd import _abi_ops as O
from paper_2609_25405_amd import ops

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include")
HEADERS = ["orthrus/kv8.h", "orthrus/score.h"]


def code_of(rc):
    return pytest.raises(A.OrthrusError, match=re.escape(f"({rc})"))


def test_headers_and_bindings_name_the_same_symbols():
    names = set()
    for h in HEADERS:
        src = re.sub(r"/\*.*?\*/", "", open(os.path.join(INCLUDE, h)).read(), flags=re.S)
        names |= set(re.findall(r"\b(orthrus_[a-z0-9_]+)\s*\(", src))
    assert names == set(O.SIGNATURES)
    lib = O.load()
    assert all(hasattr(lib, n) for n in names)


def test_ctypes_mirror_matches_the_c_compiler(tmp_path):
    lines = ["#include <stddef.h>", "#include <stdio.h>"] + [f'#include "{h}"' for h in HEADERS] + ["int main(void) {"]
    structs = ["orthrus_kv8", "orthrus_head_shape", "orthrus_segment"]
    for st in structs:
        lines.append(f'printf("{st} size %zu\\n", sizeof({st}));')
        for f, _ in getattr(O, st)._fields_:
            lines.append(f'printf("{st} {f} %zu\\n", offsetof({st}, {f}));')
    lines += [f'printf("{c} value %d\\n", {c});' for c in ("ORTHRUS_DEVERR_STALE", "ORTHRUS_MAX_TOP")] + ["return 0; }"]
    (tmp_path / "probe.c").write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", INCLUDE, str(tmp_path / "probe.c"), "-o", str(tmp_path / "probe")], check=True)
    for line in subprocess.run([str(tmp_path / "probe")], check=True, capture_output=True, text=True).stdout.split("\n")[:-1]:
        st, f, v = line.split()
        want = getattr(O, st) if f == "value" else ctypes.sizeof(getattr(O, st)) if f == "size" else getattr(getattr(O, st), f).offset
        assert int(v) == want, line


def cpu_cache(shape, n_pages=8, n_seq=4, max_blocks=8):
    return ops.DeviceKV8(shape, 1, n_pages, n_seq, max_blocks, device="cpu")


def cpu_rows(shape, *sizes):
    return ops.RaggedRows(shape, *(sizes or (64, 4, 128)), device="cpu")


@pytest.mark.parametrize("kw,rc", [
    (dict(n_q_heads=0), A.ORTHRUS_EINVAL), (dict(n_q_heads=6, n_kv_heads=4), A.ORTHRUS_EINVAL),
    (dict(n_kv_heads=-1), A.ORTHRUS_EINVAL), (dict(head_dim=96), A.ORTHRUS_EUNSUPPORTED),
    (dict(n_q_heads=68, n_kv_heads=4), A.ORTHRUS_EUNSUPPORTED), (dict(rot_dims=24), A.ORTHRUS_EUNSUPPORTED),
    (dict(rot_dims=144), A.ORTHRUS_EINVAL), (dict(rot_dims=-16), A.ORTHRUS_EINVAL), (dict(rope_base=1.0), A.ORTHRUS_EINVAL),
    (dict(rope_base=math.inf), A.ORTHRUS_EINVAL), (dict(rope_magnitude=math.nan), A.ORTHRUS_EINVAL),
    (dict(norm_eps=-1.0), A.ORTHRUS_EINVAL), (dict(rope_freq=np.full(64, math.nan)), A.ORTHRUS_EINVAL),
    (dict(rope_freq=np.ones(63)), A.ORTHRUS_EINVAL), (dict(dtype="f16"), A.ORTHRUS_EINVAL)])
def test_shapes_that_are_refused(kw, rc):
    args = dict(n_q_heads=8, n_kv_heads=4, head_dim=128)
    args.update(kw)
    with code_of(rc):
        cpu_rows(ops.HeadShape(**args))


def test_shape_without_rotation_needs_no_base():
    cpu_rows(ops.HeadShape(4, 4, 64, rot_dims=0, rope_base=0.0))


@pytest.mark.parametrize("segs,rc", [
    ([(4, 0, 1)], A.ORTHRUS_EDESC), ([(-1, 0, 1)], A.ORTHRUS_EDESC), ([(0, -1, 1)], A.ORTHRUS_EDESC), ([(0, 0, 0)], A.ORTHRUS_EDESC),
    ([(0, 0, -5)], A.ORTHRUS_EDESC), ([(0, 0, 129)], A.ORTHRUS_ECAPACITY), ([(0, 128, 1)], A.ORTHRUS_ECAPACITY),
    ([(0, 2 ** 31 - 1, 2 ** 31 - 1)], A.ORTHRUS_ECAPACITY), ([(1, 0, 2), (2, 0, 1), (1, 2, 1)], A.ORTHRUS_EDUPSEQ),
    ([(0, 0, 2 ** 31)], A.ORTHRUS_EINVAL)])
def test_segments_that_are_refused(segs, rc):
    shape = ops.HeadShape(8, 4, 128)
    with code_of(rc):
        cpu_rows(shape).items(cpu_cache(shape), segs)


def test_calls_that_are_refused_before_anything_is_enqueued():
    lib, shape = O.load(), ops.HeadShape(8, 4, 128)
    kv, rows = cpu_cache(shape), cpu_rows(shape)
    x = torch.zeros(4096, dtype=torch.float32)
    p = ctypes.c_void_p(x.data_ptr() // 256 * 256 + 256)
    st = ctypes.byref(kv.struct())
    seg = np.array([[0, 0, 1]], np.int32)
    plan = lambda handle, kvp, ws, n=1, nbytes=1 << 20: lib.orthrus_rows_plan(handle, kvp, ctypes.c_void_p(seg.ctypes.data), n, ws, nbytes, None)
    assert plan(None, st, p) == plan(rows.handle, None, p) == plan(rows.handle, st, None) == A.ORTHRUS_EINVAL
    assert plan(rows.handle, st, ctypes.c_void_p(p.value + 16)) == A.ORTHRUS_EINVAL       # not on 256 bytes
    assert plan(rows.handle, st, p, n=-1) == A.ORTHRUS_EINVAL
    assert plan(rows.handle, st, p, nbytes=64) == A.ORTHRUS_ECAPACITY
    # no plan yet
    assert lib.orthrus_kv8_append(rows.handle, st, 0, p, A.ORTHRUS_BF16, 2048, None, None, p, 1024, None) == A.ORTHRUS_EINVAL
    assert lib.orthrus_kv8_attend(rows.handle, st, 0, p, 1024, 0.0, p, 1024, None) == A.ORTHRUS_EINVAL
    assert lib.orthrus_kv8_read(rows.handle, st, 0, p, p, None) == A.ORTHRUS_EINVAL
    assert lib.orthrus_rows_create(None, ctypes.byref(ctypes.c_void_p())) == A.ORTHRUS_EINVAL
    assert lib.orthrus_rows_workspace_bytes(None, 1, 1, 1) == lib.orthrus_rows_workspace_bytes(rows.handle, -1, 1, 1) == 0
    lib.orthrus_rows_destroy(None)
    bad = kv.struct()
    bad.k_scale = None
    assert plan(rows.handle, ctypes.byref(bad), p) == A.ORTHRUS_EINVAL
    bad = kv.struct()
    bad.v_cache += 8
    assert plan(rows.handle, ctypes.byref(bad), p) == A.ORTHRUS_EINVAL


def test_caches_of_other_shapes_are_refused():
    shape = ops.HeadShape(8, 4, 128)
    kv = cpu_cache(shape)
    with code_of(A.ORTHRUS_EINVAL):
        ops.DeviceKV8.from_pools(shape, kv.k, kv.v.transpose(-1, -2), kv.k_scale, kv.v_scale, kv.block_table)
    with code_of(A.ORTHRUS_EINVAL):
        ops.DeviceKV8.from_pools(shape, kv.k, kv.v, kv.k_scale.double(), kv.v_scale, kv.block_table)
    with code_of(A.ORTHRUS_EINVAL):
        kv._fits(ops.HeadShape(8, 8, 128))


def test_score_refusals():
    lib = O.load()
    x = torch.zeros(4096, dtype=torch.float32)
    p = ctypes.c_void_p(x.data_ptr() // 16 * 16 + 16)
    call = lambda rows=1, vocab=8, stride=8, n=0, logits=p, tokens=p, lp=p, ids=None, tl=None, ws=None, nb=0: lib.orthrus_logprobs(
        logits, stride, rows, vocab, tokens, n, lp, None, None, ids, tl, ws, nb, None)
    for kw in (dict(rows=-1), dict(vocab=0), dict(n=-1), dict(n=9, ids=p), dict(vocab=100, stride=100, n=65, ids=p), dict(stride=7),
               dict(logits=None), dict(tokens=None), dict(ids=p), dict(tl=p), dict(vocab=70000, stride=70000)):
        assert call(**kw) == A.ORTHRUS_EINVAL, kw
    assert call(vocab=70000, stride=70000, ws=p, nb=16) == A.ORTHRUS_ECAPACITY
    assert call(rows=2 ** 31 - 1, vocab=70000, stride=70000, ws=p, nb=16) == A.ORTHRUS_ECAPACITY
    assert call(rows=0, logits=None) == A.ORTHRUS_OK
    b = lib.orthrus_logprobs_bytes
    assert b(0, 8, 1) == b(1, 0, 1) == b(1, 8, 9) == b(1, 8, -1) == b(1, 1000, 65) == 0
    assert b(300, 32000, 20) == b(1, 32000, 20) == 0 and b(1, 40000, 20) > 0 and b(300, 128000, 64) > 0
    with code_of(A.ORTHRUS_EINVAL):
        ops.logprobs(x[:16].view(2, 8).double())
    with code_of(A.ORTHRUS_EINVAL):
        ops.logprobs(x[:16].view(2, 8))                        # host tensors


def covered(shape, segs, counts, items):
    """Every (row, KV head) of the plan sees keys 0 .. its bound in pieces that do not overlap."""
    group = shape.n_q_heads // shape.n_kv_heads
    seen, slots, row = {}, [], 0
    first = {}
    for s, off, n in segs:
        first[s] = (row, off, n)
        row += n
    for i, (seq, r, n, pos, head, k0, k1, slot) in enumerate(items.tolist()):
        r0, off, total = first[seq]
        assert r0 <= r and r + n <= r0 + total and pos == off + r - r0 and 0 <= k0 < k1 <= pos + n
        small = i < counts[0]
        assert n * group <= (16 if small else 128) and small == (total * group <= 16)
        assert k0 % 64 == 0
        if slot >= 0:
            slots.append((slot, slot + (1 if small else 8)))
        seen.setdefault((r, n, head), []).append((k0, k1, slot))
    rows = np.zeros((row, shape.n_kv_heads), int)
    for (r, n, head), runs in seen.items():
        runs.sort()
        assert runs[0][0] == 0 and all(a[1] == b[0] for a, b in zip(runs, runs[1:]))
        s = next(s for s, (r0, off, m) in first.items() if r0 <= r < r0 + m)
        assert runs[-1][1] == first[s][1] + r - first[s][0] + n
        assert all((x[2] >= 0) == (len(runs) > 1) for x in runs)
        rows[r:r + n, head] += 1
    assert (rows == 1).all()
    slots.sort()
    assert all(a[1] <= b[0] for a, b in zip(slots, slots[1:])) and (not slots or slots[-1][1] <= counts[3])
    assert sum(len(v) > 1 for v in seen.values()) == counts[2]


@pytest.mark.parametrize("seed", range(12))
def test_plans_cover_every_key_once_and_fit_their_workspace(seed):
    rng = np.random.default_rng(seed)
    shape = ops.HeadShape(*[(4, 4, 64), (8, 2, 128), (28, 4, 128), (64, 8, 128), (16, 1, 128), (6, 2, 64)][seed % 6])
    n_seq = int(rng.integers(1, 40))
    kv = cpu_cache(shape, 1, n_seq, 12000)
    most = int(rng.choice([40, 3000, 150000]))
    segs = [(int(s), int(rng.integers(0, most)), int(rng.choice([1, 1, 2, 4, 17, 300]))) for s in rng.permutation(n_seq)]
    T, keys = sum(n for _, _, n in segs), max(o + n for _, o, n in segs)
    rows = cpu_rows(shape, T, n_seq, keys)
    counts, items = rows.items(kv, segs)
    covered(shape, segs, counts, items)
    units = sum((o + n - 1) // 16 - o // 16 + 1 for _, o, n in segs)
    meta = (144 + 5 * units + 8 * len(items) + 6 * counts[2]) * 4
    assert 256 + (meta + 255) // 256 * 256 + counts[3] * 16 * (shape.head_dim + 4) * 4 <= rows.nbytes


def test_long_ranges_come_in_pieces_and_short_ones_do_not():
    shape = ops.HeadShape(32, 8, 128)
    kv = cpu_cache(shape, 1, 300, 12000)
    rows = cpu_rows(shape, 300, 300, 150000)
    counts, _ = rows.items(kv, [(0, 150000, 1)])
    assert counts[0] >= 128 and counts[2] == 8
    counts, _ = rows.items(kv, [(s, 700, 1) for s in range(300)])
    assert counts[0] == 300 * 8 and counts[2] == counts[3] == 0
    assert rows.items(kv, [])[0] == [0, 0, 0, 0]


# ------------------------------------------------------------------ the definitions
def test_e4m3_definition_is_torchs():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    fine = codes[codes.isfinite()].double().numpy()
    np.testing.assert_array_equal(D.e4m3(fine), fine)
    x = np.concatenate([(fine[:-1] + fine[1:]) / 2, np.random.default_rng(0).uniform(-448, 448, 4000), 2.0 ** np.arange(-12, 9)])
    np.testing.assert_array_equal(D.e4m3(x), torch.tensor(x).float().to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.1, 1), (224.0, -1), (1.75, -8), (1.7500001, -7), (1.0, -8), (0.0, -100), (1e-40, -100)])
def test_page_scale(amax, e):
    assert D.page_scale(amax) == 2.0 ** e


def test_turn_keeps_pairs_lengths_and_tells_relative_positions():
    rng = np.random.default_rng(1)
    q, k, f = rng.normal(size=16), rng.normal(size=16), 10.0 ** -np.arange(4.0)
    for inter in (False, True):
        y = D.turn(q, 7, f, inter)
        np.testing.assert_array_equal(y[8:], q[8:])
        np.testing.assert_allclose(np.linalg.norm(y), np.linalg.norm(q))
        np.testing.assert_allclose(D.turn(q, 9, f, inter) @ D.turn(k, 5, f, inter), D.turn(q, 104, f, inter) @ D.turn(k, 100, f, inter))
    np.testing.assert_allclose(D.turn(q, 0, f, magnitude=2.0)[:8], 2 * q[:8])


def test_pages_keep_their_scale_while_they_fill_and_forget_at_their_start():
    c, table, one = D.Cache(2, 1, 4), [[1, 0]], lambda v: np.full((1, 1, 4), v)
    c.append(table, 0, 0, one(1.0), one(1.0))
    assert c.scale[0][1, 0] == 2.0 ** -8
    c.append(table, 0, 1, one(100.0), one(0.01))
    assert c.scale[0][1, 0] == 2.0 ** -2 and c.scale[1][1, 0] == 2.0 ** -8
    np.testing.assert_array_equal(c.rows(table, 0, 0, 2)[0][:, 0, 0], [1.0, 104.0 if abs(104 - 100) < abs(96 - 100) else 96.0])
    c.append(table, 0, 0, one(0.5), one(0.5))
    assert c.scale[0][1, 0] == 2.0 ** -9


def test_scores_definition():
    x = np.array([1.0, 3.0, -np.inf, 3.0, 0.0])
    lp, ent, rank, ids, tops = D.scores(x, 3, 3)
    p = np.exp(x - 3) / np.exp(x - 3).sum()
    assert rank == 1 and ids.tolist() == [1, 3, 0] and math.isclose(lp, math.log(p[3]))
    assert math.isclose(ent, -sum(v * math.log(v) for v in p if v > 0)) and np.allclose(tops, np.log(p[[1, 3, 0]]))


def test_work_beyond_one_launch_is_refused():
    """A launch has fewer than 2^32 threads: more rows times heads, or rows of logits, than it can serve."""
    shape = ops.HeadShape(8, 8, 64)
    kv = ops.DeviceKV8(shape, 1, 1, 1, 65537, device="cpu")
    rows = ops.RaggedRows(shape, 1, 1, 1, device="cpu")
    counts, _ = rows.items(kv, [(0, 0, 2 ** 20)])
    assert counts[1] == 8 * 2 ** 20 // 128 + counts[3] // 8 - counts[2]
    with code_of(A.ORTHRUS_ECAPACITY):
        rows.items(kv, [(0, 0, 2 ** 20 + 1)])
    x = torch.zeros(8)
    at = -(-x.data_ptr() // 16) * 16

    def call(p, n, vocab=1):
        return O.load().orthrus_logprobs(p, vocab, n, vocab, None, 0, None, None, None, None, None, None, 0, None)
    assert call(at, 2 ** 22) == call(at, 2 ** 31 - 1) == call(at, 2 ** 21, 60000) == A.ORTHRUS_ECAPACITY
    assert call(at + 2, 1) == A.ORTHRUS_EINVAL


def test_step_refusals():
    """orthrus_step_kv8 turns away what it cannot run before it touches a device."""
    from paper_2609_25405_amd import runtime as R
    from workload import Batch, DecodeRow, EmbChunk, draw_tokens, make_weights, tiny_config
    cfg = tiny_config("bf16")
    m = R.DeviceModel(cfg, make_weights(cfg, 1), device="cpu")
    shape = ops.HeadShape(4, 4, 64)
    kv = ops.DeviceKV8(shape, 2, 40, 6, 4, device="cpu")
    other = ops.DeviceKV8(shape, 2, 40, 6, 4, device="cpu")
    b = Batch([EmbChunk(0, 0, 5, True)], [DecodeRow(1, 9)], draw_tokens(1, 0, 6, cfg.vocab))
    n = O.load().orthrus_step_kv8_bytes(m.handle, m.handle, 6, 1, 1, 9)
    assert n > A.orthrus_workspace_bytes(m.handle, m.handle, 6, 1, 1, 9)
    assert O.load().orthrus_step_kv8_bytes(None, m.handle, 6, 1, 1, 9) == 0
    assert O.load().orthrus_step_kv8_bytes(m.handle, m.handle, 6, -1, 1, 9) == 0
    buf = torch.zeros(4096, dtype=torch.uint8)
    at = -(-buf.data_ptr() // 256) * 256
    out = torch.zeros(6, max(cfg.vocab, cfg.d_model))

    def call(e, g, ws=at, size=2048, batch=b):
        p = R.PackedBatch(batch)
        return O.load().orthrus_step_kv8(m.handle, m.handle, ctypes.byref(p.c), e and ctypes.byref(e), g and ctypes.byref(g),
                                         out.data_ptr(), out.data_ptr(), out.data_ptr(), out.data_ptr(), ws, size, None)

    def changed(**kw):
        s = kv.struct()
        for k, v in kw.items():
            setattr(s, k, v)
        return s

    good = kv.struct()
    assert call(good, good) == A.ORTHRUS_ECAPACITY                    # the workspace is too small: all else is in order
    assert call(good, kv.struct()) == A.ORTHRUS_ECAPACITY             # the same cache named twice
    assert call(good, other.struct()) == A.ORTHRUS_ECAPACITY
    assert call(None, good) == call(good, None) == A.ORTHRUS_EINVAL
    assert call(good, good, ws=at + 16) == call(good, good, ws=None) == A.ORTHRUS_EINVAL
    few = changed(n_layers=1)
    assert call(few, few) == A.ORTHRUS_EINVAL
    for kw in (dict(n_pages=39), dict(block_table=other.block_table.data_ptr()), dict(v_scale=other.v_scale.data_ptr()),
               dict(k_cache=other.k.data_ptr())):
        assert call(good, changed(**kw)) == A.ORTHRUS_EINVAL, kw
    for kw in (dict(k_scale=None), dict(v_cache=None), dict(k_cache=kv.k.data_ptr() + 4)):
        bad = changed(**kw)
        assert call(bad, bad) == A.ORTHRUS_EINVAL, kw
    twice = Batch([EmbChunk(1, 0, 5, True)], [DecodeRow(1, 9)], draw_tokens(1, 0, 6, cfg.vocab))
    assert call(good, good, batch=twice) == A.ORTHRUS_EDUPSEQ
    assert call(good, other.struct(), batch=twice) == A.ORTHRUS_ECAPACITY
    long = Batch([], [DecodeRow(1, 64)], draw_tokens(1, 0, 1, cfg.vocab))
    assert call(good, good, batch=long) == A.ORTHRUS_ECAPACITY
