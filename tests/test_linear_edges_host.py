"""Norms and products on the CPU: calls whose tensors or sizes would have a kernel read or write what is not theirs, or what
another call holds.  No GPU work: every call below is rejected by host checks."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2609_25405_amd import _abi as A
from paper_2609_25405_amd import _abi_linear as B
from paper_2609_25405_amd import linear as L
from paper_2609_25405_amd import ops


def weights_of(n, k, groups=1, gated=False):
    """LinearWeights as a call on the host sees them: nothing is packed."""
    w = L.LinearWeights.__new__(L.LinearWeights)
    w._sizes, w._device = (n, k, groups, gated), -1
    return w


@pytest.mark.parametrize("workspace", [torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(64, dtype=torch.uint8)[::2],
                                       torch.zeros((4, 8)).t()])
def test_workspaces_whose_bytes_are_not_side_by_side_are_refused(workspace):
    x, y = torch.zeros((3, 64), dtype=torch.bfloat16), torch.zeros((3, 48), dtype=torch.bfloat16)
    with pytest.raises(A.OrthrusError, match="workspace"):
        L.linear(weights_of(48, 64), x, y, workspace=workspace)
    with pytest.raises(A.OrthrusError, match="workspace"):
        L.linear_grouped(weights_of(48, 64, 2), x, torch.zeros(3, dtype=torch.int32), y, workspace=workspace)
    with pytest.raises(A.OrthrusError, match="workspace"):
        ops.logprobs(torch.zeros((2, 8)), logprob=torch.zeros(2), workspace=workspace)


@pytest.mark.parametrize("name", ["codes", "scales", "shape"])
def test_rows_in_blocks_stay_what_they_were_made_of(name):
    """A call hands over the addresses that were taken when the object was made: none of its tensors can be exchanged."""
    m, other = L.Mx8.empty(3, 64, device="cpu"), L.Mx8.empty(5, 64, device="cpu")
    before = bytes(m._ref)
    with pytest.raises(AttributeError):
        setattr(m, name, getattr(other, name))
    assert bytes(m._ref) == before and m.shape == m.codes.shape == (3, 64)
    at = [int.from_bytes(before[8 * i:8 * i + 8], "little") for i in range(2)]
    assert at == [m.codes.data_ptr(), m.scales.data_ptr()]


@pytest.mark.parametrize("name", ["packed", "n", "k", "groups", "gated"])
def test_weights_stay_what_was_packed(name):
    w = weights_of(48, 64, 2, True)
    with pytest.raises(AttributeError):
        setattr(w, name, 1)
    assert (w.n, w.k, w.groups, w.gated) == (48, 64, 2, True)


# ------------------------------------------------------------------------------ shared memory
MEET = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include "linear.hpp"
using namespace orthrus;
int main() {
    srand(1);
    auto any = [](int lo, int hi) { return lo + rand() % (hi - lo + 1); };
    int meet = 0;
    for (int i = 0; i < 400000; ++i) {
        Runs r[2];
        bool held[2][600] = {};
        for (int k = 0; k < 2; ++k) {
            const int bytes = any(1, 9);
            r[k] = Runs{any(0, 90), bytes + any(0, 12), bytes, any(1, 9)};
            if (k == 1 && i % 2) r[1].stride = r[0].stride, r[1].bytes = any(1, (int)r[0].stride);
            for (int row = 0; row < (int)r[k].rows; ++row) memset(&held[k][(int)(r[k].at + row * r[k].stride)], 1, (size_t)r[k].bytes);
        }
        bool want = false;
        for (int b = 0; b < 600; ++b) want = want || (held[0][b] && held[1][b]);
        if (runs_meet(r[0], r[1]) != want || runs_meet(r[1], r[0]) != want) {
            for (int k = 0; k < 2; ++k) printf("%d + %d r, %d bytes, %d rows\n", (int)r[k].at, (int)r[k].stride, (int)r[k].bytes, (int)r[k].rows);
            return 1;
        }
        meet += want;
    }
    if (runs_meet(Runs{0, 4, 4, 9}, Runs{3, 4, 0, 9}) || runs_meet(Runs{0, 4, 4, 0}, Runs{0, 4, 4, 9})) return 2;
    printf("%d of 400000 meet\n", meet);
    return meet < 100000 || meet > 390000;
}
"""


def test_what_shares_a_byte(tmp_path):
    """Rows that share a byte are told from rows that lie between each other, against a map of all bytes."""
    (tmp_path / "meet.cpp").write_text(MEET)
    root = os.path.dirname(os.path.dirname(__file__))
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(root, "include"), "-I", os.path.join(root, "paper_2609_25405_amd", "csrc"),
                    str(tmp_path / "meet.cpp"), "-o", str(tmp_path / "meet")], check=True)
    r = subprocess.run([str(tmp_path / "meet")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


BF16, F32, MX8 = A.ORTHRUS_BF16, A.ORTHRUS_F32, B.ORTHRUS_MX8
AT = [(i + 1) << 24 for i in range(8)]          # addresses far apart that nothing reads


def rows(at=0, dtype=BF16, stride=64, scale=5, scale_stride=4, off=0):
    return B.orthrus_matrix(AT[at] + off, AT[scale] if dtype == MX8 else None, stride, scale_stride, dtype)


def ref(m):
    return None if m is None else ctypes.byref(m)


@pytest.mark.parametrize("x,y", [
    (rows(0), rows(0, MX8)), (rows(0), rows(1, MX8, scale=0)), (rows(0, F32), rows(0, MX8, off=700)), (rows(0, MX8), rows(0)),
    (rows(0, MX8), rows(5)), (rows(0, stride=128), rows(0, MX8, stride=192, off=64 * 2 - 1)), (rows(0), rows(1, MX8, scale=1)),
])
def test_conversions_within_shared_memory_are_refused(x, y):
    assert B.load().orthrus_convert(ref(x), ref(y), 8, 64, None) == A.ORTHRUS_EINVAL


@pytest.mark.parametrize("kw", [
    dict(y=rows(0, F32)), dict(y=rows(0, stride=72)), dict(y=rows(0, off=2)), dict(y=rows(0, MX8)), dict(y=rows(2, MX8, scale=0)),
    dict(add=rows(1), y=rows(1, F32)), dict(add=rows(1), y=rows(2, MX8, scale=1)), dict(add=rows(1), total=rows(1, F32)),
    dict(add=rows(1), total=rows(0, off=64)), dict(add=rows(1), total=rows(0), y=rows(0)), dict(total=rows(3), y=rows(3)),
    dict(total=rows(3), y=rows(3, MX8)), dict(total=rows(3, F32, off=16), y=rows(2, MX8, scale=3)), dict(y=rows(2, MX8, scale=2)),
    dict(gain=AT[2] + 60), dict(total=rows(3), gain=AT[3]), dict(y=rows(2, MX8), gain=AT[5] + 4),
])
def test_norms_within_shared_memory_are_refused(kw):
    a = dict(dict(x=rows(0), add=None, total=None, gain=None, y=rows(2)), **kw)
    assert B.load().orthrus_norm(ref(a["x"]), ref(a["add"]), ref(a["total"]), a["gain"], 1e-5, ref(a["y"]), 8, 64, None) == A.ORTHRUS_EINVAL


@pytest.mark.parametrize("kw", [
    dict(y=rows(0)), dict(y=rows(0, F32)), dict(y=rows(0, off=64, stride=128)), dict(y=rows(1, MX8, scale=0)), dict(y=rows(1, MX8, scale=1)),
    dict(y=rows(3)), dict(y=rows(1, MX8, scale=3)), dict(bias=AT[1] + 64), dict(res=rows(1, F32)), dict(res=rows(1, stride=80)),
    dict(res=rows(1, off=2)), dict(res=rows(1), y=rows(1, MX8)), dict(res=rows(5), y=rows(1, MX8)), dict(y=rows(4), groups=2, offsets=AT[4]),
    dict(y=rows(1, MX8), groups=2, offsets=AT[5]),
])
@pytest.mark.parametrize("mx", [False, True])
def test_products_within_shared_memory_are_refused(kw, mx):
    a = dict(dict(x=rows(0, MX8 if mx else BF16, scale=6), y=rows(1), res=None, bias=None, groups=1, offsets=None), **kw)
    w = B.orthrus_linear_weights(AT[3], MX8 if mx else BF16, 48, 64, 0, a["groups"])
    e = B.orthrus_epilogue(a["bias"], 0)
    if a["res"]:
        e.residual = a["res"]
    lib = B.load()
    if a["offsets"]:
        rc = lib.orthrus_linear_grouped(ref(w), ref(a["x"]), a["offsets"], 8, ref(e), ref(a["y"]), None, 0, None)
    else:
        rc = lib.orthrus_linear(ref(w), ref(a["x"]), 8, ref(e), ref(a["y"]), None, 0, None)
    assert rc == A.ORTHRUS_EINVAL


@pytest.mark.parametrize("where", ["x", "y", "scales", "weights", "bias", "residual"])
def test_workspaces_that_others_use_are_refused(where):
    R, N, K = 100, 48, 65536
    far = lambda i: (i + 1) << 32
    x = B.orthrus_matrix(far(0), far(1), K, K // 32, MX8)
    y, res = B.orthrus_matrix(far(2), None, N, 0, F32), B.orthrus_matrix(far(3), None, N, 0, BF16)
    w = B.orthrus_linear_weights(far(4), MX8, N, K, 0, 1)
    e = B.orthrus_epilogue(far(5), 0, res)
    lib = B.load()
    nbytes = lib.orthrus_linear_bytes(ref(w), R)
    at = {"x": far(0) + (R - 1) * K, "scales": far(1), "y": far(2) + 16, "residual": far(3), "weights": far(4) + 4096, "bias": far(5)}[where]
    assert nbytes > 0 and lib.orthrus_linear(ref(w), ref(x), R, ref(e), ref(y), at, nbytes, None) == A.ORTHRUS_EINVAL


def test_packing_over_its_own_matrices_is_refused():
    lib = B.load()
    for dtype in (BF16, MX8):
        w = B.orthrus_linear_weights(AT[0], dtype, 48, 64, 1, 2)
        for m, up in ((rows(0, dtype, off=64), rows(1, dtype)), (rows(1, dtype), rows(0, dtype, off=64))):
            assert lib.orthrus_linear_pack(ref(w), ref(m), ref(up), None) == A.ORTHRUS_EINVAL
    assert lib.orthrus_linear_pack(ref(w), ref(rows(1, MX8, scale=0)), ref(rows(2, MX8)), None) == A.ORTHRUS_EINVAL


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls below pass the host's checks")
def test_rows_that_share_nothing_pass():
    """The calls above, and rows that lie between each other or are the other's themselves: only the missing device ends them."""
    lib, passed = B.load(), A.ORTHRUS_EHIP
    convert = lambda x, y: lib.orthrus_convert(ref(x), ref(y), 8, 64, None)
    assert convert(rows(0), rows(1, MX8)) == passed and convert(rows(0, stride=256), rows(0, MX8, stride=512, off=128)) == passed
    norm = lambda x=rows(0), add=None, total=None, gain=None, y=rows(2): lib.orthrus_norm(ref(x), ref(add), ref(total), gain, 1e-5, ref(y), 8, 64, None)
    assert norm() == norm(y=rows(0)) == norm(add=rows(1), y=rows(1)) == norm(add=rows(0)) == passed
    assert norm(add=rows(1), total=rows(0)) == norm(add=rows(1), total=rows(1), y=rows(0)) == norm(gain=AT[2] - 256) == passed
    assert norm(x=rows(0, stride=128), y=rows(0, stride=128, off=128)) == norm(x=rows(0, stride=128), y=rows(0, F32, stride=64, off=128 + 8 * 256)) == passed
    for mx in (False, True):
        x, w = rows(0, MX8 if mx else BF16, scale=6, stride=128, scale_stride=8), B.orthrus_linear_weights(AT[3], MX8 if mx else BF16, 48, 64, 0, 1)
        linear = lambda y, res=None: lib.orthrus_linear(ref(w), ref(x), 8, ref(B.orthrus_epilogue(AT[4], 0, res or B.orthrus_matrix())), ref(y), None, 0, None)
        assert linear(rows(1)) == linear(rows(1), rows(1)) == linear(rows(1, MX8), rows(2)) == passed
        assert linear(rows(0, stride=128 // (1 + mx), off=128)) == (A.ORTHRUS_EINVAL if mx else passed)


# ------------------------------------------------------------------------------ sizes
@pytest.mark.parametrize("R,N,K,groups", [(1 << 30, 1, 1, 1), ((1 << 31) - 1, 1, 1, 1), ((1 << 31) - 1, 1, 1, 1 << 28), (3, (1 << 26) + 1, 64, 1),
                                          (3, (1 << 31) - 1, 64, 1), (3, (1 << 31) - 15, 64, 1), (3, 1, (1 << 22) + 1, 1), (3, 1, (1 << 31) - 1, 1),
                                          ((1 << 30) - 1, 2048, 64, 1), ((1 << 30) - 1, 64, 64, 1 << 27)])
def test_sizes_past_a_launch_are_refused(R, N, K, groups):
    lib = B.load()
    w = B.orthrus_linear_weights(1 << 40, BF16, N, K, 0, groups)
    x, y = B.orthrus_matrix(1 << 60, None, -(-K // 8) * 8, 0, BF16), B.orthrus_matrix(1 << 61, None, N, 0, BF16)
    args = [] if groups == 1 else [1 << 20]
    f = lib.orthrus_linear if groups == 1 else lib.orthrus_linear_grouped
    assert f(ref(w), ref(x), *args, R, None, ref(y), 1 << 59, 1 << 40, None) == A.ORTHRUS_ECAPACITY
    if K > 1 << 22 or N > 1 << 26:
        assert lib.orthrus_linear_packed_bytes(ref(w)) == lib.orthrus_linear_bytes(ref(w), 3) == 0
        assert lib.orthrus_linear_pack(ref(w), ref(B.orthrus_matrix(1 << 60, None, K, 0, BF16)), None, None) == A.ORTHRUS_ECAPACITY


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls below pass the host's checks")
@pytest.mark.parametrize("R,N,gated", [(1 << 20, 14336, 1), (1 << 28, 16, 0), (4 << 20, 14336, 0), (200000, 1 << 20, 0)])
def test_sizes_that_a_launch_holds_pass(R, N, gated):
    w = B.orthrus_linear_weights(1 << 40, BF16, N, 64, gated, 1)
    x, y = B.orthrus_matrix(1 << 60, None, 64, 0, BF16), B.orthrus_matrix(1 << 61, None, N, 0, BF16)
    assert B.load().orthrus_linear(ref(w), ref(x), R, None, ref(y), None, 0, None) == A.ORTHRUS_EHIP


class PackedShape(ctypes.Structure):
    _fields_ = [("tiles", ctypes.c_int), ("steps", ctypes.c_int), ("quads", ctypes.c_int), ("tile_bytes", ctypes.c_size_t),
                ("scale_at", ctypes.c_size_t), ("bytes", ctypes.c_size_t)]


class ProductPlan(ctypes.Structure):
    _fields_ = [("shape", ctypes.c_int), ("splits", ctypes.c_int), ("m_tiles_most", ctypes.c_int)]


def packed_shape(dtype, n, k, gated):
    tiles, steps = -(-n // 16) * (2 if gated else 1), -(-k * (1 if dtype == MX8 else 2) // 128)
    at = tiles * steps * 2048
    return PackedShape(tiles, steps, -(-tiles // 4), steps * 2048, at, at + (-(-tiles // 4) * steps * 256 if dtype == MX8 else 0))


def cover(dtype, rows, n, k, gated=False, groups=1):
    """The cover that a product takes (shape of tiles or -1, parts of K)."""
    f = B.load()["_ZN7orthrus12plan_productERKNS_11PackedShapeEiib"]
    f.restype, f.argtypes = ProductPlan, [ctypes.POINTER(PackedShape), ctypes.c_int, ctypes.c_int, ctypes.c_bool]
    return f(packed_shape(dtype, n, k, gated), rows, groups, groups == 1)


@pytest.mark.parametrize("dtype", [BF16, MX8])
@pytest.mark.parametrize("n", [1, 48, 1000, 4096, 14336, 32000, 200000])
@pytest.mark.parametrize("gated", [0, 1])
def test_workspaces_hold_every_smaller_call_and_only_cut_sums_need_one(dtype, n, gated):
    cut = 0
    for k in (64, 400, 1000, 4096, 14336, 65536):
        w = B.orthrus_linear_weights(None, dtype, n, k, gated, 1)
        room = lambda rows: B.load().orthrus_linear_bytes(ref(w), rows)
        shape, most = packed_shape(dtype, n, k, gated), 0
        for rows in list(range(1, 70)) + list(range(70, 700, 37)) + [1024, 1280, 2000, 4096, 5000, 8192, 100000]:
            plan = cover(dtype, rows, n, k, gated)
            if plan.splits > 1:
                most = max(most, plan.splits * rows * shape.tiles * 64)
                cut += 1
            assert most <= room(rows) <= 64 << 20, (k, rows)
        if shape.steps < 8 or n > 150000:            # parts of fewer than four steps, or more tiles than two rounds: never cut
            assert room(8192) == room(1) == 0
    assert cut > 0 or n > 20000


# ------------------------------------------------------------------------------ where rows begin
@pytest.mark.parametrize("rows,width,pad,off", [(3, 64, 0, 0), (3, 128, 0, 0), (1, 33, 3, 0), (4, 130, 6, 0), (4, 128, 16, 16), (4, 100, 12, 4), (5, 1, 0, 0)])
def test_aligned_rows_are_the_same_or_a_copy(rows, width, pad, off):
    nb = -(-width // 32)
    codes = torch.arange(rows * (width + pad + off), dtype=torch.uint8).view(rows, -1)[:, off:off + width].view(torch.float8_e4m3fn)
    scales = torch.arange(rows * (nb + pad), dtype=torch.uint8).view(rows, -1)[:, :nb].view(torch.float8_e8m0fnu)
    m = L.Mx8(codes, scales)
    a = L.aligned(m)
    assert torch.equal(a.codes.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(a.scales.view(torch.uint8), scales.view(torch.uint8))
    for t, kept, to in ((a.codes, codes, 16), (a.scales, scales, 4)):
        fits = lambda t: t.data_ptr() % to == 0 and (rows == 1 or t.stride(0) % to == 0)
        assert fits(t) and (t.data_ptr() == kept.data_ptr()) == fits(kept)
    assert L.aligned(a) is a
    b = torch.zeros((rows, width + 1), dtype=torch.bfloat16)[:, 1:]
    assert L.aligned(b).data_ptr() % 16 == 0 and L.aligned(L.aligned(b)).shape == b.shape
