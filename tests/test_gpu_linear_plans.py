"""Every kernel of the products, by the cover that a size takes: each shape of tiles, whole, with K cut and grouped, alone and in pairs of
weights, in both types, and the few-row kernel with each number of weight tiles.  That a size takes the cover it stands for is
checked here beside its results (and on the CPU alone), so that a change of the planner's constants cannot leave a kernel untested.  128 x
256 tiles with K cut are not listed: no size was found that takes them."""
import ctypes

import pytest
import torch

from paper_2609_25405_amd import _abi_linear as B
from tests.test_gpu_linear_covers import run
from tests.test_linear_edges_host import BF16, MX8, PackedShape, cover, packed_shape

TILES = {0: "256x256", 1: "128x256", 2: "128x128", 3: "64x128", 4: "64x256", -1: "few"}
# cover, kind, gated, rows, n, bytes of a row of K, groups
SIZES = [
    ("256x256", "whole", False, 3414, 2379, 69, 1), ("256x256", "whole", True, 1425, 2829, 65, 1), ("256x256", "whole", False, 2600, 5000, 600, 1),
    ("256x256", "cut", False, 1280, 4096, 14336, 1), ("256x256", "cut", True, 450, 4505, 8788, 1),
    ("256x256", "grouped", False, 2535, 2951, 67, 8), ("256x256", "grouped", True, 4344, 946, 65, 3), ("256x256", "grouped", False, 4000, 3000, 420, 2),
    ("128x256", "whole", False, 1846, 2248, 65, 1), ("128x256", "whole", True, 5537, 346, 66, 1), ("128x256", "whole", False, 1500, 4000, 600, 1),
    ("128x256", "grouped", False, 970, 3908, 65, 3), ("128x256", "grouped", True, 901, 2152, 73, 3),
    ("128x128", "whole", False, 5739, 274, 552, 1), ("128x128", "whole", True, 724, 1345, 516, 1),
    ("128x128", "cut", False, 5487, 18, 4834, 1), ("128x128", "cut", True, 74, 2906, 6966, 1),
    ("128x128", "grouped", False, 2589, 673, 564, 8), ("128x128", "grouped", True, 1903, 540, 520, 3),
    ("64x128", "whole", False, 17, 26, 64, 1), ("64x128", "whole", True, 17, 19, 66, 1), ("64x128", "whole", False, 200, 1000, 900, 1),
    ("64x128", "cut", False, 17, 17, 2238, 1), ("64x128", "cut", True, 23, 17, 2188, 1),
    ("64x128", "grouped", False, 37, 18, 68, 2), ("64x128", "grouped", True, 38, 20, 80, 2),
    ("64x256", "whole", False, 675, 5379, 1110, 1), ("64x256", "whole", True, 1080, 1817, 1086, 1),
    ("64x256", "cut", False, 143, 6402, 10804, 1), ("64x256", "cut", True, 1, 4126, 10330, 1), ("64x256", "cut", True, 17, 5703, 15924, 1),
    ("64x256", "grouped", False, 229, 684, 1110, 64), ("64x256", "grouped", False, 1280, 6144, 4096, 2), ("64x256", "grouped", True, 11, 7247, 1170, 3),
    ("few", "whole", False, 1, 18, 68, 1), ("few", "whole", True, 4, 16, 66, 1), ("few", "grouped", False, 2, 17, 78, 2), ("few", "grouped", True, 2, 18, 64, 2),
]


def of(dtype, gated, rows, n, row_bytes, groups):
    p = cover(dtype, rows, n, row_bytes // (1 if dtype == MX8 else 2), gated, groups)
    return TILES[p.shape], "cut" if p.splits > 1 else "whole" if groups == 1 else "grouped"


def test_sizes_take_every_cover():
    taken = set()
    for tiles, kind, gated, *size in SIZES:
        for dtype in (BF16, MX8):
            got = of(dtype, gated, *size)
            taken.add((*got, gated, dtype))
            assert got == (tiles, kind), (tiles, kind, gated, dtype, size, got)
    every = {(t, kind, gated, dtype) for t in TILES.values() for kind in ("whole", "cut", "grouped") for gated in (False, True) for dtype in (BF16, MX8)}
    assert every - taken == {(t, "cut", gated, dtype) for t in ("128x256", "few") for gated in (False, True) for dtype in (BF16, MX8)}


def offsets(rows, groups):
    """Ragged groups, some of them empty, rows ahead of the first and behind the last."""
    if groups == 1:
        return None
    if groups == 2:
        return [0, rows - rows // 5, rows]
    at = [min(rows, rows // 40 + (rows * g // groups if g % 4 else rows * (g - g % 2) // groups)) for g in range(groups)]
    return sorted(at) + [rows - rows // 50]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["mx8", "bf16"])
@pytest.mark.parametrize("tiles,kind,gated,rows,n,row_bytes,groups", SIZES)
def test_results_by_cover(tiles, kind, gated, rows, n, row_bytes, groups, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    t = MX8 if dtype == "mx8" else BF16
    print(f"\n[case] {tiles} {kind} {gated} {rows} {n} {row_bytes} {groups} {dtype}", flush=True)
    assert of(t, gated, rows, n, row_bytes, groups) == (tiles, kind)
    k = row_bytes // (1 if dtype == "mx8" else 2)
    for y in ("bf16", "f32", "mx8") if n >= 128 else ("bf16", "f32"):      # (blocks are sampled, of four or more)
        run(rows, n, k, dtype, gated, y, "silu" if gated else "gelu", offsets(rows, groups), seed=rows)


FEW = [(1, False, 100, "bf16"), (2, False, 6144, "bf16"), (4, False, 12300, "bf16"), (2, False, 100, "mx8"), (4, False, 12300, "mx8"), (2, True, 100, "f32"),
       (4, True, 6150, "f32"), (4, True, 100, "mx8")]


def few_tiles(dtype, rows, n, k, gated, y):
    f = B.load()["_ZN7orthrus9few_tilesERKNS_11PackedShapeEiiii"]
    f.restype, f.argtypes = ctypes.c_int, [ctypes.POINTER(PackedShape)] + [ctypes.c_int] * 4
    return f(packed_shape(dtype, n, k, gated), rows, 1, int(gated), {"bf16": BF16, "f32": 0, "mx8": MX8}[y])


def test_few_rows_take_every_number_of_weight_tiles():
    for nt, gated, n, y in FEW:
        for dtype in (BF16, MX8):
            for k in (20, 300, 1200):
                assert few_tiles(dtype, 9, n, k, gated, y) == nt and of(dtype, gated, 9, n, k * (1 if dtype == MX8 else 2), 1)[0] == "few", (nt, n, k, y)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["mx8", "bf16"])
@pytest.mark.parametrize("nt,gated,n,y", FEW)
@pytest.mark.parametrize("k", [20, 300, 1200])
def test_few_rows_by_weight_tiles(nt, gated, n, y, k, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(f"\n[case] few {nt} {gated} {n} {y} {k} {dtype}", flush=True)
    run(9, n, k, dtype, gated, y, "silu" if gated else "gelu_tanh")
