"""Norms and products on the GPU: memory that streams hand to one another, in place calls, scales that no rounding makes, and
more work than small grids hold."""
import math

import numpy as np
import pytest
import torch

from paper_2609_25405_amd import linear as L
from tests.linear_common import check, host, mx_values, product_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu(request):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(f"\n[case] {request.node.name}", flush=True)


# ------------------------------------------------------------------------------ streams
@pytest.mark.parametrize("side", ["pool", "default"])
def test_weights_packed_on_another_stream(side):
    """Weights packed on a stream of the caller's, into memory that the current stream has just given back and still has a
    kernel queued on."""
    m = torch.randn((512, 1024), device="cuda").to(torch.bfloat16)
    want = L.LinearWeights(m).packed.clone()
    torch.cuda.synchronize()
    default = torch.cuda.default_stream()
    here, there = (default, torch.cuda.Stream()) if side == "pool" else (torch.cuda.Stream(), default)
    with torch.cuda.stream(here):
        for _ in range(3):
            block = torch.empty_like(want)
            torch.cuda._sleep(20_000_000)
            block.fill_(7)
            del block
            w = L.LinearWeights(m, stream=there.cuda_stream)
            torch.cuda.synchronize()
            assert torch.equal(w.packed, want)
            # dropped at once: the memory is not another's before it is packed
            torch.cuda._sleep(1)
            there.wait_stream(here)
            with torch.cuda.stream(there):
                torch.cuda._sleep(20_000_000)
            L.LinearWeights(m, stream=there.cuda_stream)
            after = torch.full_like(want, 9)
            torch.cuda.synchronize()
            assert (after == 9).all()


# ------------------------------------------------------------------------------ memory that arguments share
@pytest.mark.parametrize("width", [300, 301, 4096, 20000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("which", ["x", "add"])
def test_norm_in_place(width, dtype, which):
    """y over x or add, the total over the other one: the bits of the call that writes elsewhere."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(width)
    rows = 1500 if width < 1000 else 20
    a, b = (torch.randn((rows, width), generator=gen, device="cuda").to(dtype) for _ in range(2))
    y, total = torch.empty_like(a), torch.empty_like(a)
    L.norm(a, y, add=b, total=total)
    c, d = a.clone(), b.clone()
    L.norm(c, c if which == "x" else d, add=d, total=d if which == "x" else c)
    assert torch.equal(c if which == "x" else d, y) and torch.equal(d if which == "x" else c, total)


def test_columns_of_one_buffer():
    """x, residual and y side by side in the rows of one buffer share no byte."""
    room = torch.randn((200, 3 * 128), device="cuda").to(torch.bfloat16)
    before = room.clone()
    x, res, y = room[:, :128], room[:, 128:256], room[:, 256:]
    w = L.LinearWeights(torch.randn((128, 128), device="cuda").to(torch.bfloat16))
    L.linear(w, x, y, residual=res)
    apart = torch.empty((200, 128), dtype=torch.bfloat16, device="cuda")
    L.linear(w, x.contiguous(), apart, residual=res.contiguous())
    assert torch.equal(y, apart) and torch.equal(room[:, :256], before[:, :256])
    with pytest.raises(L.A.OrthrusError):
        L.linear(w, x, room[:, 64:192])


# ------------------------------------------------------------------------------ sizes
@pytest.mark.parametrize("rows,n,k,gated", [((1 << 28) + 5, 16, 16, False), ((1 << 20) + 3, 14336, 32, True)])
def test_millions_of_tiles(rows, n, k, gated):
    """More than 2^22 tiles of 16 weight rows by a workgroup's rows."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    x = torch.empty((rows, k), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    ws = [torch.randn((n, k), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(1 + gated)]
    y = torch.full((rows, n), -77.0, dtype=torch.bfloat16, device="cuda")
    w = L.LinearWeights(ws[0], up=ws[1] if gated else None)
    L.linear(w, x, y, act="silu" if gated else None, workspace=L.linear_workspace(w, rows))
    at = torch.tensor([0, 1, 255, 256, 65535, rows // 2, rows // 2 + 77, rows - 257, rows - 2, rows - 1], device="cuda")
    want, bound = product_bound(host(x[at]), host(ws[0]), host(ws[1]) if gated else None, None, "silu" if gated else None, None, "bf16")
    check(y[at], want, bound, (rows, n, k))


# ------------------------------------------------------------------------------ activations
# Bounds relative to the result, u = 2^-24 (a hardware exponential or reciprocal is off by 2 u at most).
# over 1 + exp(-a): the argument a log2(e) is rounded once and its constant by less than u / 2 of itself, 1.5 |a| u; exponential and
#   reciprocal 4 u, a sum and a product 2 u: (6 + 1.5 |a|) u.  The tanh form's argument takes five roundings more: 5 |a| u.
# gelu: q's polynomial 1.2e-7 = 2 u; nine steps of Horner, each at most the sum of the coefficients' magnitudes over the value,
#   0.93 / 0.5, off: 17 u; the reciprocal's 2 u (and its argument's u) through a slope of the logarithm of at most sum i |c_i| / 0.5 = 8: 24 u; two roundings
#   and the constant's of the exponent, v^2 / 2 of them each: 1.25 v^2 u; exponential, two products, a sum: 5 u.
@pytest.mark.parametrize("act,limit", [("silu", lambda v: 6 + 1.5 * np.abs(v)), ("gelu", lambda v: 48 + 1.25 * v * v),
                                       ("gelu_tanh", lambda v: 6 + 6.5 * 1.6 * np.abs(v + 0.044715 * v ** 3))])
@pytest.mark.parametrize("rows", [3, 70])
def test_activations_of_far_values(act, limit, rows):
    """Values from the bias alone, out to where the results are tiny: relative to the results."""
    n = 4096
    far = {"silu": 80, "gelu": 12.9, "gelu_tanh": 9}[act]
    v = np.linspace(-far, far, n).astype(np.float32)
    w = L.LinearWeights(torch.ones((n, 16), dtype=torch.bfloat16, device="cuda"))
    y = torch.empty((rows, n), device="cuda")
    L.linear(w, torch.zeros((rows, 16), dtype=torch.bfloat16, device="cuda"), y, bias=torch.tensor(v, device="cuda"), act=act, workspace=L.linear_workspace(w, rows))
    v = v.astype(np.float64)
    if act == "gelu":
        want = v * 0.5 * np.array([math.erfc(-c / math.sqrt(2)) for c in v])
    else:
        want = v / (1 + np.exp(-(v if act == "silu" else 2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))))
    got = host(y)
    assert (got == got[0]).all()
    off = np.abs(got[0] - want) / (limit(v) * 2.0 ** -24 * np.abs(want) + 1e-37)
    assert off.max() <= 1, (v[off.argmax()], off.max())
    print(act, "largest part of the bound", off.max())


# ------------------------------------------------------------------------------ scales of any byte
def blocks_of(codes, scales):
    """Mx8 of uint8 arrays."""
    to = lambda a: torch.tensor(np.ascontiguousarray(a), dtype=torch.uint8, device="cuda")
    return L.Mx8.of(to(codes).view(torch.float8_e4m3fn), to(scales))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_read_back_of_every_code_under_every_scale(dtype):
    """The value, rounded to the type read into: exact in fp32 under bytes up to 246, in bfloat16 under bytes 3 to 246."""
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.tile(np.arange(256, dtype=np.uint8)[:, None], (1, 8))
    m = blocks_of(codes, scales)
    y = torch.empty((256, 256), dtype=dtype, device="cuda")
    L.convert(m, y)
    code = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    exact = code[None] * 2.0 ** (np.arange(256, dtype=np.float64)[:, None] - 127)
    exact[255] = np.nan
    want = torch.tensor(exact).to(torch.float32).to(dtype).double().numpy()
    got = host(y)
    bad = ~((got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), [(int(r), hex(int(c)), got[r, c], want[r, c]) for r, c in np.argwhere(bad)[:5]]
    sure = slice(0 if dtype == torch.float32 else 3, 247)
    assert np.array_equal(got[sure], exact[sure], equal_nan=True)


@pytest.mark.parametrize("rows", [7, 80])
@pytest.mark.parametrize("a,b", [(0, 254), (254, 0), (1, 250), (100, 154), (3, 130), (246, 1)])
def test_products_under_far_scales(rows, a, b):
    """Scales of x and of the weights at the ends of their range, whose product is ordinary."""
    rng = np.random.default_rng(a)
    code = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    fine = np.flatnonzero(np.isfinite(code) & (np.abs(code) >= 2.0 ** -6) & (np.abs(code) < 16))
    cx, cw = (rng.choice(fine, (r, 160)).astype(np.uint8) for r in (rows, 48))
    x, m = blocks_of(cx, np.full((rows, 5), a)), blocks_of(cw, np.full((48, 5), b))
    y = torch.empty((rows, 48), device="cuda")
    w = L.LinearWeights(m)
    L.linear(w, x, y, workspace=L.linear_workspace(w, rows))
    scale = 2.0 ** (a + b - 254)
    want, bound = product_bound(code[cx], code[cw], None, None, None, None, "mx8")
    check(y, want * scale, bound * scale, (a, b))


# ------------------------------------------------------------------------------ wide rows
@pytest.mark.parametrize("width", [16384, 16385, 1 << 20, (1 << 24) + 3])
@pytest.mark.parametrize("value", [1.0, 1.0437, 1.3, None])
def test_norm_of_wide_rows(width, value):
    """A row's squares are sixteen or fewer additions in fp32 deep, four more between lanes, halved by the root; the factor's and the products'
    roundings are three: 2^-20 of the value (u = 2^-24), whatever the width.  Equal elements are the worst for longer sums, whose
    roundings then all fall on one side."""
    x = torch.full((2, width), value or 0.0, device="cuda")
    if value is None:
        x.normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    y = torch.empty_like(x)
    L.norm(x, y)
    s = x.double()
    want = s / (s.square().mean(-1, keepdim=True) + 1e-5).sqrt()
    assert ((y.double() - want).abs() <= 2.0 ** -20 * want.abs()).all(), float(((y.double() - want).abs() / want.abs()).max() * 2 ** 24)


def test_wide_rows_past_the_range():
    """Squares whose sum passes fp32's range make a row zero, not a number makes it so, of wide rows as of narrow ones."""
    for width in (4096, 40000):
        x = torch.ones((3, width), device="cuda")
        x[0], x[1, width - 1] = 1e20, float("nan")
        y = torch.full_like(x, 5.0)
        L.norm(x, y)
        assert (y[0] == 0).all() and y[1].isnan().all() and ((y[2] - 1).abs() < 1e-4).all()


@pytest.mark.parametrize("rows", [9, 200])
def test_blocks_read_back_give_exact_products(rows):
    """What the matrix cores cut of 8-bit products is all there in bfloat16 products of the same values."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows)
    n, k = 100, 1000
    x8, w8 = L.Mx8.empty(rows, k), L.Mx8.empty(n, k)
    for m in (x8, w8):
        L.convert(torch.randn(m.shape, generator=gen, device="cuda") * torch.exp(2 * torch.randn((1, k), generator=gen, device="cuda")), m)
    x, w = (torch.empty(m.shape, dtype=torch.bfloat16, device="cuda") for m in (x8, w8))
    L.convert(x8, x)
    L.convert(w8, w)
    y = torch.empty((rows, n), device="cuda")
    weights = L.LinearWeights(w)
    L.linear(weights, L.aligned(x), y, workspace=L.linear_workspace(weights, rows))
    check(y, *product_bound(mx_values(x8)[0], mx_values(w8)[0], None, None, None, None, "bf16"), rows)


@pytest.mark.parametrize("rows,k", [(5, 70), (90, 333)])
def test_rows_that_begin_anywhere_once_aligned(rows, k):
    """8-bit rows side by side without padding, refused as they lie, give the product of the same rows laid out."""
    m, w8 = L.Mx8.empty(rows, k), L.Mx8.empty(40, k)
    for t in (m, w8):
        L.convert(torch.randn(t.shape, device="cuda"), t)
    packed = L.Mx8(*[t.view(torch.uint8).contiguous().view(t.dtype) for t in (m.codes, m.scales)])
    w = L.LinearWeights(w8)
    y, z = (torch.empty((rows, 40), device="cuda") for _ in range(2))
    ws = L.linear_workspace(w, rows)
    L.linear(w, m, y, workspace=ws)
    with pytest.raises(L.A.OrthrusError):
        L.linear(w, packed, z, workspace=ws)
    L.linear(w, L.aligned(packed), z, workspace=ws)
    assert torch.equal(y, z)
