"""The norm's codes where they are hard to tell: rows made so that nearly every element of the definition lies within three steps of
fp32 of the middle between two codes, on either side, with sums that round.

An element's side is told by s, gain and a row's factor.  The kernel adds the squares in 64 bits and keeps the factor, the sum and the
products in two parts of fp32, whose ends are off by a few u^2 (u = 2^-24): elements nearer to a middle than 2^-40 are left out, of which
there is hardly one.  Plain fp32 (a sum, two products, a factor that rounds two or three times: about u in all) has thousands of the others on
the wrong side, which `test_plain_form_fails` shows on the CPU.
"""
import numpy as np
import pytest
import torch

from oracle import linear as D
from paper_2609_25405_amd import linear as L
from tests.linear_common import mx_values

U = 2.0 ** -24
WIDTHS = [(300, 400), (512, 200), (2048, 60), (4096, 60), (4104, 40), (8192, 30), (16384, 12), (20000, 10)]


def hard_rows(width, rows, add, seed=0):
    """x, add (or None), gain [width] a row, the definition, and which elements lie beside a middle."""
    rng = np.random.default_rng([seed, width, rows])
    f32 = lambda a: a.astype(np.float32)
    x = f32(rng.standard_normal((rows, width)) * np.exp(rng.standard_normal((1, width))))
    x += f32(np.where(np.abs(x) < 0.01, 0.5, 0.0))
    b = f32(rng.standard_normal((rows, width)) * 0.3) if add else None
    s = x.astype(np.float64) + (b.astype(np.float64) if add else 0.0)
    factor = 1 / np.sqrt((s * s).mean(-1, keepdims=True) + 1e-5)
    # middles between codes of three mantissa bits, and in each block one that holds its scale at 1
    middle = (1 + (2 * rng.integers(0, 8, (rows, width)) + 1) / 16) * 2.0 ** rng.integers(-6, 7, (rows, width))
    middle[:, ::32] = 300.0
    gain = f32(middle * (1 + 3 * U * rng.uniform(-1, 1, (rows, width))) / np.abs(s * factor))
    y = s * factor * gain.astype(np.float64)
    off = np.abs(np.abs(y) / middle - 1)
    hard = (off > 2.0 ** -40 + (U if add else 0)) & (off < 4 * U)
    hard[:, ::32] = False
    return x, b, gain, y, hard


def test_plain_form_fails():
    for width, rows in WIDTHS[:4]:
        x, b, gain, y, hard = hard_rows(width, rows, True)
        s = x + b
        m = (s * s).mean(-1, keepdims=True, dtype=np.float64).astype(np.float32) + np.float32(1e-5)
        plain = s * (np.float32(1) / np.sqrt(m)) * gain
        # the factor without an error, and one product rounded before it
        exact = 1 / np.sqrt((s.astype(np.float64) ** 2).mean(-1, keepdims=True) + 1e-5)
        once = ((s * gain).astype(np.float64) * exact).astype(np.float32)
        for form in (plain, once):
            wrong = (D.to_blocks(form)[0] != D.to_blocks(y)[0])[hard]
            assert hard.mean() > 0.4 and wrong.mean() > 0.002, (width, hard.mean(), wrong.mean())


@pytest.mark.gpu
@pytest.mark.parametrize("add", ["", "add", "in place"])
@pytest.mark.parametrize("width,rows", WIDTHS)
def test_codes_on_borders(width, rows, add):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(f"\n[case] {width} {rows} {add}", flush=True)
    x, b, gain, y, hard = hard_rows(width, rows, bool(add))
    t = lambda a: torch.tensor(a, device="cuda")
    tx, tb, out = t(x), t(b) if add else None, L.Mx8.empty(rows, width)
    for r in range(rows):       # a gain for each row
        at = slice(r, r + 1)
        one = L.Mx8(out.codes[at], out.scales[at])
        L.norm(tx[at], one, gain=t(gain[r]), add=tb[at] if add else None, total=(tx if r % 2 else tb)[at] if add == "in place" else None)
    values, scales = D.to_blocks(y)
    got, held = mx_values(out)
    assert np.array_equal(held, scales)
    wrong = (got != values) & hard
    assert not wrong.any(), (wrong.sum(), hard.sum(), np.argwhere(wrong)[:5])
    assert (np.abs(got - values) <= 2.0 ** -3 * np.abs(values)).all()
