"""Scores of rows with large, far apart and masked logits, against the float64 definition (bounds as in
test_gpu_logprobs.py: an entry's distance from the largest is one rounding, and entries far below weigh nothing)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_logprobs import call, check

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu(request):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(f"\n[case] {request.node.name}", flush=True)


def tokens(*t):
    return torch.tensor(t, dtype=torch.int32, device="cuda")


VOCABS = [100, 1003, 9000, 32000, 70001]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("top", [2.0 ** 124, 2.0 ** 126, 2.0 ** 127, 1e30, 3e38])
def test_one_logit_far_above_ordinary_ones(vocab, top):
    """Its row's entropy is zero, wherever among the entries it stands; so with all others far below."""
    rng = np.random.default_rng(vocab)
    at = [0, 1, vocab // 3, vocab - 2, vocab - 1, vocab // 2]
    x = rng.normal(size=(6, vocab)) * 2
    x[5] = -2e37
    x[range(6), at] = top
    check(torch.tensor(x, dtype=torch.float32, device="cuda"), tokens(0, 1, 5, vocab - 2, 3, 7), 3)


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("mask", [-1e9, -2.9e9, -6.4e9, -1e10, -1e30, -3e38])
def test_finite_masks(vocab, mask):
    """Most entries at a finite mask: scattered, all but a short run (whole threads, and slices of a long row, hold masked
    entries alone), none but one left, and nothing but the mask."""
    rng = np.random.default_rng(7)
    x = rng.normal(size=(5, vocab)) * 3
    x[0, rng.random(vocab) < 0.9] = mask
    x[1, :vocab - 70] = mask
    x[2, 70:] = mask
    x[3] = mask
    x[3, vocab // 2] = 1.5
    x[4] = mask
    x[0, 11] = 2.0
    check(torch.tensor(x, dtype=torch.float32, device="cuda"), tokens(11, vocab - 5, 3, vocab // 2, vocab - 1), 9)


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("base", [1e9, -2.9e9, 6.4e9, 1e30, -1e38, 3.4e38])
def test_large_logits_close_together(vocab, base):
    """Rows whose entries are a few steps of fp32 apart, or all the same."""
    rng = np.random.default_rng(3)
    b = np.float32(base)
    x = np.full((3, vocab), b)
    x[0] = b - np.abs(np.spacing(b)) * rng.integers(0, 3, vocab).astype(np.float32)
    x[2, vocab // 2] = b - 64 * np.abs(np.spacing(b))
    check(torch.tensor(x, device="cuda"), tokens(vocab - 1, 0, vocab // 2), 5)


@pytest.mark.parametrize("vocab", [5, 1003, 20000, 66000])
def test_a_row_whose_first_logit_is_not_a_number(vocab):
    x = torch.randn((3, vocab), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    x[0, 0] = float("nan")
    x[1, 0], x[1, 3] = -float("nan"), float("nan")
    o = call(x, tokens(0, 3, 0), 3)
    rest = x[0].cpu().numpy().copy()
    rest[0] = -np.inf
    assert o["top_ids"][0].tolist() == [0] + np.argsort(-rest, kind="stable")[:2].tolist()
    assert o["top_ids"][1][:2].tolist() == [0, 3] and o["rank"].tolist()[:2] == [0, 1]
    assert np.isnan(o["logprob"][:2]).all() and np.isfinite(o["logprob"][2])
