"""Scores of tokens under logits against the float64 definition.

Bounds: x - m is one rounding of the difference (2^-24 of up to 2^7 here: 2^-17 in the exponent at worst, but such
terms weigh e^-|x - m|), the exponential and each sum's 2^-24 per addition on a path of at most 32 + 6 + 16 additions:
log Z errs by less than 2^-18; logprob adds the rounding of its own size (2^-23 of it), and the entropy a sum of
e (x - m) whose terms are at most 1/e of Z each: 2^-17 (1 + entropy).
"""
import math

import numpy as np
import pytest
import torch

from oracle import kv8 as D
from paper_2609_25405_amd import _abi as A
from paper_2609_25405_amd import ops, runtime as R

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu(request):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(f"\n[case] {request.node.name}", flush=True)


def call(x, tok, n, ws_extra=0):
    Rr, V = x.shape
    o = dict(logprob=torch.full((Rr,), 5.0, device="cuda"), entropy=torch.full((Rr,), 5.0, device="cuda"),
             rank=torch.full((Rr,), 77, dtype=torch.int32, device="cuda"))
    if n:
        o.update(top_ids=torch.full((Rr, n), -7, dtype=torch.int32, device="cuda"), top_logprobs=torch.full((Rr, n), 5.0, device="cuda"))
    ops.logprobs(x, tok, workspace=ops.logprobs_workspace(Rr, V, n), **o)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in o.items()}


def check(x, tok, n, some=None):
    o = call(x, tok, n)
    xs, ts = x.cpu().numpy(), tok.cpu().numpy()
    for r in some if some is not None else range(len(xs)):
        lp, ent, rank, ids, tops = D.scores(xs[r], ts[r], n)
        if math.isinf(lp):
            assert o["logprob"][r] == lp
        else:
            assert abs(o["logprob"][r] - lp) <= 2.0 ** -18 + 2.0 ** -23 * abs(lp), r
        assert abs(o["entropy"][r] - ent) <= 2.0 ** -17 * (1 + ent), r
        assert o["rank"][r] == rank
        if n:
            np.testing.assert_array_equal(o["top_ids"][r], ids)
            fine = np.isfinite(tops)
            assert (np.abs(o["top_logprobs"][r] - tops)[fine] <= 2.0 ** -18 + 2.0 ** -23 * np.abs(tops[fine])).all()
            np.testing.assert_array_equal(o["top_logprobs"][r][~fine], tops[~fine])
    return o


@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 64, 65, 500, 1023, 1024, 1025, 4097, 8190, 8191, 8193, 32000, 32765, 32766, 32768, 50001, 131072])
@pytest.mark.parametrize("n", [0, 1, 5, 64])
def test_sizes(vocab, n):
    rng = np.random.default_rng(vocab + n)
    rows = 3 if vocab > 5000 else 9
    x = torch.tensor(rng.normal(size=(rows, vocab)) * 3, dtype=torch.float32, device="cuda")
    tok = torch.tensor(rng.integers(0, vocab, rows), dtype=torch.int32, device="cuda")
    tok[0] = x[0].argmax()
    check(x, tok, min(n, vocab))


@pytest.mark.parametrize("rows,vocab", [(300, 32000), (257, 4099), (600, 513), (300, 70001)])
def test_many_rows(rows, vocab):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((rows, vocab), generator=g, device="cuda") * 2.5
    tok = torch.randint(0, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
    check(x, tok, 20, some=range(0, rows, 37))
    out = torch.empty(rows, dtype=torch.int32, device="cuda")
    R.sample_greedy(x, out)
    assert np.array_equal(call(x, tok, 2)["top_ids"][:, 0], out.cpu().numpy())


@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("vocab", [5, 1000, 33000])
def test_strides_and_alignments(shift, vocab):
    rng = np.random.default_rng(shift)
    buf = torch.full((4, vocab + 6), float("nan"), device="cuda")
    x = buf[:, shift:shift + vocab]
    x.copy_(torch.tensor(rng.normal(size=(4, vocab)) * 4))
    check(x, torch.tensor(rng.integers(0, vocab, 4), dtype=torch.int32, device="cuda"), 4)


@pytest.mark.parametrize("vocab", [100, 9000, 40000])
def test_ties_masks_and_order(vocab):
    """Equal entries rank by index; -inf entries count for nothing; ascending, descending and constant rows;
    signed zeros are equal; one entry far above all others; all but one masked."""
    rng = np.random.default_rng(vocab)
    x = np.zeros((9, vocab), np.float32)
    x[0] = rng.integers(0, 3, vocab)
    x[1] = np.arange(vocab) / vocab
    x[2] = -np.arange(vocab) / vocab
    x[4] = np.where(rng.random(vocab) < 0.9, -np.inf, rng.normal(size=vocab))
    x[4, 17] = 1.0
    x[5] = np.where(rng.random(vocab) < 0.5, 0.0, -0.0)
    x[6, vocab // 2] = 90.0
    x[7] = -np.inf
    x[7, vocab - 1] = 2.0
    x[8] = np.finfo(np.float32).min
    x[8, 3] = 0.0
    tok = torch.tensor([vocab - 1, 0, vocab - 1, vocab // 2, 17, vocab - 2, vocab // 2, vocab - 1, 5], dtype=torch.int32, device="cuda")
    check(torch.tensor(x, device="cuda"), tok, 33)
    # a masked token: log probability -inf, behind every entry that is not, by index among the masked
    o = call(torch.tensor(x[7:8], device="cuda"), torch.tensor([4], dtype=torch.int32, device="cuda"), 3)
    assert o["logprob"][0] == -np.inf and o["rank"][0] == 5 and o["top_ids"][0].tolist() == [vocab - 1, 0, 1]


@pytest.mark.parametrize("vocab", [60, 20000, 66000])
def test_rows_without_a_distribution(vocab):
    x = torch.randn((5, vocab), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    x[0] = -float("inf")
    x[1, 11] = float("nan")
    x[2, 12] = float("inf")
    x[3, 5], x[3, 50] = float("nan"), -float("nan")
    tok = torch.tensor([7, 11, 3, 50, 1], dtype=torch.int32, device="cuda")
    o = call(x, tok, 3)
    for k in ("logprob", "entropy"):
        assert np.isnan(o[k][:4]).all() and np.isfinite(o[k][4]), k
    assert np.isnan(o["top_logprobs"][:4]).all()
    assert o["rank"].tolist()[:2] == [7, 0] and o["rank"][3] == 1
    assert o["top_ids"][0].tolist() == [0, 1, 2] and o["top_ids"][1][0] == 11 and o["top_ids"][2][0] == 12 and o["top_ids"][3][:2].tolist() == [5, 50]


def test_tokens_outside_the_vocabulary_and_absent_outputs():
    x = torch.randn((4, 3000), device="cuda")
    tok = torch.tensor([-1, 3000, 2 ** 31 - 1, 5], dtype=torch.int32, device="cuda")
    o = call(x, tok, 2)
    assert np.isnan(o["logprob"][:3]).all() and (o["rank"][:3] == -1).all() and np.isfinite(o["logprob"][3])
    ent, ids = torch.empty(4, device="cuda"), torch.empty((4, 2), dtype=torch.int32, device="cuda")
    ws = ops.logprobs_workspace(4, 3000, 2)
    ops.logprobs(x, entropy=ent, top_ids=ids, workspace=ws)
    assert np.array_equal(ent.cpu().numpy(), o["entropy"]) and np.array_equal(ids.cpu().numpy(), o["top_ids"])
    ops.logprobs(x[:0], tok[:0], logprob=ent[:0])


def test_small_workspace_is_refused():
    x = torch.zeros((1, 70000), device="cuda")
    with pytest.raises(A.OrthrusError, match=r"\(-4\)"):
        ops.logprobs(x, entropy=torch.empty(1, device="cuda"), workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("rows,vocab", [(2, 32000), (40, 1000)])
def test_captured_and_replayed(rows, vocab):
    x = torch.zeros((rows, vocab), device="cuda")
    tok = torch.arange(rows, dtype=torch.int32, device="cuda")
    lp, ids, tl = torch.empty(rows, device="cuda"), torch.empty((rows, 6), dtype=torch.int32, device="cuda"), torch.empty((rows, 6), device="cuda")
    ws = ops.logprobs_workspace(rows, vocab, 6)
    run = lambda: ops.logprobs(x, tok, logprob=lp, top_ids=ids, top_logprobs=tl, workspace=ws)
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for i in range(4):
        x.copy_(torch.randn((rows, vocab), device="cuda") * (i + 1))
        g.replay()
        got = [t.clone() for t in (lp, ids, tl)]
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (lp, ids, tl)))
