"""The mixed step through 8-bit caches, with the sampler and the token scores behind it, against the float64 oracle.

An e4m3 value next to a rounding boundary may fall either way, so the oracle does not round by itself: every key and
value that it writes is compared with what the device holds at its place, and later rows read what the device holds.
Bounds: of a held value half a step of e4m3 (2^-4 of the value, 2^-10 of the page's scale where that is coarser) and
the step's own bound on stored head vectors (tests/parity.py: the projection's arithmetic, relative to the vector's
largest entry), which passes through the rounding (times 1 + 2^-4); logits, embeddings and pooling states the step's
own bounds, since attention over the held values errs by no more than over a bfloat16 or fp32 cache.
"""
import numpy as np
import pytest
import torch

from oracle import OracleKV, step_oracle
from oracle import kv8 as D
from paper_2609_25405_amd import _abi as A
from paper_2609_25405_amd import ops
from paper_2609_25405_amd import runtime as R
from tests.parity import TOL, TOL_STATE, assert_vectors_close
from workload import Batch, DecodeRow, EmbChunk, GenChunk, as_float64, draw_tokens, make_lora, make_weights, tiny_config

pytestmark = pytest.mark.gpu
PAGE = 16


@pytest.fixture(autouse=True)
def _need_gpu(request):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(f"\n[case] {request.node.name}", flush=True)


class Held(OracleKV):
    """What the device holds after a step, read back by the oracle; what the oracle writes is compared with it."""

    def __init__(self, cfg, kv, table):
        s = lambda t: t.double().cpu().numpy()[..., None, None]
        k = kv.k.float().cpu().numpy() * s(kv.k_scale)
        v = kv.v.float().cpu().numpy().transpose(0, 1, 2, 3, 6, 5, 4)       # [.., slot / 4, slot % 4, dim / 16, dim % 16]
        v = v.reshape(*v.shape[:3], PAGE, cfg.head_dim) * s(kv.v_scale)
        super().__init__(k, v, table, PAGE)
        self.scales = s(kv.k_scale)[..., 0], s(kv.v_scale)[..., 0]
        self.rel = TOL_STATE[cfg.dtype]["rel"]

    def write(self, layer, seq, positions, k_rows, v_rows):
        pages, offs = self.slots(seq, positions)
        for pool, scale, x in ((self.k, self.scales[0], k_rows), (self.v, self.scales[1], v_rows)):
            held, sc = pool[layer, pages, :, offs, :], scale[layer, pages]
            err = self.rel * np.abs(x).max(axis=-1, keepdims=True) * (1 + 2.0 ** -4)
            assert np.all(np.abs(held - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * sc + err), (layer, seq)


class Served:
    """Models, caches and states of a run, stepped on the device and by the oracle."""

    def __init__(self, dtype, two_models=False, two_caches=False, n_seq=8, max_blocks=24, max_tokens=700, cfg=None, lora=0):
        cfg = self.cfg = cfg or tiny_config(dtype).replace(n_kv_heads=2)
        self.W = [make_weights(cfg, 301), make_weights(cfg, 302, model_tag=1) if two_models else None]
        if lora:
            self.W[0]["adapters"] = [make_lora(cfg, 303, 16, tag=t) for t in range(lora)]
        self.dm = [R.DeviceModel(cfg, self.W[0])]
        self.dm.append(R.DeviceModel(cfg, self.W[1]) if two_models else self.dm[0])
        e = (cfg, as_float64(self.W[0]))
        self.ref = [e, (cfg, as_float64(self.W[1])) if two_models else e]
        shape = ops.HeadShape(cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, dtype)
        rng = np.random.default_rng(5)
        self.kv, self.table = [], []
        for _ in range(1 + two_caches):
            n = n_seq * max_blocks + 3
            kv = ops.DeviceKV8(shape, cfg.n_layers, n, n_seq, max_blocks)
            t = rng.permutation(n)[:n_seq * max_blocks].reshape(n_seq, max_blocks).astype(np.int32)
            kv.set_block_table(t)
            kv.k.view(torch.uint8).fill_(0x7f)
            kv.v.view(torch.uint8).fill_(0xff)
            kv.k_scale.fill_(float("nan"))
            kv.v_scale.fill_(float("nan"))
            self.kv.append(kv)
            self.table.append(t)
        self.kv, self.table = (self.kv * 2)[:2], (self.table * 2)[:2]
        self.S, self.Wsum = np.zeros((n_seq, cfg.d_model)), np.zeros(n_seq)
        self.acc_sum = torch.zeros((n_seq, cfg.d_model), device="cuda")
        self.acc_w = torch.zeros(n_seq, device="cuda")
        self.ws = ops.WorkspaceKV8(*self.dm, max_tokens, 8, 8, max_blocks * PAGE)

    def enqueue(self, batch, stream=None, hidden=None):
        """(logits, sampled tokens, their scores, embeddings) of one step."""
        nc, nd = len(batch.chunks), batch.n_logit_rows
        logits = torch.full((max(1, nd), self.cfg.vocab), float("nan"), device="cuda")
        emb = torch.full((max(1, nc), self.cfg.d_model), float("nan"), device="cuda")
        ops.step_kv8(*self.dm, batch, *self.kv, self.acc_sum, self.acc_w, logits, emb, self.ws, stream=stream, hidden=hidden)
        logits, tok = logits[:nd], torch.full((nd,), -1, dtype=torch.int32, device="cuda")
        out = dict(logprob=torch.zeros(nd, device="cuda"), entropy=torch.zeros(nd, device="cuda"),
                   rank=torch.full((nd,), -1, dtype=torch.int32, device="cuda"),
                   top_ids=torch.full((nd, 3), -1, dtype=torch.int32, device="cuda"), top_logprobs=torch.zeros((nd, 3), device="cuda"))
        if nd:
            R.sample_greedy(logits, tok, stream=stream)
            ops.logprobs(logits, tok, workspace=ops.logprobs_workspace(nd, self.cfg.vocab, 3), stream=stream, **out)
        return logits, tok, out, emb

    def step(self, batch):
        hidden = None
        if batch.hidden_stride:
            hidden = torch.full((self.kv[0].n_seq, batch.hidden_stride, self.cfg.d_model), float("nan"), device="cuda")
        logits, tok, out, emb = self.enqueue(batch, hidden=hidden)
        torch.cuda.synchronize()
        assert self.ws.device_error() == 0
        held = [Held(self.cfg, kv, t) for kv, t in zip(self.kv, self.table)]
        if self.kv[0] is self.kv[1]:
            held[1] = held[0]
        ref = step_oracle(*self.ref, batch, *held, self.S, self.Wsum)
        dt = self.cfg.dtype
        if len(logits):
            print("logits", assert_vectors_close(logits.cpu().numpy(), ref["logits"], dt, "logits", TOL), flush=True)
            assert (tok.cpu().numpy() == logits.argmax(1).cpu().numpy()).all()
            for i, row in enumerate(logits.double().cpu().numpy()):
                lp, ent, rank, ids, top = D.scores(row, int(tok[i]), 3)
                # fp32 sums of a row: at most 2^-16 of a logarithm, whose size is at most ln(vocab) here
                b = 2.0 ** -16 * np.log(self.cfg.vocab)
                assert abs(float(out["logprob"][i]) - lp) <= b and abs(float(out["entropy"][i]) - ent) <= b
                assert int(out["rank"][i]) == rank == 0 and out["top_ids"][i].tolist() == ids.tolist()
                assert np.abs(out["top_logprobs"][i].double().cpu().numpy() - top).max() <= b
        for i, c in enumerate(batch.chunks):
            if c.pool == "buffer":
                assert_vectors_close(hidden[c.seq, c.offset:c.offset + c.len].cpu().numpy(), ref["hidden"][i], dt, "buffered rows")
            elif c.last:
                assert_vectors_close(emb[i].cpu().numpy(), ref["out_emb"][i], dt, "embedding")
            else:
                assert torch.isnan(emb[i]).all()
        np.testing.assert_array_equal(self.acc_w.double().cpu().numpy(), ref["acc_w"])
        live = [s for s in sorted({c.seq for c in batch.chunks if c.pool != "none"}) if np.any(ref["acc_sum"][s])]
        if live:
            assert_vectors_close(self.acc_sum[live].cpu().numpy(), ref["acc_sum"][live], dt, "pooling state")
        self.S, self.Wsum = ref["acc_sum"], ref["acc_w"]
        return tok.cpu().numpy()


def batch_of(vocab, tag, chunks=(), gen=(), rows=(), decode_ids=()):
    n = sum(c.len for c in chunks) + sum(c.len for c in gen)
    ids = np.concatenate([draw_tokens(77, tag, n, vocab) if n else np.zeros(0, np.int32), np.asarray(decode_ids, np.int32)])
    return Batch(list(chunks), list(rows), ids.astype(np.int32), gen_chunks=list(gen))


@pytest.mark.parametrize("dtype,two_models,two_caches", [("bf16", False, False), ("f32", False, False), ("f32", False, True),
                                                         ("f32", True, False), ("bf16", True, True)])
def test_serving_run(dtype, two_models, two_caches):
    """Chunks, prompts and decoded tokens over five steps: segments that begin and end inside pages, one-token
    segments, steps of one kind, a second request in a sequence that another left."""
    m = Served(dtype, two_models, two_caches)
    v = m.cfg.vocab
    a = m.step(batch_of(v, 1, [EmbChunk(0, 0, 37, False, "mean"), EmbChunk(1, 0, 1, True, "last")],
                        [GenChunk(3, 0, 21, True), GenChunk(4, 0, 33, False)]))
    b = m.step(batch_of(v, 2, [EmbChunk(0, 37, 150, True, "mean"), EmbChunk(2, 0, 16, False, "cls")],
                        [GenChunk(4, 33, 200, True), GenChunk(5, 0, 1, True)], [DecodeRow(3, 21)], a))
    assert len(b) == 3
    c = m.step(batch_of(v, 3, [EmbChunk(2, 16, 1, True, "cls")], [], [DecodeRow(4, 233), DecodeRow(5, 1), DecodeRow(3, 22)], b))
    m.step(batch_of(v, 4, [], [], [DecodeRow(5, 2), DecodeRow(4, 234), DecodeRow(3, 23)], c[[1, 0, 2]]))
    m.step(batch_of(v, 5, [EmbChunk(0, 0, 24, True, "mean"), EmbChunk(1, 0, 48, True, "mean")]))


def test_many_rows():
    """More rows than one 128-row tile takes of one head group, beside a decode row; one sequence fills its table."""
    m = Served("bf16", cfg=tiny_config("bf16").replace(n_q_heads=8, n_kv_heads=2, head_dim=128, n_layers=1))
    a = m.step(batch_of(m.cfg.vocab, 1, [EmbChunk(0, 0, 300, False, "mean")], [GenChunk(3, 0, 383, True)]))
    m.step(batch_of(m.cfg.vocab, 2, [EmbChunk(0, 300, 84, True, "mean")], [], [DecodeRow(3, 383)], a))


@pytest.mark.parametrize("two", [False, True])
def test_projection_in_two_parts(two):
    """Wide enough that the projection of few rows is split over its sum: the append adds the parts."""
    m = Served("bf16", two, two, cfg=tiny_config("bf16").replace(d_model=1024, n_q_heads=8, n_kv_heads=4, head_dim=128, d_ff=512))
    a = m.step(batch_of(m.cfg.vocab, 1, [EmbChunk(0, 0, 50, True, "mean")], [GenChunk(3, 0, 40, True), GenChunk(5, 0, 3, True)]))
    m.step(batch_of(m.cfg.vocab, 2, [], [], [DecodeRow(3, 40), DecodeRow(5, 3)], a))


@pytest.mark.parametrize("dtype,two", [("bf16", False), ("f32", True)])
def test_adapters_and_buffered_rows(dtype, two):
    m = Served(dtype, two, two, lora=2)
    b = batch_of(m.cfg.vocab, 1, [EmbChunk(0, 0, 23, False, "buffer"), EmbChunk(1, 0, 40, True, "mean"), EmbChunk(2, 0, 9, True, "last")],
                 [GenChunk(3, 0, 21, True)])
    b.chunk_adapter, b.hidden_stride = [1, 0, -1], 64
    a = m.step(b)
    b = batch_of(m.cfg.vocab, 2, [EmbChunk(0, 23, 30, True, "buffer")], [], [DecodeRow(3, 21)], a)
    b.chunk_adapter, b.hidden_stride = [1], 64
    m.step(b)


def drawn_steps(v):
    yield batch_of(v, 1, [EmbChunk(0, 0, 20, False, "mean")], [GenChunk(3, 0, 40, True), GenChunk(4, 0, 18, True)])
    for i in range(4):
        yield batch_of(v, 2 + i, [EmbChunk(0, 20 + 9 * i, 9, i == 3, "mean")], [], [DecodeRow(3, 40 + i), DecodeRow(4, 18 + i)],
                       draw_tokens(9, i, 2, v))


@pytest.mark.parametrize("two", [False, True])
def test_steps_back_to_back_and_on_another_stream(two):
    """Steps enqueued without a wait between them give the bits of steps that are waited for, as do those on a stream of
    the caller's."""
    got = []
    for how in range(3):
        m = Served("bf16", two, two)
        s = torch.cuda.Stream() if how == 2 else torch.cuda.current_stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            outs = []
            for b in drawn_steps(m.cfg.vocab):
                outs.append(m.enqueue(b))
                if how == 0:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert m.ws.device_error() == 0
        got.append([(o[0].cpu(), o[1].cpu(), o[2]["logprob"].cpu()) for o in outs] + [(m.acc_sum.cpu(),)])
    for other in got[1:]:
        for x, y in zip(got[0], other):
            assert all(torch.equal(p, q) for p, q in zip(x, y))


@pytest.mark.parametrize("two", [False, True])
def test_threads_that_share_a_model(two):
    """Two threads, each with caches, states, a workspace and a stream of its own, step the same models at once."""
    import threading
    m = Served("bf16", two, two)
    want = [[x.cpu() for x in m.enqueue(b)[:2]] for b in drawn_steps(m.cfg.vocab)]
    others, got, failed = [Served("bf16", two, two) for _ in range(2)], [[], []], []
    for o in others:
        o.dm = m.dm
        o.stream = torch.cuda.Stream()
    torch.cuda.synchronize()

    def run(i):
        try:
            with torch.cuda.stream(others[i].stream):
                outs = [others[i].enqueue(b)[:2] for b in drawn_steps(m.cfg.vocab)]
            others[i].stream.synchronize()
            got[i] = [[x.cpu() for x in o] for o in outs]
        except Exception as e:          # reported by the main thread
            failed.append(e)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for i in range(2):
        assert others[i].ws.device_error() == 0
        assert all(torch.equal(p, q) for x, y in zip(want, got[i]) for p, q in zip(x, y)) and len(got[i]) == len(want)


def test_bad_page_is_flagged_and_other_rows_keep_their_results():
    got = []
    for bad in (False, True):
        m = Served("bf16")
        steps = list(drawn_steps(m.cfg.vocab))
        m.enqueue(steps[0])
        if bad:
            m.table[0][4][1] = m.kv[0].n_pages            # sequence 4's second page
            m.kv[0].set_block_table(m.table[0])
        got.append(m.enqueue(steps[1])[0].cpu())
        torch.cuda.synchronize()
        assert m.ws.device_error() == (A.ORTHRUS_DEVERR_PAGE if bad else 0)
    assert torch.equal(got[0][0], got[1][0]) and not torch.equal(got[0][1], got[1][1])


def test_launches_are_timed_under_their_names_and_a_capture_is_refused():
    m = Served("bf16", two_models=True, two_caches=True)
    R.profile_begin(m.dm[0])
    m.enqueue(next(drawn_steps(m.cfg.vocab)))
    names = R.profile_end(m.dm[0])
    for n in ("kv8_append", "kv8_attend"):
        assert names[n][0] == names[n + "@gen"][0] == m.cfg.n_layers
    assert not any("rope" in n or n.startswith("attention") for n in names)
    g, b = torch.cuda.CUDAGraph(), batch_of(m.cfg.vocab, 3, [EmbChunk(1, 0, 3, False, "mean")])
    emb = torch.zeros((1, m.cfg.d_model), device="cuda")
    with torch.cuda.graph(g):
        emb.add_(1)
        with pytest.raises(A.OrthrusError) as e:
            ops.step_kv8(*m.dm, b, *m.kv, m.acc_sum, m.acc_w, None, emb, m.ws)
    assert e.value.code == A.ORTHRUS_EUNSUPPORTED
