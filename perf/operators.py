"""Measured calls of the operators a generator's rows go through when they are served from an
8-bit paged cache: head norms, rotation and append (with the read-back of what the cache holds),
attention over the cache, and log probabilities of sampled tokens.

One case is one call on one layer: a batch of segments (consecutive new tokens of one sequence
each; a decode row is a segment of one token) on one head layout, or the logits of a batch of
rows.  `prepare` makes what a serving process holds before the call, `run` is the call, in the
plain form or through the framework, and `exact` its definition in 64 bits.

The cache: pages of 16 tokens, e4m3 codes with a power-of-two scale for each page and KV head,
keys and values apart.  Keys are [page][kv head][slot][dim]; values
[page][kv head][slot / 4][dim % 16][dim / 16][slot % 4].
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

PAGE = 16
E4M3_MAX = 448.0
LEAST_EXP = -100        # scale of a page that holds only zeros: 2^-100

# query heads, KV heads, head width: the decoders of this repository's checks and workloads, then a
# wide group and an odd one
HEADS = {"tiny": (4, 4, 64), "narrow": (8, 2, 128), "mid": (16, 8, 128), "7b": (32, 8, 128), "group8": (64, 8, 128), "group7": (28, 4, 128)}

APPEND = dict(op="append", heads="7b", dtype="bf16", segments=1, len_lo=1, len_hi=1, ctx_lo=0, ctx_hi=0, norms=False, rot=0,
              interleaved=False, slow=1.0)
ATTEND = dict(op="attend", heads="7b", dtype="bf16", rows=0, ctx_lo=0, ctx_hi=0, chunks=0, len_lo=1, len_hi=1, before_lo=0, before_hi=0)
SCORE = dict(op="logprobs", rows=1, vocab=32000, top=5)


def listed():
    append = lambda name, **kw: dict(APPEND, name=name, **kw)
    attend = lambda name, **kw: dict(ATTEND, name=name, **kw)
    score = lambda name, **kw: dict(SCORE, name=name, **kw)
    return [
        # One user's next token in one layer: launches and latency.
        append("append-1", ctx_lo=700, ctx_hi=700),
        # A full decode batch of a model with head norms that turns half of each head, pairs side by side.
        append("append-256-norms", segments=256, ctx_lo=16, ctx_hi=4090, norms=True, rot=64, interleaved=True),
        # Prompt chunks that fill a large token budget, ragged, on positions slowed for a long context.
        append("append-prompts", segments=16, len_lo=301, len_hi=777, ctx_lo=0, ctx_hi=2000, slow=4.0),
        # One user's token: few keys, one row.
        attend("attend-1", rows=1, ctx_lo=700, ctx_hi=700),
        # The usual decode batch.
        attend("attend-64", rows=64, ctx_lo=1024, ctx_hi=4096),
        # Decode-heavy serving of long contexts: the cache is all there is.
        attend("attend-256-long", rows=256, ctx_lo=4096, ctx_hi=8192),
        # Fresh prompts of uneven lengths, a whole token budget.
        attend("attend-prompts", chunks=4, len_lo=400, len_hi=623),
        # Document chunks far into their documents, running decode rows beside them.
        attend("attend-documents", chunks=2, len_lo=512, len_hi=512, before_lo=7680, before_hi=7680, rows=14, ctx_lo=2048, ctx_hi=2048),
        # Rows of a model in fp32, small heads, odd lengths.
        attend("attend-ragged-f32", heads="tiny", dtype="f32", chunks=3, len_lo=33, len_hi=201, before_lo=0, before_hi=300, rows=9, ctx_lo=1, ctx_hi=999),
        # One sampled token's score.
        score("logprobs-1"),
        # A decode batch with the usual choice of alternatives.
        score("logprobs-256", rows=256, top=20),
        # The tokens of a long prompt scored under a large vocabulary.
        score("logprobs-prompt", rows=1999, vocab=131072, top=1),
    ]


def draw(rng: random.Random):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "append", "attend", "attend", "attend", "logprobs", "logprobs"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "append":
        c = dict(APPEND, heads=rng.choice(list(HEADS)), dtype=dtype, norms=rng.random() < 0.5, interleaved=rng.random() < 0.5,
                 slow=rng.choice([1.0, rng.uniform(1.0, 16.0)]))
        c["rot"] = rng.choice([0, 16 * rng.randint(1, HEADS[c["heads"]][2] // 16)])
        if rng.random() < 0.5:
            c.update(segments=log_int(1, 256), ctx_lo=log_int(1, 4096))
        else:
            c.update(segments=rng.randint(1, 12), len_lo=log_int(2, 512), ctx_lo=rng.choice([0, log_int(1, 30000)]))
        c["len_hi"] = min(700, c["len_lo"] * rng.randint(1, 3))
        c["ctx_hi"] = c["ctx_lo"] + log_int(1, 2000)
        return c
    if op == "attend":
        c = dict(ATTEND, heads=rng.choice(list(HEADS)), dtype=dtype)
        kind = rng.choice(["rows", "chunks", "both"])
        if kind != "chunks":
            c.update(rows=log_int(1, 200 if kind == "rows" else 16), ctx_lo=log_int(1, 4096 if kind == "rows" else 1500))
            c["ctx_hi"] = min(6000, c["ctx_lo"] * rng.randint(1, 4))
        if kind != "rows":
            c.update(chunks=rng.randint(1, 4), len_lo=log_int(2, 400), before_lo=rng.choice([0, log_int(1, 3000)]))
            c["len_hi"] = min(512, c["len_lo"] * rng.randint(1, 3))
            c["before_hi"] = c["before_lo"] + rng.randint(0, 500)
        return c
    c = dict(SCORE, rows=log_int(1, 1024), vocab=log_int(500, 160000), top=rng.choice([0, 1, rng.randint(2, 32)]))
    c["rows"] = min(c["rows"], 200_000_000 // c["vocab"])
    return c


# ------------------------------------------------------------------------------ layout of a case
def _rng(case, seed):
    """Lengths belong to the case; only the values come from the seed."""
    return np.random.default_rng([len(case["op"]), sum(map(ord, str(sorted((k, v) for k, v in case.items() if k != "name")))) % 100003])


def _segments(case, seed=0):
    """(cached tokens, new tokens) of each segment; chunks first, decode rows behind them."""
    rng = _rng(case, seed)
    between = lambda lo, hi, n: rng.integers(lo, max(lo, hi) + 1, size=n)
    if case["op"] == "append":
        ctx, new = between(case["ctx_lo"], case["ctx_hi"], case["segments"]), between(case["len_lo"], case["len_hi"], case["segments"])
    else:
        ctx = np.concatenate([between(case["before_lo"], case["before_hi"], case["chunks"]), between(case["ctx_lo"], case["ctx_hi"], case["rows"])])
        new = np.concatenate([between(case["len_lo"], case["len_hi"], case["chunks"]), np.ones(case["rows"], np.int64)])
    return [(int(c), int(n)) for c, n in zip(ctx, new)]


def _frequencies(case, hd):
    """Angle per position of each pair: base 10000 over the dims that turn; `slow` > 1 slows the
    pairs whose wavelength is longer than 512 positions."""
    rot = case["rot"] or hd
    f = 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    return np.where(2 * math.pi / f > 512, f / case["slow"], f)


def _magnitude(case):
    return 1.0 if case["slow"] == 1.0 else 0.1 * math.log(case["slow"]) + 1.0


def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _scale_of(amax):
    """The least power of two with amax <= 448 * scale (elementwise, fp32)."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(amax > 0, e, torch.full_like(e, LEAST_EXP)).clamp(min=LEAST_EXP)
    return torch.ldexp(torch.ones_like(amax), e)


def _keys_of(codes, scale):
    """Codes [..., kv head, 16, hd] and scales [..., kv head] as fp32 values."""
    return codes.view(torch.float8_e4m3fn).float() * scale[..., None, None]


def _values_to_tile(v):
    """[..., 16, hd] by slot to the cache's tile [..., 4, 16, hd / 16, 4]."""
    *b, _, hd = v.shape
    return v.reshape(*b, 4, 4, hd // 16, 16).transpose(-1, -3).contiguous()


def _tile_to_values(t):
    """The cache's tile [..., 4, 16, hd / 16, 4] to [..., 16, hd] by slot."""
    *b, _, _, db, _ = t.shape
    return t.transpose(-1, -3).reshape(*b, 16, 16 * db)


def _cache(n_pages, nkv, hd, gen, dev):
    """Pools of a cache whose every page holds 16 tokens' rounded keys and values."""
    def pool():
        codes = torch.empty((n_pages, nkv, PAGE, hd), dtype=torch.uint8, device=dev)
        scale = torch.empty((n_pages, nkv), dtype=torch.float32, device=dev)
        for i in range(0, n_pages, 8192):
            n = min(8192, n_pages - i)
            x = torch.randn((n, nkv, PAGE, hd), generator=gen, device=dev)
            x *= torch.exp(0.5 * torch.randn((n, nkv, 1, 1), generator=gen, device=dev))
            s = _scale_of(x.abs().amax(dim=(-1, -2)))
            scale[i:i + n] = s
            codes[i:i + n] = (x / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        return codes, scale

    k, ks = pool()
    v, vs = pool()
    return k, _values_to_tile(v), ks, vs


# ------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    if case["op"] == "logprobs":
        R, V = case["rows"], case["vocab"]
        x = torch.randn((R, V), generator=gen, device=dev) * 2.0
        tok = torch.randint(0, V, (R,), generator=gen, device=dev)
        x.scatter_add_(1, tok[:, None], torch.rand((R, 1), generator=gen, device=dev) * 14.0)   # some likely, some not
        st = dict(case=case, logits=x, tokens=tok.to(torch.int32))
        if own:
            from paper_2609_25405_amd import ops

            n = case["top"]
            f32, i32 = dict(dtype=torch.float32, device=dev), dict(dtype=torch.int32, device=dev)
            st["out"] = dict(logprob=torch.empty(R, **f32), entropy=torch.empty(R, **f32), rank=torch.empty(R, **i32))
            if n:
                st["out"].update(top_ids=torch.empty((R, n), **i32), top_logprobs=torch.empty((R, n), **f32))
            st["ws"] = ops.logprobs_workspace(R, V, n, device=dev)
        return st

    nq, nkv, hd = HEADS[case["heads"]]
    dt = _torch_dtype(case)
    segs = _segments(case)
    S, T = len(segs), sum(n for _, n in segs)
    pages = [-(-(c + n) // PAGE) for c, n in segs]
    B, P = max(pages), sum(pages) + 3
    # page ids scattered over the pool; table entries past a sequence's pages are -1
    order = torch.randperm(P, generator=gen, device=dev).to(torch.int32)
    table = torch.full((S, B), -1, dtype=torch.int32)
    at = np.concatenate([[0], np.cumsum(pages)])
    order_h = order.cpu()
    for s in range(S):
        table[s, :pages[s]] = order_h[at[s]:at[s + 1]]
    table = table.to(dev)
    k, v, ks, vs = _cache(P, nkv, hd, gen, dev)
    st = dict(case=case, segs=segs, k=k, v=v, ks=ks, vs=vs, table=table, seg=torch.tensor(segs, device=dev))
    row0 = np.concatenate([[0], np.cumsum([n for _, n in segs])])
    st["row0"] = torch.tensor(row0[:-1], device=dev)
    st["row_seg"] = torch.tensor(np.repeat(np.arange(S), [n for _, n in segs]), device=dev)
    st["pos"] = torch.tensor(np.concatenate([np.arange(c, c + n) for c, n in segs]), device=dev)
    if case["op"] == "append":
        st["qkv"] = (torch.randn((T, (nq + 2 * nkv) * hd), generator=gen, device=dev) * 1.5).to(dt)
        st["gains"] = [1.0 + 0.2 * torch.randn(hd, generator=gen, device=dev) for _ in range(2)] if case["norms"] else [None, None]
        st["freq"] = torch.tensor(_frequencies(case, hd), dtype=torch.float64, device=dev)
        # touched pages: (segment, page of the sequence), and the positions they hold now
        touched = [(s, p) for s, (c, n) in enumerate(segs) for p in range(c // PAGE, (c + n - 1) // PAGE + 1)]
        st["unit"] = torch.tensor(touched, device=dev)
        first = np.concatenate([[0], np.cumsum([(c + n - 1) // PAGE - c // PAGE + 1 for c, n in segs])])
        st["unit_of_row"] = torch.tensor(np.concatenate([first[s] + np.arange(c, c + n) // PAGE - c // PAGE for s, (c, n) in enumerate(segs)]), device=dev)
        back = [(s, c // PAGE * PAGE, c + n) for s, (c, n) in enumerate(segs)]
        st["back"] = torch.tensor(np.concatenate([np.stack([np.full(e - b, s), np.arange(b, e)], 1) for s, b, e in back]), device=dev)
    else:
        st["q"] = (torch.randn((T, nq * hd), generator=gen, device=dev) * 1.5).to(dt)
        st["longest"] = (max(n for _, n in segs), max(c + n for c, n in segs))
    if own:
        from paper_2609_25405_amd import ops

        rope = {}
        if case["op"] == "append":
            rope = dict(rot_dims=case["rot"] or hd, interleaved=case["interleaved"], rope_freq=_frequencies(case, hd), rope_magnitude=_magnitude(case))
        shape = ops.HeadShape(nq, nkv, hd, dtype=case["dtype"], **rope)
        kv = ops.DeviceKV8.from_pools(shape, k[None].view(torch.float8_e4m3fn), v[None].view(torch.float8_e4m3fn), ks[None], vs[None], table)
        rows = ops.RaggedRows(shape, T, S, max(c + n for c, n in segs))
        rows.plan(kv, [(s, c, n) for s, (c, n) in enumerate(segs)])
        st.update(kv=kv, rows=rows)
        if case["op"] == "append":
            N = st["back"].shape[0]
            st["q_out"] = torch.empty((T, nq * hd), dtype=dt, device=dev)
            st["held"] = ops.RaggedRows(shape, N, S, max(c + n for c, n in segs))
            st["held"].plan(kv, [(s, b, e - b) for s, b, e in back])
            st["k_out"] = torch.empty((N, nkv * hd), dtype=torch.bfloat16, device=dev)
            st["v_out"] = torch.empty((N, nkv * hd), dtype=torch.bfloat16, device=dev)
        else:
            st["out"] = torch.empty((T, nq * hd), dtype=dt, device=dev)
    return st


# ------------------------------------------------------------------------------ the call
def run(st):
    op = st["case"]["op"]
    if own:
        from paper_2609_25405_amd import ops

        if op == "append":
            ops.kv8_append(st["rows"], st["kv"], 0, st["qkv"], st["q_out"], q_gain=st["gains"][0], k_gain=st["gains"][1])
            ops.kv8_read(st["held"], st["kv"], 0, st["k_out"], st["v_out"])
            return st["q_out"], st["k_out"], st["v_out"]
        if op == "attend":
            ops.kv8_attend(st["rows"], st["kv"], 0, st["q"], st["out"])
            return st["out"]
        ops.logprobs(st["logits"], st["tokens"], workspace=st["ws"], **st["out"])
        return st["out"]
    return {"append": _plain_append, "attend": _plain_attend, "logprobs": _plain_logprobs}[op](st)


def _turn(x, cos, sin, rot, interleaved):
    """Rotation of the first `rot` dims of x [T, heads, hd] by cos, sin [T, 1, rot / 2]."""
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _plain_append(st):
    case = st["case"]
    nq, nkv, hd = HEADS[case["heads"]]
    T = st["qkv"].shape[0]
    x = st["qkv"].float().view(T, nq + 2 * nkv, hd)
    q, k, v = x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:]
    if case["norms"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + 1e-6) * st["gains"][0]
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + 1e-6) * st["gains"][1]
    angle = st["pos"].double()[:, None] * st["freq"]        # far positions: the angle needs 64 bits
    cos = (angle.cos() * _magnitude(case)).float()[:, None]
    sin = (angle.sin() * _magnitude(case)).float()[:, None]
    rot = case["rot"] or hd
    q, k = _turn(q, cos, sin, rot, case["interleaved"]), _turn(k, cos, sin, rot, case["interleaved"])

    unit, of = st["unit"], st["unit_of_row"]
    page = st["table"][unit[:, 0], unit[:, 1]].long()
    slot = st["pos"] % PAGE
    ctx, new = st["seg"][unit[:, 0], 0], st["seg"][unit[:, 0], 1]
    at = unit[:, 1, None] * PAGE + torch.arange(PAGE, device=page.device)       # positions of the touched pages
    old, live = at < ctx[:, None], at < (ctx + new)[:, None]
    old_k = st["k"][page].view(torch.float8_e4m3fn).float()
    old_v = _tile_to_values(st["v"][page]).view(torch.float8_e4m3fn).float()
    for pool, scales, held, fresh in ((st["k"], st["ks"], old_k, k), (st["v"], st["vs"], old_v, v)):
        tile = torch.zeros((len(unit), PAGE, nkv, hd), device=page.device)
        tile[of, slot] = fresh
        tile = tile.transpose(1, 2)                                             # [page, kv head, slot, dim]
        amax = torch.where(tile.isfinite(), tile.abs(), 0.0).amax(dim=(-1, -2))
        grown, was = _scale_of(amax), scales[page]
        scale = torch.where(old[:, :1], torch.maximum(was, grown), grown)
        held_now = held * (was / scale)[..., None, None]
        codes = torch.where(old[:, None, :, None], held_now, tile / scale[..., None, None])
        codes = torch.where(live[:, None, :, None], codes, held).to(torch.float8_e4m3fn).view(torch.uint8)
        pool[page] = codes if pool is st["k"] else _values_to_tile(codes)
        scales[page] = scale

    back = st["back"]
    page, slot = st["table"][back[:, 0], back[:, 1] // PAGE].long(), back[:, 1] % PAGE
    held_k = st["k"][page, :, slot].view(torch.float8_e4m3fn).float() * st["ks"][page][..., None]
    held_v = st["v"][page, :, slot // 4, :, :, slot % 4].transpose(-1, -2).reshape(len(back), nkv, hd)
    held_v = held_v.view(torch.float8_e4m3fn).float() * st["vs"][page][..., None]
    return q.reshape(T, nq * hd).to(st["qkv"].dtype), held_k.reshape(len(back), -1).bfloat16(), held_v.reshape(len(back), -1).bfloat16()


def _plain_attend(st):
    case = st["case"]
    nq, nkv, hd = HEADS[case["heads"]]
    G, (most, keys) = nq // nkv, st["longest"]
    T, S = st["q"].shape[0], len(st["segs"])
    page = st["table"].clamp(min=0).long()                                      # [S, B]
    k = _keys_of(st["k"][page], st["ks"][page]).transpose(1, 2).reshape(S, nkv, -1, hd)
    v = _tile_to_values(st["v"][page])
    v = _keys_of(v, st["vs"][page]).transpose(1, 2).reshape(S, nkv, -1, hd)
    i = torch.arange(most, device=page.device)
    ctx, new = st["seg"][:, 0, None], st["seg"][:, 1, None]
    row = st["row0"][:, None] + torch.minimum(i, new - 1)                       # padded rows repeat the last one
    q = st["q"].float().view(T, nkv, G, hd)[row].permute(0, 2, 3, 1, 4).reshape(S, nkv, G * most, hd)
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()) * hd ** -0.5
    sees = torch.arange(k.shape[2], device=page.device) <= torch.minimum(ctx + i, ctx + new - 1)[..., None]
    s = s.view(S, nkv, G, most, -1).masked_fill(~sees[:, None, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.matmul(p.view(S, nkv, G * most, -1), v) / p.sum(-1).view(S, nkv, G * most, 1)
    o = o.view(S, nkv, G, most, hd).permute(0, 3, 1, 2, 4)                      # [S, most, nkv, G, hd]
    first = st["row0"][st["row_seg"]]
    out = o[st["row_seg"], torch.arange(T, device=page.device) - first]
    return out.reshape(T, nq * hd).to(st["q"].dtype)


def _order(x):
    """Integers that order fp32 values as the sampler does (NaN above everything, -0 = +0)."""
    b = (x + 0.0).view(torch.int32)
    return torch.where(x.isnan(), 2 ** 31 - 1, b ^ ((b >> 31) & 0x7fffffff)).long()


def _plain_logprobs(st):
    x, tok, n = st["logits"], st["tokens"].long()[:, None], st["case"]["top"]
    V = x.shape[1]
    y = x - x.amax(-1, keepdim=True)
    e = torch.exp(y)
    z = e.sum(-1, keepdim=True)
    logz = torch.log(z)
    key = _order(x) * 2 ** 32 + (V - 1 - torch.arange(V, device=x.device))      # larger first, then the lowest index
    out = dict(logprob=(y.gather(1, tok) - logz)[:, 0], entropy=(logz - (e * y).sum(-1, keepdim=True) / z)[:, 0],
               rank=(key > key.gather(1, tok)).sum(-1).to(torch.int32))
    if n:
        ids = V - 1 - (key.topk(n, dim=-1).values % 2 ** 32)
        out.update(top_ids=ids.to(torch.int32), top_logprobs=y.gather(1, ids) - logz)
    return out


# ------------------------------------------------------------------------------ work and definition
def work(case):
    if case["op"] == "logprobs":
        R, V, n = case["rows"], case["vocab"], case["top"]
        return {"bytes": 4 * R * V + R * (16 + 8 * n), "flops": 4 * R * V}
    nq, nkv, hd = HEADS[case["heads"]]
    segs = _segments(case)
    T, es = sum(n for _, n in segs), 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "append":
        held = sum(c % PAGE + n for c, n in segs)
        units = sum((c + n - 1) // PAGE - c // PAGE + 1 for c, n in segs)
        b = T * (nq + 2 * nkv) * hd * es + T * nq * hd * es + T * 2 * nkv * hd + units * nkv * 8   # append
        b += held * 2 * nkv * hd * (1 + 2) + units * nkv * 8                                       # read back
        return {"bytes": b, "flops": 8 * T * (nq + 2 * nkv) * hd}
    keys = sum(c + n for c, n in segs)
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in segs)
    pages = sum(-(-(c + n) // PAGE) for c, n in segs)
    return {"bytes": keys * 2 * nkv * hd + pages * (nkv * 8 + 4) + 2 * T * nq * hd * es, "flops": 4 * pairs * nq * hd}


def _to_e4m3(x):
    """The nearest e4m3 value of each |x| <= 448, ties to even, in float64 (not a number: stays)."""
    ax = x.abs().clamp(min=2.0 ** -30)
    step = torch.exp2(torch.floor(torch.log2(ax)).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _exact_append(st):
    case = st["case"]
    nq, nkv, hd = HEADS[case["heads"]]
    rot = case["rot"] or hd
    mag = _magnitude(case)
    half = torch.arange(rot // 2, device=st["qkv"].device)
    lo, hi = (2 * half, 2 * half + 1) if case["interleaved"] else (half, half + rot // 2)
    x = st["qkv"].double().view(-1, nq + 2 * nkv, hd)
    heads = x.clone()
    for first, n, gain in ((0, nq, st["gains"][0]), (nq, nkv, st["gains"][1])):
        h = x[:, first:first + n]
        if gain is not None:
            h = h * gain.double() / (h.pow(2).sum(-1, keepdim=True) / hd + 1e-6).sqrt()
        th = (st["pos"].double()[:, None] * st["freq"])[:, None]
        y = h.clone()
        y[..., lo] = mag * (h[..., lo] * th.cos() - h[..., hi] * th.sin())
        y[..., hi] = mag * (h[..., hi] * th.cos() + h[..., lo] * th.sin())
        heads[:, first:first + n] = y
    table, ks, vs = st["table"].cpu().numpy(), st["ks"].double(), st["vs"].double()
    outs, r = ([], []), 0
    for s, (c, n) in enumerate(st["segs"]):
        b = c // PAGE * PAGE
        for which in range(2):
            fresh = heads[r:r + n, nq + which * nkv:nq + (which + 1) * nkv]
            scales = (ks, vs)[which]
            for p in range(b, c + n, PAGE):
                pg = int(table[s, p // PAGE])
                new = fresh[max(p, c) - c:p + PAGE - c]
                amax = torch.where(new.isfinite(), new.abs(), 0.0).amax(dim=(0, 2))
                e = torch.ceil(torch.log2(amax.clamp(min=1e-300) / E4M3_MAX)).clamp(min=LEAST_EXP)
                scale = torch.exp2(e)
                if p < c:
                    held = st["k"][pg] if which == 0 else _tile_to_values(st["v"][pg])
                    held = held.view(torch.float8_e4m3fn).double()[:, :c - p] * scales[pg][:, None, None]
                    scale = torch.maximum(scale, scales[pg])
                    outs[which].append(_to_e4m3(held.transpose(0, 1) / scale[:, None]) * scale[:, None])
                outs[which].append(_to_e4m3(new / scale[:, None]) * scale[:, None])
        r += n
    k, v = (torch.cat(o).reshape(-1, nkv * hd) for o in outs)
    return heads[:, :nq].reshape(-1, nq * hd), k, v


def _exact_attend(st):
    nq, nkv, hd = HEADS[st["case"]["heads"]]
    G, out, r = nq // nkv, [], 0
    for s, (c, n) in enumerate(st["segs"]):
        page = st["table"][s, :-(-(c + n) // PAGE)].long()
        k = st["k"][page].view(torch.float8_e4m3fn).double() * st["ks"][page].double()[..., None, None]
        v = _tile_to_values(st["v"][page]).view(torch.float8_e4m3fn).double() * st["vs"][page].double()[..., None, None]
        k, v = (t.transpose(0, 1).reshape(nkv, -1, hd)[:, :c + n] for t in (k, v))
        q = st["q"][r:r + n].double().view(n, nkv, G, hd)
        o = torch.empty((n, nkv, G, hd), dtype=torch.float64, device=q.device)
        hidden = torch.arange(c + n, device=q.device) > c + torch.arange(n, device=q.device)[:, None]
        for h in range(nkv):
            for g in range(G):
                w = (q[:, h, g] @ k[h].T) / math.sqrt(hd)
                w[hidden] = -math.inf
                o[:, h, g] = torch.softmax(w, -1) @ v[h]
        out.append(o.reshape(n, nq * hd))
        r += n
    return torch.cat(out)


def _exact_logprobs(st):
    outs = {"logprob": [], "entropy": [], "rank": [], "top_ids": [], "top_logprobs": []}
    n = st["case"]["top"]
    for i in range(0, len(st["tokens"]), 256):
        x, tok = st["logits"][i:i + 256], st["tokens"][i:i + 256].long()[:, None]
        lp = torch.log_softmax(x.double(), -1)
        at = x.gather(1, tok)
        before = (x > at) | ((x == at) & (torch.arange(x.shape[1], device=x.device) < tok))
        ids = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :n]
        for name, t in (("logprob", lp.gather(1, tok)[:, 0]), ("entropy", -(lp.exp() * lp).sum(-1)), ("rank", before.sum(-1)),
                        ("top_ids", ids), ("top_logprobs", lp.gather(1, ids))):
            outs[name].append(t)
    outs = {name: torch.cat(t) for name, t in outs.items() if n or not name.startswith("top")}
    return {name: t if t.is_floating_point() else t.to(torch.int32) for name, t in outs.items()}


def exact(case, seed):
    return {"append": _exact_append, "attend": _exact_attend, "logprobs": _exact_logprobs}[case["op"]](prepare(case, seed))
