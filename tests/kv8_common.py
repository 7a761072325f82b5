"""A cache on the GPU and its float64 definition side by side, and the bounds the operators are held to.

Bounds (a rounding is off by half a step: relative 2^-8 to bfloat16, 2^-24 to fp32, 2^-4 to e4m3):
  * rotated heads: the rounding to their type, plus 2^-19 of the pair's length for fp32 arithmetic: the mean
    square of up to 128 elements in a tree (20 roundings, halved by the root), division, product with the
    gain, sine and cosine (2 steps each), the rotation's three roundings: under 2^5 roundings of 2^-24;
  * held values: half a step of e4m3 under the page's own scale (2^-4 of the value, 2^-10 of the scale below
    2^-6), plus the same arithmetic; values that no arithmetic touches are the definition's bit for bit;
  * attention: softmax weights off by 2^-8 (bfloat16 rows) or less than 2^-16 (fp32 rows, three parts), the output's own
    rounding, and fp32 scores: products of at most 128 terms err by less than 2^-19 of the sum of their
    magnitudes, an absolute error of the exponent, so of every weight (twice: weight and sum); sums over keys
    add 2^-16 of the magnitudes.
"""
import numpy as np
import torch

from oracle import kv8 as D
from paper_2609_25405_amd import ops

PAGE = 16


def tensor(x, dtype="f32"):
    return torch.tensor(np.asarray(x), device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def host(t):
    return t.double().cpu().numpy()


class Both:
    def __init__(self, shape, n_seq, max_blocks, n_pages=None, seed=0, layers=1, layer=0):
        self.shape, self.layer = shape, layer
        n_pages = n_pages or n_seq * max_blocks + 3
        rng = self.rng = np.random.default_rng(seed)
        self.kv = ops.DeviceKV8(shape, layers, n_pages, n_seq, max_blocks)
        self.table = rng.permutation(n_pages)[:n_seq * max_blocks].reshape(n_seq, max_blocks).astype(np.int32)
        self.kv.set_block_table(self.table)
        # what no token wrote may be anything: codes of not-a-number
        self.kv.k.view(torch.uint8).fill_(0x7f)
        self.kv.v.view(torch.uint8).fill_(0xff)
        self.kv.k_scale.fill_(float("nan"))
        self.kv.v_scale.fill_(float("nan"))
        self.ref = D.Cache(1, shape.n_kv_heads, shape.head_dim)
        self.adopt()

    def held(self):
        """Device contents of the layer: values [pages][nkv][16][hd] of k and v, scales."""
        s = self.shape
        k = host(self.kv.k[self.layer].float()) * host(self.kv.k_scale[self.layer])[..., None, None]
        v = self.kv.v[self.layer].float().cpu().numpy().astype(np.float64)
        v = v.transpose(0, 1, 2, 5, 4, 3).reshape(*v.shape[:2], PAGE, s.head_dim) * host(self.kv.v_scale[self.layer])[..., None, None]
        return k, v

    def adopt(self):
        """The definition takes over what the device holds (so that later errors do not add up)."""
        k, v = self.held()
        self.ref.val = [k, v]
        self.ref.scale = [host(self.kv.k_scale[self.layer]), host(self.kv.v_scale[self.layer])]

    def fill(self, lengths, spread=1.0):
        """Caches of `lengths[seq]` random tokens, written straight into the pools."""
        s, rng = self.shape, self.rng
        nkv, hd = s.n_kv_heads, s.head_dim
        kc, vc = self.kv.k[self.layer].view(torch.uint8).cpu(), self.kv.v[self.layer].view(torch.uint8).cpu()
        ks, vs = self.kv.k_scale[self.layer].cpu(), self.kv.v_scale[self.layer].cpu()
        for seq, n in lengths.items():
            for b in range(-(-n // PAGE)):
                page, m = int(self.table[seq][b]), min(PAGE, n - b * PAGE)
                for codes, scale, is_v in ((kc, ks, False), (vc, vs, True)):
                    x = torch.tensor(rng.normal(size=(nkv, m, hd)) * spread * 2.0 ** rng.integers(-2, 3, size=(nkv, 1, 1)))
                    sc = torch.tensor([D.page_scale(float(x[h].abs().max())) for h in range(nkv)])
                    c = (x / sc[:, None, None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
                    scale[page] = sc.float()
                    if is_v:
                        tile = codes[page].permute(0, 1, 4, 3, 2).reshape(nkv, PAGE, hd)
                        tile[:, :m] = c
                        codes[page] = tile.reshape(nkv, 4, 4, hd // 16, 16).permute(0, 1, 4, 3, 2)
                    else:
                        codes[page][:, :m] = c
        self.kv.k[self.layer].view(torch.uint8).copy_(kc)
        self.kv.v[self.layer].view(torch.uint8).copy_(vc)
        self.kv.k_scale[self.layer].copy_(ks)
        self.kv.v_scale[self.layer].copy_(vs)
        self.adopt()

    def rows(self, segs):
        r = ops.RaggedRows(self.shape, sum(n for _, _, n in segs), len(segs), max(o + n for _, o, n in segs))
        r.plan(self.kv, segs)
        return r

    def check_attend(self, segs, q, out, scale=None, some=None, skip=()):
        """Every row of `out` (or `some` rows of it) against the definition."""
        s = self.shape
        hd, nq = s.head_dim, s.n_q_heads
        bf = s.dtype == "bf16"
        q, out = host(q).reshape(-1, nq, hd), host(out).reshape(-1, nq, hd)
        sc = hd ** -0.5 if scale is None else scale
        row, worst = 0, 0.0
        for seq, off, n in segs:
            for t in range(n):
                if some is None or row in some:
                    o, mag, size = self.ref.attend(self.table, seq, off + t, q[row], sc, skip)
                    tol = mag * (2.0 ** (-8 if bf else -16) + 2.0 ** -16 + 2 * size * 2.0 ** -19) + np.abs(o) * 2.0 ** (-8 if bf else -24) + 1e-30
                    err = np.abs(out[row] - o)
                    assert np.isfinite(out[row]).all() and (err <= tol).all(), (seq, off + t, float((err / tol).max()))
                    worst = max(worst, float((err / tol).max()))
                row += 1
        return worst
