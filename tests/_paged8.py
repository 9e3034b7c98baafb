"""The paged cache in 8 bits, in plain Python and 64 bits, for the tests. Imported only by tests marked ``gpu``."""
import math

import torch

import _paged as P
M = P.M
F8 = torch.float8_e4m3fn
TOP = 448.0 * 2.0 ** 60


def scale_of(top):
    """2^e with the least e in -60 .. 60 with top <= 448 * 2^e, element by element (on the CPU)."""
    def one(t):
        e = -60
        while e < 60 and t > 448 * 2.0 ** e:
            e += 1
        return 2.0 ** e
    return torch.tensor([one(float(t)) for t in top.flatten().cpu()], dtype=torch.float64, device=top.device).view(top.shape)


def eighths(x):
    """x in 64 bits to the nearest of 1 sign, 4 exponent and 3 mantissa bits, ties to the even one; NaN stays."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def held(x):
    """x in 64 bits, with NaN for what 8 bits do not hold."""
    return torch.where(x.abs() <= TOP, x, torch.nan)


def largest(x, dims):
    return torch.where(x.abs() <= TOP, x.abs(), 0.0).amax(dims)


class Cache(P.Cache):
    """A paged cache in 8 bits on the GPU and, beside it, what its bookkeeping has to be."""

    def __init__(self, layers=1, q_heads=4, kv_heads=2, d=64, page=16, n_pages=40, max_seqs=8, max_pages=16, seed=0, **rot):
        self.L, self.Hq, self.H, self.d, self.P = layers, q_heads, kv_heads, d, page
        self.n_pages, self.max_seqs, self.max_pages, self.dtype = n_pages, max_seqs, max_pages, "bf16"
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.k, self.v = (self.normal(layers, n_pages, kv_heads, page, d).mul_(64).to(F8) for _ in range(2))
        e = torch.randint(-9, -3, (2, layers, n_pages, kv_heads), generator=self.gen, device="cuda")
        self.ks, self.vs = torch.exp2(e.float())
        self.table = torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(max_seqs, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.c = M.paged_cache(self.k, self.v, self.table, self.lens, self.refs, self.ks, self.vs)
        self.h = M.mot_create_paged8(M.make_paged_config(layers, q_heads, kv_heads, d, page, n_pages, max_seqs, max_pages, **rot))
        self.t = [[] for _ in range(max_seqs)]
        self.n = [0] * max_seqs
        self.r = [0] * n_pages

    def pools(self):
        """Keys and values in 64 bits, [layers][pages][heads][page][d]."""
        return [x.double() * s.double()[..., None, None] for x, s in ((self.k, self.ks), (self.v, self.vs))]

    def bytes(self):
        return [x.view(torch.uint8).clone() for x in (self.k, self.v)] + [self.ks.clone(), self.vs.clone()]

    def rows(self, s, layer=0, pools=None):
        return super().rows(s, layer, pools or self.pools())


def joined(old, was, new):
    """A page's rows after new ones join it, for one head: old [n][d] in units of the scale `was`, new [m][d] values;
    both in units of the scale that is returned first. 64 bits."""
    scale = scale_of(largest(new, (0, 1)))
    if len(old):
        scale = torch.maximum(scale, was)
        old = eighths(old * (was / scale))
    return scale, old, eighths(held(new) / scale)


def same(a, b):
    """Equal, NaN with NaN."""
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


assert math.isclose(TOP, 448.0 * 2.0 ** 60)


def check_attention(c, seqs, new, q, out, layer=0, label=""):
    """out against the formula in 64 bits, for the slots' last `new` positions."""
    at = 0
    for s, m in zip(seqs, new):
        K, V = c.rows(s, layer)
        n = K.shape[1]
        ref, absv, slop = P.attention(q[at:at + m], K, V)
        # beside what 16-bit pages are off by: the exponent of a page's value scale, 60 at most, is added to a score
        # (61 roundings' worth of 2^-24, in the numerator and the sum); a weight is rounded to fp16, whose steps
        # are 2^-10 above a power of two (11 bits): by 2^-11 of it, or by 2^-25 of the row's largest weight times its
        # value scale, half the smallest step
        tol = 2.0 ** -8 * ref.abs() + slop + (2.0 ** -17 + 2.0 ** -11) * absv + 1e-30
        if m and n:
            of = torch.tensor([c.t[s][j // c.P] for j in range(n)], device=q.device)
            sv = c.vs[layer][of].double().T.repeat_interleave(c.Hq // c.H, 0)   # [Hq][n]
            v8 = (V.abs().nan_to_num(0.0) / c.vs[layer][of].double().T[..., None]).repeat_interleave(c.Hq // c.H, 0).cumsum(1)
            for r in range(m):
                p = n - m + r
                if p < 0:
                    continue
                w = torch.softmax(torch.einsum("hd,hnd->hn", q[at + r].double(), K[:, :p + 1].repeat_interleave(c.Hq // c.H, 0))
                                  / math.sqrt(c.d), 1)
                # a query's element is off by 2^-17 of its row's largest at most, and every score by that
                qmax = q[at + r].double().abs().amax(1)
                off = 2.0 ** -17 * qmax * K[:, :p + 1].abs().sum(2).amax(1).repeat_interleave(c.Hq // c.H) / math.sqrt(c.d)
                tol[r] += 2 * off[:, None] * absv[r]
                tol[r] += 2.0 ** -25 * (w * sv[:, :p + 1]).amax(1)[:, None] * v8[:, p]
        P.assert_close(out[at:at + m], ref, tol, f"{label} slot {s}")
        at += m
