"""The paged cache in plain Python and 64 bits, for the tests: its bookkeeping on lists, the append
and the attention by their formulas. Imported only by tests marked ``gpu``."""
import math

import numpy as np
import torch

import _gpu as G
M = G.M

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}   # a rounding, relative to the value


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Cache:
    """A paged cache on the GPU and, beside it, what its bookkeeping has to be."""

    def __init__(self, layers=1, q_heads=4, kv_heads=2, d=64, page=16, n_pages=40, max_seqs=8, max_pages=16,
                 dtype="bf16", seed=0, **rot):
        self.L, self.Hq, self.H, self.d, self.P = layers, q_heads, kv_heads, d, page
        self.n_pages, self.max_seqs, self.max_pages, self.dtype = n_pages, max_seqs, max_pages, dtype
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.k, self.v = (self.normal(layers, n_pages, kv_heads, page, d) for _ in range(2))
        self.table = torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(max_seqs, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.c = M.paged_cache(self.k, self.v, self.table, self.lens, self.refs)
        self.h = M.mot_create_paged(M.make_paged_config(layers, q_heads, kv_heads, d, page, n_pages, max_seqs,
                                                        max_pages, dtype=dtype, **rot))
        self.t = [[] for _ in range(max_seqs)]   # a slot's pages
        self.n = [0] * max_seqs
        self.r = [0] * n_pages

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda").to(DT[self.dtype])

    def status(self):
        return M.mot_get_device_status(self.h)

    def pages(self, n):
        return -(-n // self.P)

    def take(self, count):
        got = [p for p in range(self.n_pages) if self.r[p] == 0][:count]
        assert len(got) == count
        for p in got:
            self.r[p] = 1
        return got

    def batch(self, seqs, new):
        starts = [sum(new[:i]) for i in range(len(new) + 1)]
        return M.paged_batch(i32(seqs), i32(starts), len(seqs), starts[-1], max(new, default=0))

    # each: the call, then the same on the lists
    def reserve(self, seqs, new, ok=True):
        M.mot_paged_reserve(self.h, self.c, self.batch(seqs, new))
        if ok:
            for s, m in zip(seqs, new):
                self.t[s] += self.take(self.pages(self.n[s] + m) - self.pages(self.n[s]))
                self.n[s] += m

    def fork(self, src, dst, ok=True):
        M.mot_paged_fork(self.h, self.c, i32(src), i32(dst), len(src))
        copies = []
        if ok:
            for a, b in zip(src, dst):
                full, part = divmod(self.n[a], self.P)
                self.t[b] = self.t[a][:full]
                for p in self.t[b]:
                    self.r[p] += 1
                if part:
                    self.t[b] += self.take(1)
                    copies.append((self.t[a][full], self.t[b][full], part))
                self.n[b] = self.n[a]
        return copies

    def free(self, seqs, ok=True):
        M.mot_paged_free(self.h, self.c, i32(seqs), len(seqs))
        if ok:
            for s in seqs:
                for p in self.t[s]:
                    self.r[p] -= 1
                self.t[s], self.n[s] = [], 0

    def compact(self, live=None):
        M.mot_paged_compact(self.h, self.c, live)
        used = sum(x > 0 for x in self.r)
        moves = list(zip([p for p in range(used, self.n_pages) if self.r[p]], [p for p in range(used) if not self.r[p]]))
        to = dict(moves)
        for a, b in moves:
            self.r[b], self.r[a] = self.r[a], 0
        self.t = [[to.get(p, p) for p in row] for row in self.t]
        return moves

    def check(self, label=""):
        torch.cuda.synchronize()
        want = np.full((self.max_seqs, self.max_pages), -1, dtype=np.int32)
        for s, row in enumerate(self.t):
            want[s, :len(row)] = row
        np.testing.assert_array_equal(self.table.cpu().numpy(), want, err_msg=f"table {label}")
        np.testing.assert_array_equal(self.lens.cpu().numpy(), self.n, err_msg=f"lens {label}")
        np.testing.assert_array_equal(self.refs.cpu().numpy(), self.r, err_msg=f"refs {label}")

    def rows(self, s, layer=0, pools=None):
        """Keys and values of slot s, [heads][len][d] in 64 bits."""
        out = []
        for x in pools or (self.k, self.v):
            if not self.t[s]:
                out.append(torch.zeros((self.H, 0, self.d), dtype=torch.float64, device="cuda"))
            else:
                out.append(x[layer, self.t[s]].permute(1, 0, 2, 3).reshape(self.H, -1, self.d)[:, :self.n[s]].double())
        return out


def attention(q, K, V):
    """q [m][Hq][d] as the last m of K's, V's positions ([H][n][d]): the result and a bound on what
    bf16 probabilities and 32-bit sums may be off, both in 64 bits."""
    m, Hq, d = q.shape
    H, n = K.shape[:2]
    out = torch.zeros((m, Hq, d), dtype=torch.float64, device=q.device)
    absv, slop = torch.zeros_like(out), torch.zeros_like(out)
    for r in range(m):
        p = n - m + r
        if p < 0:
            continue
        Kr, Vr = (x[:, :p + 1].repeat_interleave(Hq // H, 0) for x in (K, V))
        prod = q[r].double()[:, None] * Kr / math.sqrt(d)
        w = torch.softmax(prod.sum(2), 1)
        out[r] = torch.einsum("hn,hnd->hd", w, Vr)
        absv[r] = torch.einsum("hn,hnd->hd", w, Vr.abs())
        # a score of d products is off by (d + 4) 2^-24 of their absolute sum, its weight relative to
        # the largest by twice that and two exponentials of 2^-21; the sums over n keys by n 2^-24 each
        big = prod.abs().sum(2).amax(1)[:, None]
        slop[r] = absv[r] * (2 * (d + 4) * 2.0 ** -24 * big + 2.0 ** -20 + 2 * (p + 9) * 2.0 ** -24)
    return out, absv, slop


def assert_close(got, want, tol, label=""):
    g = got.double()
    bad = ~((g - want).abs() <= tol)
    assert not bool(bad.any()), (f"{label}: {int(bad.sum())} of {bad.numel()} off, first at "
                                 f"{torch.nonzero(bad)[0].tolist()}: {g[bad][0]:.6g} for {want[bad][0]:.6g}, "
                                 f"allowed {(tol + 0 * want)[bad][0]:.3g}")


def check_attention(c, seqs, new, q, out, layer=0, label=""):
    """out against the formula, for the slots' last `new` positions."""
    at = 0
    for s, m in zip(seqs, new):
        K, V = c.rows(s, layer)
        ref, absv, slop = attention(q[at:at + m], K, V)
        half = HALF[c.dtype]
        tol = half * ref.abs() + slop + 1e-30
        if c.dtype == "bf16":
            tol = tol + half * absv   # the probabilities are rounded to bf16 too
        assert_close(out[at:at + m], ref, tol, f"{label} slot {s}")
        at += m
