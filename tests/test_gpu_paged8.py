"""The paged cache in 8 bits on the GPU through the C ABI: its pages and scales against the rule they follow, the
append and the attention against their formulas in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import _paged as P   # noqa: E402
import _paged8 as P8   # noqa: E402
M = P.M
i32 = P.i32


# ---------------------------------------------------------------- pages

def _stored(x):
    """One page's rows x [heads][rows][d] as they are held: values and scales [heads]."""
    s = P8.scale_of(P8.largest(x, (1, 2)))
    return P8.eighths(P8.held(x) / s[:, None, None]) * s[:, None, None], s


def _kept(x, P_):
    """x [layers][heads][len][d] in 64 bits as 8-bit pages of P_ positions hold it."""
    out = x.clone()
    for l in range(x.shape[0]):
        for j in range(0, x.shape[2], P_):
            out[l, :, j:j + P_] = _stored(x[l, :, j:j + P_])[0]
    return out


@pytest.mark.parametrize("page,d,h", [(16, 64, 3), (32, 128, 1), (64, 64, 2), (128, 128, 2)])
def test_pages_over_a_random_run(page, d, h):
    """Reserve, fork, free, compact, store and load in a random order: the bookkeeping as lists have it, and every
    sequence's positions hold what was stored, with their scales, whatever moves and is shared around them."""
    rng = np.random.default_rng(page + d)
    c = P8.Cache(layers=2, kv_heads=h, q_heads=h, d=d, page=page, n_pages=19, max_seqs=6, max_pages=5)
    want = [None] * c.max_seqs
    S = c.max_pages * page
    for step in range(40):
        used = [s for s in range(c.max_seqs) if c.n[s]]
        empty = [s for s in range(c.max_seqs) if not c.n[s]]
        free = sum(x == 0 for x in c.r)
        op = rng.choice(["grow", "grow", "fork", "free", "compact"])
        if op == "grow":
            seqs = [int(s) for s in rng.permutation(c.max_seqs)[:rng.integers(1, 4)]]
            new = [int(rng.integers(0, 2 * page + 2)) for _ in seqs]
            if any(c.n[s] + m > S for s, m in zip(seqs, new)):
                continue
            if sum(c.pages(c.n[s] + m) - c.pages(c.n[s]) for s, m in zip(seqs, new)) > free:
                continue
            c.reserve(seqs, new)
            alone = [s for s in seqs if all(c.r[p] == 1 for p in c.t[s])]
            if alone:
                flat = [c.normal(c.L, len(alone) + 1, c.H, S, d) * 2.0 ** int(rng.integers(-20, 20)) for _ in range(2)]
                M.mot_paged_store(c.h, c.c, i32(alone), len(alone), *flat)
                for i, s in enumerate(alone):
                    want[s] = [_kept(x[:, i, :, :c.n[s]].double(), page) for x in flat]
            pools = c.pools()
            for s in set(seqs) - set(alone):   # stale contents behind the old length
                want[s] = [x[:, c.t[s]].permute(0, 2, 1, 3, 4).reshape(c.L, c.H, -1, d)[:, :, :c.n[s]] for x in pools]
        elif op == "fork" and used and empty:
            k = int(rng.integers(1, len(empty) + 1))
            src, dst = [int(rng.choice(used)) for _ in range(k)], empty[:k]
            if sum(c.n[s] % page != 0 for s in src) > free:
                continue
            before = c.bytes()
            for a, b, part in c.fork(src, dst):
                for x in before[:2]:
                    x[:, b, :, :part] = x[:, a, :, :part]
                for x in before[2:]:
                    x[:, b] = x[:, a]
            for a, b in zip(src, dst):
                want[b] = want[a]
            assert all(torch.equal(x, y) for x, y in zip(before, c.bytes()))   # nothing else changes
        elif op == "free" and used:
            c.free([int(s) for s in rng.permutation(used)[:rng.integers(1, len(used) + 1)]])
        elif op == "compact":
            before = c.bytes()
            for a, b in c.compact():
                for x in before:
                    x[:, b] = x[:, a]
            assert all(torch.equal(x, y) for x, y in zip(before, c.bytes()))
        c.check(f"step {step} {op}")
        used = [s for s in range(c.max_seqs) if c.n[s]]
        if used:
            flat = [torch.full((c.L, len(used), c.H, S, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            M.mot_paged_load(c.h, c.c, i32(used), len(used), *flat)
            for i, s in enumerate(used):
                for x, y in zip(flat, want[s]):
                    assert torch.equal(x[:, i, :, :c.n[s]].double(), y), (step, op, s)
                    assert bool((x[:, i, :, c.n[s]:] == 7.0).all())   # other positions are left
    assert c.status() == M.MOT_OK


@pytest.mark.parametrize("d,page", [(64, 16), (128, 16), (64, 128), (128, 64), (128, 128)])
def test_store_takes_the_least_scale_and_rounds_once(d, page):
    """Pages whose largest values lie at the borders of a scale, pages of zeros, of tiny and of huge values, and
    values that 8 bits do not hold; the unfilled rows of a page and the other pages stay."""
    c = P8.Cache(layers=3, kv_heads=2, d=d, page=page, n_pages=40, max_pages=8)
    n = 4 * page + 5
    c.reserve([2, 0], [n, 1])
    flat = [c.normal(2, 3, 2, n + 2, d) for _ in range(2)]
    k = flat[0]
    k[0, 0, 0, :page] = 0.0                              # nothing but zeros: the least scale
    k[0, 0, 1, :page] = k[0, 0, 1, :page].clamp(-1, 1)
    k[0, 0, 1, 3, 5] = 1.75 * 2.0 ** 11                  # 448 2^3 exactly
    k[0, 0, 0, page:2 * page] *= 0.1
    k[0, 0, 0, page, 0] = -1.7578125 * 2.0 ** 11         # the next bf16 above it
    k[0, 0, 1, page:2 * page] *= 2.0 ** -90              # below the least scale
    k[1, 0, 0, page:2 * page] *= 2.0 ** 66               # near the largest
    k[1, 0, 1, page, :6] = torch.tensor([math.inf, -math.inf, math.nan, 3e38, 1.75 * 2.0 ** 68, -1.7578125 * 2.0 ** 68])
    k[1, 0, 0, 2 * page, 1] = math.nan                   # in a page of ordinary ones
    k[1, 0, 1, 2 * page:3 * page] = math.inf             # nothing that is held
    before = c.bytes()
    M.mot_paged_store(c.h, c.c, i32([2, 0]), 2, *flat, first_layer=1)
    assert c.status() == M.MOT_OK
    want = [None, None]
    for x, (raw, scale, f) in enumerate(((before[0], before[2], flat[0]), (before[1], before[3], flat[1]))):
        want[x] = raw.view(P8.F8).double()
        for i, s in ((0, 2), (1, 0)):
            for j, p in enumerate(c.t[s]):
                m = min(page, c.n[s] - j * page)
                for l in range(2):
                    y, sc = _stored(f[l, i, :, j * page:j * page + m].double())
                    scale[1 + l, p] = sc.float()
                    want[x][1 + l, p, :, :m] = y / sc[:, None, None]
    assert torch.equal(c.ks, before[2]) and torch.equal(c.vs, before[3])
    for got, y in zip((c.k, c.v), want):
        assert P8.same(got.double(), y)
    back = [torch.zeros_like(f) for f in flat]
    M.mot_paged_load(c.h, c.c, i32([2, 0]), 2, *back, first_layer=1)
    assert c.status() == M.MOT_OK
    pools = c.pools()
    for i, s in ((0, 2), (1, 0)):
        for b, x in zip(back, pools):
            y = x[1:3, c.t[s]].permute(0, 2, 1, 3, 4).reshape(2, 2, -1, d)[:, :, :c.n[s]]
            assert P8.same(b[:, i, :, :c.n[s]].double(), y.bfloat16().double())
            assert not bool(b[:, i, :, c.n[s]:].any()) and not bool(b[:, 2].any())


@pytest.mark.parametrize("factor", [0.25, 64.0])
def test_a_store_that_cuts_a_page_keeps_the_rows_behind_it(factor):
    """A contiguous cache that ends inside a page: the rows behind it stay, rounded again where the scale rises."""
    c = P8.Cache(layers=1, d=64, page=32, n_pages=9)
    c.reserve([1], [50])
    M.mot_paged_store(c.h, c.c, i32([1]), 1, *[c.normal(1, 1, 2, 50, 64) for _ in range(2)])
    assert c.status() == M.MOT_OK
    old, was = [x.double() for x in (c.k, c.v)], [c.ks.double(), c.vs.double()]
    flat = [c.normal(1, 1, 2, 40, 64) * factor for _ in range(2)]
    M.mot_paged_store(c.h, c.c, i32([1]), 1, *flat)
    assert c.status() == M.MOT_ERR_PAGES   # it says that the sequence is longer
    p = c.t[1][1]
    for x, s, o, w, f in zip((c.k, c.v), (c.ks, c.vs), old, was, flat):
        for hk in range(2):
            sc, kept, new = P8.joined(o[0, p, hk, 8:18], w[0, p, hk], f[0, 0, hk, 32:].double())
            assert float(s[0, p, hk]) == float(sc)
            assert torch.equal(x[0, p, hk, :8].double(), new) and torch.equal(x[0, p, hk, 8:18].double(), kept)
            assert torch.equal(x[0, p, hk, 18:].double(), o[0, p, hk, 18:])


def test_scales_without_an_initial_value():
    """NaN in the scales' memory: stores write them, and nothing of it is met."""
    c = P8.Cache(layers=2, d=64, page=16, n_pages=5)
    c.ks.fill_(math.nan)
    c.vs.fill_(math.nan)
    c.reserve([0], [20])
    flat = [c.normal(2, 1, 2, 20, 64) for _ in range(2)]
    M.mot_paged_store(c.h, c.c, i32([0]), 1, *flat)
    assert c.status() == M.MOT_OK
    for x, f in zip(c.pools(), flat):
        assert torch.equal(x[:, c.t[0]].permute(0, 2, 1, 3, 4).reshape(2, 2, -1, 64)[:, :, :20], _kept(f[:, 0].double(), 16))


def test_refusals():
    c = P8.Cache()
    c.reserve([0], [2])

    def refused(call, status=M.MOT_ERR_INVALID_ARG):
        with pytest.raises(M.MotError) as e:
            call()
        assert e.value.status == status

    refused(lambda: M.mot_create_paged8(M.make_paged_config(1, 4, 2, 64, 16, 40, 8, 16, dtype="fp32")), M.MOT_ERR_UNSUPPORTED)
    flat = [c.normal(1, 1, 2, 16, 64) for _ in range(2)]
    parts = dict(k=c.k, v=c.v, table=c.table, lens=c.lens, refs=c.refs, k_scale=c.ks, v_scale=c.vs)

    def with_(**change):
        return M.paged_cache(**dict(parts, **change))

    for change in (dict(k_scale=None), dict(v_scale=None), dict(k_scale=c.ks.double()), dict(v_scale=c.vs[:, :20].contiguous()),
                   dict(k_scale=c.ks.cpu()), dict(k_scale=c.vs), dict(v_scale=c.ks.data_ptr() + 2),
                   dict(k_scale=c.v.data_ptr()), dict(k=c.normal(1, 40, 2, 16, 64)), dict(v=c.v[:, :39])):
        refused(lambda: M.mot_paged_store(c.h, with_(**change), i32([0]), 1, *flat))
        refused(lambda: M.mot_paged_free(c.h, with_(**change), i32([0]), 1))
    refused(lambda: M.mot_paged_load(c.h, c.c, i32([0]), 1, flat[0], flat[0]))
    fp = [x.float() for x in flat]
    refused(lambda: M.mot_paged_store(c.h, c.c, i32([0]), 1, *fp))
    plain = P.Cache()   # a cache of 16 bits with a handle of 8, and the other way round
    refused(lambda: M.mot_paged_free(c.h, plain.c, i32([0]), 1))
    refused(lambda: M.mot_paged_free(plain.h, c.c, i32([0]), 1))
    M.mot_paged_store(c.h, c.c, i32([0]), 1, *flat)
    assert c.status() == M.MOT_OK
