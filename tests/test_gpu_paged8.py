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


# ---------------------------------------------------------------- append

def _turned(x, angle, pairs):
    y, rot = x.clone(), 2 * angle.shape[1]
    if not rot:
        return y
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * c - b * s, b * c + a * s
    if pairs:
        y[..., 0:rot:2], y[..., 1:rot:2] = u, v
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = u, v
    return y


def _check_pages(c, before, layer, seqs, new, keys, slop, values):
    """The pools and scales after an append, from those before it ([k, v, k scales, v scales] in 64 bits) and the
    rows' keys and values in 64 bits: values, old rows and what was not touched exactly, new keys within their
    rounding and `slop` (largest of a row's, [rows][heads])."""
    at = 0
    now = [x.double() for x in (c.k, c.v, c.ks, c.vs)]
    touched = torch.ones((c.L, c.n_pages), dtype=torch.bool, device="cuda")
    for s, m in zip(seqs, new):
        a = c.n[s] - m
        while a < c.n[s]:
            b = min(c.n[s], (a // c.P + 1) * c.P)
            p, o, r = c.t[s][a // c.P], a % c.P, slice(at, at + b - a)
            touched[layer, p] = False
            for hk in range(c.H):
                was, old = before[3][layer, p, hk], before[1][layer, p, hk, :o]
                sc, kept, fresh = P8.joined(old, was, values[r, hk])
                assert float(now[3][layer, p, hk]) == float(sc), (s, a, hk)
                assert P8.same(now[1][layer, p, hk, :o], kept) and P8.same(now[1][layer, p, hk, o:o + b - a], fresh)
                was, old, x = before[2][layer, p, hk], before[0][layer, p, hk, :o], keys[r, hk]
                top, off = P8.largest(x, (0, 1)), slop[r, hk].max()
                sc = now[2][layer, p, hk]
                lo, hi = (P8.scale_of((top + e * off).clamp_min(0)) for e in (-1, 1))
                if o:
                    lo, hi = torch.maximum(lo, was), torch.maximum(hi, was)
                assert float(sc) in (float(lo), float(hi)), (s, a, hk)
                if o:
                    assert P8.same(now[0][layer, p, hk, :o], P8.eighths(old * (was / sc)))
                got = now[0][layer, p, hk, o:o + b - a] * sc
                # half a step: 2^-4 of the value, 2^-10 of the scale at the least
                P.assert_close(got, x, 2.0 ** -4 * x.abs() + 2.0 ** -10 * sc + 2 * slop[r, hk][:, None], f"k {s} {a} {hk}")
                for x_, y_ in ((now[0], before[0]), (now[1], before[1])):   # the page's rows behind
                    assert P8.same(x_[layer, p, hk, o + b - a:], y_[layer, p, hk, o + b - a:])
            at += b - a
            a = b
    for x, y in zip(now, before):
        assert P8.same(x[touched], y[touched])


APPEND = [
    # q heads, kv heads, d, page, rot, pairs, norm, axes
    (12, 2, 128, 16, 128, False, False, False),
    (5, 5, 64, 32, 64, True, True, False),
    (14, 2, 64, 64, 32, False, True, True),
    (16, 1, 128, 128, 0, False, True, False),
    (3, 3, 128, 16, 48, True, False, True),
    (12, 12, 64, 16, 0, False, False, False),
    (28, 4, 128, 64, 128, False, True, True),
]


@pytest.mark.parametrize("new", [[5, 2, 0, 1], [1, 1, 1, 1], [150, 2, 37, 1], [16, 1, 0, 64]])
@pytest.mark.parametrize("hq,h,d,page,rot,pairs,norm,axes", APPEND)
def test_append_matches_the_formula(hq, h, d, page, rot, pairs, norm, axes, new):
    base, eps = 1e6, 1e-5
    c = P8.Cache(layers=2, q_heads=hq, kv_heads=h, d=d, page=page, n_pages=60, max_pages=20, rot_dim=rot, rot_pairs=pairs,
                 rot_base=base, norm_eps=eps)
    seqs = [3, 0, 5, 2]
    c.reserve(seqs, [m + x for m, x in zip(new, (page + 3, 0, 19, 5))])
    rows = sum(new)
    x = c.normal(rows + 3, hq + 2 * h, d) * 3
    x[:, :, d // 2] *= 6
    w = [(1 + 0.2 * c.normal(d)).bfloat16() for _ in range(2)] if norm else [None, None]
    starts = [1 + sum(new[:i]) for i in range(5)]
    b = M.paged_batch(i32(seqs), i32(starts), 4, rows + 3, max(new))
    out = torch.full((rows + 3, hq, d), 9.0, dtype=torch.bfloat16, device="cuda")
    before = [t.double() for t in (c.k, c.v, c.ks, c.vs)]
    args = x[:, :hq], x[:, hq:hq + h], x[:, hq + h:], out, *w
    rate = base ** (-2 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / max(rot, 1))
    if axes:
        at = torch.randint(-5000, 5000, (3, rows + 3), generator=c.gen, device="cuda", dtype=torch.int32)
        M.mot_paged_set_axes(c.h, 3, [i % 3 for i in range(rot // 2)])
        M.mot_paged_append_at(c.h, 1, c.c, b, at, *args)
        angle = at[torch.arange(rot // 2, device="cuda") % 3].T[1:1 + rows].double() * rate
    else:
        M.mot_paged_append(c.h, 1, c.c, b, *args)
        pos = torch.cat([torch.arange(c.n[s] - m, c.n[s]) for s, m in zip(seqs, new)]).cuda()
        angle = pos.double()[:, None] * rate
    assert c.status() == M.MOT_OK
    y = x[1:1 + rows].double()

    def expect(z, weight):
        if weight is not None:
            z = z * (z.square().mean(2, keepdim=True) + eps).rsqrt() * weight.double()
        # fp32 on the way, as in 16 bits; without norm and rotation the values are the inputs
        return _turned(z, angle, pairs), (2.0 ** -20 if norm or rot else 0.0) * z.abs().amax(2, keepdim=True)

    want, slop = expect(y[:, :hq], w[0])
    half = P.HALF["bf16"] if norm or rot else 0.0
    P.assert_close(out[1:1 + rows], want, half * want.abs() + slop, "q")
    assert bool((out[0] == 9).all()) and bool((out[1 + rows:] == 9).all())
    keys, slop = expect(y[:, hq:hq + h], w[1])
    _check_pages(c, before, 1, seqs, new, keys, slop[..., 0], y[:, hq + h:])


def test_rows_that_come_one_by_one_and_grow():
    """Single tokens into two pages, each of a larger range than the one before, then smaller ones: a scale only
    rises, old rows are rounded again and again; zeros first, and values that 8 bits do not hold among them."""
    c = P8.Cache(q_heads=2, kv_heads=2, d=64, page=16, n_pages=6, rot_dim=0)
    c.ks.fill_(math.nan)
    c.vs.fill_(math.nan)
    for step in range(40):
        c.reserve([1, 4], [1, 1])
        x = c.normal(2, 6, 64) * (0.0 if step == 0 else 2.0 ** (step % 16 if step < 24 else 16 - step % 16))
        if step == 3:
            x[0, 2, 5], x[1, 4, 6], x[1, 5, :] = math.inf, math.nan, -math.inf
        out = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
        before = [t.double() for t in (c.k, c.v, c.ks, c.vs)]
        M.mot_paged_append(c.h, 0, c.c, c.batch([1, 4], [1, 1]), x[:, :2], x[:, 2:4], x[:, 4:], out)
        assert c.status() == M.MOT_OK
        y = x.double()
        if step != 3:
            _check_pages(c, before, 0, [1, 4], [1, 1], y[:, 2:4], torch.zeros((2, 2), dtype=torch.float64, device="cuda"), y[:, 4:])
        else:
            assert bool(c.k[0, c.t[1][0], 0, 3, 5].double().isnan()) and int(c.k.double().isnan().sum()) == 1
            assert bool(c.v[0, c.t[4][0], 1, 3].double().isnan().all()) and int(c.v.double().isnan().sum()) == 65
            assert bool(torch.isfinite(c.ks[0, [c.t[1][0], c.t[4][0]]]).all())


@pytest.mark.parametrize("d,page,new", [(128, 128, 300), (64, 128, 200), (128, 64, 70), (64, 32, 40), (128, 16, 5)])
def test_values_that_8_bits_do_not_hold_among_many_rows(d, page, new):
    """Infinities, NaN and values above 448 2^60, in the first rows of a page, its last, and alone in one: they become
    NaN and have no part in the scale, in rows that stay in registers, that wait in shared memory and that do not."""
    c = P8.Cache(q_heads=2, kv_heads=2, d=d, page=page, n_pages=30, max_pages=24)
    c.reserve([2], [new + 3])
    x = c.normal(new, 6, d)
    x[0, 2, 1], x[1, 3, d - 1], x[2, 4, 5], x[3, 5, 7] = math.inf, math.nan, -3e38, 1.7578125 * 2.0 ** 68
    x[new - 1, 2:, 3] = torch.tensor([math.nan, -math.inf, 1.75 * 2.0 ** 68, math.inf], device="cuda").bfloat16()
    x[new // 2, 3], x[new // 2, 4] = math.inf, math.nan
    out = torch.zeros((new, 2, d), dtype=torch.bfloat16, device="cuda")
    before = [t.double() for t in (c.k, c.v, c.ks, c.vs)]
    M.mot_paged_append(c.h, 0, c.c, c.batch([2], [new]), x[:, :2], x[:, 2:4], x[:, 4:], out)
    assert c.status() == M.MOT_OK
    y = x.double()
    for pool, scale, old_pool, was, z in ((c.k, c.ks, before[0], before[2], y[:, 2:4]), (c.v, c.vs, before[1], before[3], y[:, 4:])):
        a = 3
        while a < c.n[2]:
            b = min(c.n[2], (a // page + 1) * page)
            p, o = c.t[2][a // page], a % page
            for hk in range(2):
                sc, kept, fresh = P8.joined(old_pool[0, p, hk, :o], was[0, p, hk], z[a - 3:b - 3, hk])
                assert float(scale[0, p, hk]) == float(sc), (a, hk)
                assert P8.same(pool[0, p, hk, :o].double(), kept) and P8.same(pool[0, p, hk, o:o + b - a].double(), fresh)
            a = b


@pytest.mark.parametrize("n,hints", [(700, (14, 1)), (1500, (14, 17))])
def test_many_entries_and_a_hint_that_is_wrong(n, hints):
    """More entries than a block has threads, some without rows; the same with a max_chunk of one, which bounds nothing
    that is right, and with one that picks the other way of dealing out the pages."""
    got = []
    for hint in hints:
        c = P8.Cache(q_heads=2, kv_heads=1, d=64, page=16, n_pages=2 * n, max_seqs=n, max_pages=3, rot_dim=64, seed=1)
        new = [(i * 7) % 15 for i in range(n)]
        c.reserve(list(range(n)), [m + i % 9 for i, m in enumerate(new)])
        rows = sum(new)
        x = c.normal(rows, 4, 64)
        starts = [sum(new[:i]) for i in range(n + 1)]
        out = torch.zeros((rows, 2, 64), dtype=torch.bfloat16, device="cuda")
        before = [t.double() for t in (c.k, c.v, c.ks, c.vs)]
        M.mot_paged_append(c.h, 0, c.c, M.paged_batch(i32(list(range(n))), i32(starts), n, rows, hint), x[:, :2], x[:, 2:3],
                           x[:, 3:], out)
        assert c.status() == M.MOT_OK
        got.append(c.bytes() + [out])
    assert all(torch.equal(a, b) for a, b in zip(*got))
    if n > 1000:
        return
    y = x.double()
    pos = torch.cat([torch.arange(c.n[s] - m, c.n[s]) for s, m in enumerate(new)]).cuda()
    angle = pos.double()[:, None] * 1e4 ** (-2 * torch.arange(32, dtype=torch.float64, device="cuda") / 64)
    keys = _turned(y[:, 2:3], angle, False)
    _check_pages(c, before, 0, list(range(n)), new, keys, 2.0 ** -20 * keys.abs().amax(2), y[:, 3:])


def test_append_and_store_do_nothing_behind_a_refused_change():
    c = P8.Cache(n_pages=4, max_pages=4)
    c.reserve([0], [20])
    before = c.bytes()
    c.reserve([1], [64], ok=False)
    x, out = c.normal(3, 8, 64), torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    M.mot_paged_store(c.h, c.c, i32([0]), 1, *[c.normal(1, 1, 2, 32, 64) for _ in range(2)])
    M.mot_paged_append(c.h, 0, c.c, c.batch([0], [3]), x[:, :4], x[:, 4:6], x[:, 6:], out)
    assert c.status() == M.MOT_ERR_PAGES
    assert all(torch.equal(a, b) for a, b in zip(before, c.bytes())) and not bool(out.any())


def test_appends_of_entries_out_of_range_write_nothing():
    """A slot outside the table, a table entry outside the pool, rows before position 0, a negative length."""
    c = P8.Cache(n_pages=8, max_pages=4, rot_dim=64)
    c.reserve([0, 1, 2, 3], [20, 20, 3, 5])
    c.table[1, 1] = 4711
    c.lens[3] = -5
    before = [t.double() for t in (c.k, c.v, c.ks, c.vs)]
    for new in ([2, 2, 5, 2, 2], [1, 1, 1, 1, 1], [19, 19, 4, 3, 1]):
        x = c.normal(sum(new), 8, 64)
        out = torch.zeros((sum(new), 4, 64), dtype=torch.bfloat16, device="cuda")
        M.mot_paged_append(c.h, 0, c.c, c.batch([99, 1, 2, 3, 0], new), x[:, :4], x[:, 4:6], x[:, 6:], out)
        assert c.status() == M.MOT_ERR_PAGES
        mine = set(c.t[0] + c.t[1][:1] + c.t[2])
        others = torch.tensor([p for p in range(8) if p not in mine], device="cuda")
        for a, b in zip((c.k, c.v, c.ks, c.vs), before):
            assert P8.same(a.double()[:, others], b[:, others])


# ---------------------------------------------------------------- attention

def _attend(c, seqs, new, layer=0, hint=None, q=None):
    q = c.normal(sum(new), c.Hq, c.d) if q is None else q
    out = torch.full((sum(new) + 1, c.Hq, c.d), 9.0, dtype=torch.bfloat16, device="cuda")
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    M.mot_paged_attention(c.h, layer, c.c, M.paged_batch(i32(seqs), i32(starts), len(seqs), sum(new),
                                                         max(new, default=0) if hint is None else hint), q, out)
    assert bool((out[-1] == 9).all())
    return q, out[:-1]


SHAPES = [
    # q heads, kv heads, d, page
    (12, 2, 128, 16), (7, 7, 64, 32), (14, 2, 64, 64), (16, 1, 128, 128), (28, 4, 128, 64), (3, 1, 64, 16),
]


@pytest.mark.parametrize("hq,h,d,page", SHAPES)
@pytest.mark.parametrize("lens,new", [
    ([1, 2, 15, 16, 17, 31], [1, 1, 1, 1, 1, 1]),                    # single tokens on the shortest sequences
    ([127, 128, 129, 300, 511], [1, 1, 1, 1, 1]),                    # around the tiles' ends
    ([1000, 3, 64, 500, 33], [2, 3, 1, 0, 4]),                       # a few tokens, an entry without any
    ([40, 200, 1, 129, 300], [40, 17, 1, 129, 33]),                  # chunks: whole sequences and pieces
    ([700], [300]), ([513], [257]),
])
def test_attention_matches_the_formula(hq, h, d, page, lens, new):
    c = P8.Cache(layers=2, q_heads=hq, kv_heads=h, d=d, page=page, n_pages=130, max_seqs=8, max_pages=64, seed=len(lens))
    seqs = [3, 0, 5, 2, 7, 1][:len(lens)]
    c.reserve(seqs, lens)
    q, out = _attend(c, seqs, new, layer=1)
    assert c.status() == M.MOT_OK
    P8.check_attention(c, seqs, new, q, out, layer=1)


@pytest.mark.parametrize("hint", [1, 5000])
def test_a_hint_of_the_chunks_that_is_wrong(hint):
    """max_chunk bounds the work, never the result: the same rows under hints that pick other kernels."""
    c = P8.Cache(q_heads=6, kv_heads=2, d=128, page=32, n_pages=60, max_pages=32)
    c.reserve([0, 1, 2], [300, 64, 700])
    q, out = _attend(c, [0, 1, 2], [200, 1, 30], hint=hint)
    assert c.status() == M.MOT_OK
    P8.check_attention(c, [0, 1, 2], [200, 1, 30], q, out)


@pytest.mark.parametrize("new", [1, 70])
def test_scales_of_very_different_pages(new):
    """Value scales from 2^-60 to 2^60 from page to page, in front and behind; key scales of several steps."""
    for order in (1, -1):
        c = P8.Cache(q_heads=4, kv_heads=2, d=64, page=16, n_pages=40, max_pages=32)
        c.reserve([0], [400])
        e = torch.linspace(-60 * order, 60 * order, 25).round().cuda()
        c.vs[0, c.t[0]] = torch.exp2(e)[:, None].expand(-1, 2)
        c.ks[0, c.t[0]] = torch.exp2(-10 + torch.arange(25, device="cuda").float() % 5)[:, None]
        q, out = _attend(c, [0], [new])
        assert c.status() == M.MOT_OK
        P8.check_attention(c, [0], [new], q, out, label=f"order {order}")
        # pages of small values whose keys have all the weight: what is left of the large ones decides
        c.vs[0, c.t[0]] = torch.exp2(torch.tensor([-60.0, 60.0, 0.0, -30.0] * 7, device="cuda")[:25])[:, None]
        q, out = _attend(c, [0], [new])
        P8.check_attention(c, [0], [new], q, out, label=f"mixed {order}")


@pytest.mark.parametrize("new", [1, 3, 90])
def test_what_is_not_seen_is_not_met(new):
    """NaN in every position behind the sequence, in pages that nobody holds, in their scales, and in the new
    positions that a row does not see."""
    c = P8.Cache(q_heads=8, kv_heads=2, d=128, page=64, n_pages=12, max_pages=8)
    c.reserve([0, 1], [203, 150])
    nan = torch.tensor(127, dtype=torch.uint8, device="cuda")
    held = {p for s in (0, 1) for p in c.t[s]}
    for x in (c.k.view(torch.uint8), c.v.view(torch.uint8)):
        for s in (0, 1):
            x[0, c.t[s][-1], :, c.n[s] % 64:] = nan
        for p in range(12):
            if p not in held:
                x[0, p] = nan
    for p in range(12):
        if p not in held:
            c.ks[0, p], c.vs[0, p] = math.nan, math.inf
    q, clean = _attend(c, [0, 1], [new, new])
    P8.check_attention(c, [0, 1], [new, new], q, clean)
    # the last new position of slot 0 holds NaN in one dimension of one head's value: that row's heads alone meet it
    p, o = c.t[0][202 // 64], 202 % 64
    c.v.view(torch.uint8)[0, p, 1, o, 77] = 255
    _, out = _attend(c, [0, 1], [new, new], q=q)
    want = clean.clone()
    want[new - 1, 4:, 77] = math.nan
    assert P8.same(out, want)
    # the same of a key: the rows that see it are NaN in that head
    c.k.view(torch.uint8)[0, p, 0, o, 5] = 127
    _, out = _attend(c, [0, 1], [new, new], q=q)
    want[new - 1, :4] = math.nan
    assert P8.same(out, want)
    assert c.status() == M.MOT_OK


@pytest.mark.parametrize("new", [2, 200])
def test_a_value_that_is_nan_in_the_middle_of_what_rows_see(new):
    """A NaN value that the first rows of a chunk do not see and the later ones do."""
    c = P8.Cache(q_heads=4, kv_heads=1, d=64, page=16, n_pages=40, max_pages=32)
    c.reserve([0], [333])
    q, clean = _attend(c, [0], [new])
    at = 333 - new + new // 2
    c.v.view(torch.uint8)[0, c.t[0][at // 16], 0, at % 16, [0, 31, 63]] = 127
    _, out = _attend(c, [0], [new], q=q)
    want = clean.clone()
    want[new // 2:, :, [0, 31, 63]] = math.nan
    assert P8.same(out, want)


@pytest.mark.parametrize("new", [1, 60])
def test_queries_of_every_size_and_ones_that_are_not_finite(new):
    """Rows of zeros, of the smallest and of large values; an infinity or a NaN makes its own row NaN."""
    c = P8.Cache(q_heads=8, kv_heads=1, d=64, page=16, n_pages=20)
    c.reserve([0], [200])
    q = c.normal(new, 8, 64)
    q[:, 0] = 0.0
    q[:, 1] *= 2.0 ** -130
    q[:, 2] *= 2.0 ** -20
    q[:, 3] *= 2.0 ** 6
    q[:, 4, 1:] *= 2.0 ** -40
    q[:, 5, 9], q[:, 6, 63] = math.inf, math.nan
    _, out = _attend(c, [0], [new], q=q)
    assert bool(out[:, 5:7].isnan().all())
    q[:, 5:7], out[:, 5:7] = q[:, :1], out[:, :1]
    P8.check_attention(c, [0], [new], q, out)


def test_rows_before_the_first_position_are_zeros():
    c = P8.Cache(q_heads=4, kv_heads=2, d=64, page=16, n_pages=20)
    for n, new in ((3, 5), (0, 2), (50, 90)):
        c.reserve([1], [n])
        q, out = _attend(c, [1], [new])
        assert not bool(out[:new - n].any())
        P8.check_attention(c, [1], [new], q, out)
        c.free([1])


def test_entries_out_of_range_are_reported():
    c = P8.Cache(q_heads=4, kv_heads=2, d=64, page=16, n_pages=20)
    c.reserve([0, 1], [100, 90])
    c.table[1, 2] = 20
    for new in (1, 50):
        q, out = _attend(c, [0, 1], [new, new])
        assert c.status() == M.MOT_ERR_PAGES
        P8.check_attention(c, [0], [new], q, out)
        q, out = _attend(c, [0, 44], [new, new])
        assert c.status() == M.MOT_ERR_PAGES
        P8.check_attention(c, [0], [new], q, out)


def test_many_sequences_of_different_lengths():
    rng = np.random.default_rng(5)
    n = 150
    c = P8.Cache(q_heads=8, kv_heads=2, d=64, page=32, n_pages=4000, max_seqs=n, max_pages=40)
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(1200), n))]
    c.reserve(list(range(n)), lens)
    for new in ([1] * n, [min(x, int(rng.integers(0, 9))) for x in lens], [min(x, 1 + 30 * (i % 40 == 0)) for i, x in enumerate(lens)]):
        q, out = _attend(c, list(range(n)), new)
        assert c.status() == M.MOT_OK
        P8.check_attention(c, list(range(n)), new, q, out)


def test_offsets_beyond_32_bits():
    """Pages whose bytes lie behind 2^32 of a pool, in a later layer."""
    c = P8.Cache(layers=1, q_heads=2, kv_heads=1, d=128, page=128, n_pages=4, max_pages=4)
    pages = 1 << 18   # 4 GB a layer
    pool = [torch.zeros((2, pages, 1, 128, 128), dtype=torch.uint8, device="cuda").view(P8.F8) for _ in range(2)]
    scales = [torch.ones((2, pages, 1), device="cuda") for _ in range(2)]
    table, lens = i32([[pages - 1, 7, pages - 2]]), i32([300])
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    h = M.mot_create_paged8(M.make_paged_config(2, 2, 1, 128, 128, pages, 1, 3))
    cache = M.paged_cache(*pool, table, lens, refs, *scales)
    c.reserve([0], [300])
    for mine, there in zip((c.k, c.v, c.ks, c.vs), (*pool, *scales)):
        for a, b in zip(c.t[0], (pages - 1, 7, pages - 2)):
            there[1, b].copy_(mine[0, a])
    for new in (1, 100):
        q, out = _attend(c, [0], [new])
        far = torch.zeros((new, 2, 128), dtype=torch.bfloat16, device="cuda")
        M.mot_paged_attention(h, 1, cache, M.paged_batch(i32([0]), i32([0, new]), 1, new), q, far)
        assert M.mot_get_device_status(h) == M.MOT_OK
        assert torch.equal(out, far)
    x = c.normal(40, 4, 128)
    outs = [torch.zeros((40, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    M.mot_paged_append(c.h, 0, c.c, c.batch([0], [40]), x[:, :2], x[:, 2:3], x[:, 3:], outs[0])
    M.mot_paged_append(h, 1, cache, M.paged_batch(i32([0]), i32([0, 40]), 1, 40), x[:, :2], x[:, 2:3], x[:, 3:], outs[1])
    for mine, there in zip((c.k, c.v, c.ks, c.vs), (*pool, *scales)):
        for a, b in zip(c.t[0], (pages - 1, 7, pages - 2)):
            assert torch.equal(mine[0, a].view(torch.uint8), there[1, b].view(torch.uint8))
    flat = [torch.zeros((1, 1, 1, 300, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    M.mot_paged_load(h, cache, i32([0]), 1, *flat, first_layer=1)
    for f, x in zip(flat, c.rows(0)):
        assert torch.equal(f[0, 0].double(), x)


# ---------------------------------------------------------------- together

def test_from_a_translated_context_to_branches_that_grow():
    """A contiguous context stored, forked to branches, each with a prompt and then single tokens, captured and
    replayed on another stream: every step's attention is that of the rows held, and branches do not meet."""
    Hq, H, d, L = 8, 2, 64, 2
    c = P8.Cache(layers=L, q_heads=Hq, kv_heads=H, d=d, page=16, n_pages=120, max_seqs=6, max_pages=16, rot_dim=64)
    c.reserve([0], [75])
    flat = [c.normal(L, 1, H, 75, d) for _ in range(2)]
    M.mot_paged_store(c.h, c.c, i32([0]), 1, *flat)
    c.fork([0, 0, 0], [1, 3, 5])
    c.check("fork")
    kids = [1, 3, 5]
    for new in ([20, 1, 64], [1, 1, 1]):
        c.reserve(kids, new)
        rows = sum(new)
        b = c.batch(kids, new)
        for l in range(L):
            x = c.normal(rows, Hq + 2 * H, d)
            q = torch.zeros((rows, Hq, d), dtype=torch.bfloat16, device="cuda")
            out = torch.zeros_like(q)
            before = [t.double() for t in (c.k, c.v, c.ks, c.vs)]
            M.mot_paged_append(c.h, l, c.c, b, x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], q)
            M.mot_paged_attention(c.h, l, c.c, b, q, out)
            pos = torch.cat([torch.arange(c.n[s] - m, c.n[s]) for s, m in zip(kids, new)]).cuda()
            angle = pos.double()[:, None] * 1e4 ** (-2 * torch.arange(32, dtype=torch.float64, device="cuda") / 64)
            keys = _turned(x[:, Hq:Hq + H].double(), angle, False)
            _check_pages(c, before, l, kids, new, keys, 2.0 ** -20 * keys.abs().amax(2), x[:, Hq + H:].double())
            P8.check_attention(c, kids, new, q, out, layer=l)
    # a decoding step as a graph
    st = torch.cuda.Stream()
    seqs, starts = i32(kids), i32([0, 1, 2, 3])
    b = M.paged_batch(seqs, starts, 3, 3, 1)
    x = c.normal(L, 3, Hq + 2 * H, d)
    q, out = (torch.zeros((L, 3, Hq, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def step(stream):
        M.mot_paged_reserve(c.h, c.c, b, stream=stream)
        for l in range(L):
            y = x[l]
            M.mot_paged_append(c.h, l, c.c, b, y[:, :Hq], y[:, Hq:Hq + H], y[:, Hq + H:], q[l], stream=stream)
            M.mot_paged_attention(c.h, l, c.c, b, q[l], out[l], stream=stream)

    def follow():   # the same on the lists
        for s in kids:
            c.t[s] += c.take(c.pages(c.n[s] + 1) - c.pages(c.n[s]))
            c.n[s] += 1

    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        step(st)
    follow()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        step(torch.cuda.current_stream())
    for _ in range(20):
        x.copy_(c.normal(L, 3, Hq + 2 * H, d))
        g.replay()
        follow()
        torch.cuda.synchronize()
        for l in range(L):
            P8.check_attention(c, kids, [1, 1, 1], q[l], out[l], layer=l)
    c.check("replays")
    back = [torch.zeros((L, 1, H, 75, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    M.mot_paged_load(c.h, c.c, i32([0]), 1, *back)   # the context itself is as it was stored
    for x, y in zip(back, flat):
        assert torch.equal(x[:, 0].double(), _kept(y[:, 0].double(), 16))
    assert c.status() == M.MOT_OK


def test_two_handles_on_two_streams_serve_one_cache():
    """Sequences of one cache under a handle of their own each, at the same time: both give what they give alone."""
    shape = dict(q_heads=6, kv_heads=2, d=128, page=32, n_pages=200, max_seqs=8, max_pages=64)
    c = P8.Cache(**shape)
    other = M.mot_create_paged8(M.make_paged_config(1, *shape.values()))
    c.reserve(list(range(6)), [900, 33, 700, 1500, 64, 5])
    parts = []
    for h, seqs, new in ((c.h, [0, 1, 2], [200, 1, 30]), (other, [3, 4, 5], [100, 2, 5]), (c.h, [2, 0], [1, 1]), (other, [5, 3], [1, 1])):
        rows = sum(new)
        x = c.normal(rows, 10, 128)
        q, out = (torch.zeros((rows, 6, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        parts.append((h, c.batch(seqs, new), x, q, out, torch.cuda.Stream()))

    def step(part, stream):
        h, b, x, q, out, _ = part
        M.mot_paged_append(h, 0, c.c, b, x[:, :6], x[:, 6:8], x[:, 8:], q, stream=stream)
        M.mot_paged_attention(h, 0, c.c, b, q, out, stream=stream)

    for a, b in (parts[:2], parts[2:]):   # chunks, then single tokens
        for part in (a, b):
            step(part, None)
        torch.cuda.synchronize()
        want = [part[4].clone() for part in (a, b)], c.bytes()
        for _ in range(20):
            for part in (a, b):
                part[4].zero_()
            torch.cuda.synchronize()
            for part in (a, b):
                step(part, part[5])
            torch.cuda.synchronize()
            for x, y in zip([part[4] for part in (a, b)] + c.bytes(), want[0] + want[1]):
                assert torch.equal(x, y)
    assert c.status() == M.MOT_OK and M.mot_get_device_status(other) == M.MOT_OK


@pytest.mark.parametrize("new", [[1, 1, 1], [150, 3, 40]])
def test_a_captured_step_behind_work_of_two_streams(new):
    """Calls whose launches may begin before the kernels in front of them have ended see what these write: inputs that
    two streams make, pages that the call before has written, one replay after another."""
    H, Hq, d = 2, 6, 128
    seqs, rows = [0, 1, 2], sum(new)
    pair = []
    for _ in range(2):
        c = P8.Cache(q_heads=Hq, kv_heads=H, d=d, page=32, n_pages=120, max_pages=32, rot_dim=d, seed=7)
        c.reserve(seqs + [3], [m + x for m, x in zip(new, (300, 33, 700))] + [90])
        x = c.normal(rows, Hq + 2 * H, d)
        flat, back = [[torch.zeros((1, 1, H, 90, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
        q, out = (torch.zeros((rows, Hq, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        pair.append((c, x, flat, back, q, out, c.batch(seqs, new), i32([3]), x.clone(), flat[0].clone()))

    def step(s, side):
        c, x, flat, back, q, out, b, slot, src, kv = s
        st = torch.cuda.current_stream()
        if side is not None:
            side.wait_stream(st)
        with torch.cuda.stream(side or st):
            for f in flat:
                f.copy_(kv).mul_(2)
        x.copy_(src).mul_(0.5)
        if side is not None:
            st.wait_stream(side)
        M.mot_paged_append(c.h, 0, c.c, b, x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], q)
        M.mot_paged_attention(c.h, 0, c.c, b, q, out)
        M.mot_paged_store(c.h, c.c, slot, 1, *flat)
        M.mot_paged_load(c.h, c.c, slot, 1, *back)
        x.copy_(out.repeat_interleave(2, 1)[:, :Hq + 2 * H])   # behind the calls: a kernel that overlaps nothing
        src.add_(x)

    eager, graph = pair
    st, side = torch.cuda.Stream(), torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        step(graph, side)
    for k in range(10):
        kv = torch.full_like(eager[9], 0.25 * (k + 1))
        for s in pair:
            s[9].copy_(kv)
        step(eager, side if k % 2 else None)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip((eager[1], *eager[3], eager[4], eager[5]), (graph[1], *graph[3], graph[4], graph[5])):
            assert torch.equal(a, b)
        assert torch.equal(eager[3][0], 2 * kv) and bool(eager[5].isfinite().all())
    for a, b in zip(eager[0].bytes(), graph[0].bytes()):
        assert torch.equal(a, b)
    assert eager[0].status() == M.MOT_OK and graph[0].status() == M.MOT_OK


def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right():
    """The first block loads nothing: every wait of the kernel ends, and nothing is left behind for the next call."""
    for d, new in ((64, 300), (128, 300), (64, 1), (128, 1), (128, 5)):
        c = P8.Cache(q_heads=4, kv_heads=2, d=d, page=16, n_pages=130, max_pages=128)
        c.reserve([0], [2000])
        q, want = _attend(c, [0], [new])
        M.mot_debug_set(c.h, True, 1_000_000)
        _attend(c, [0], [new], q=q)
        assert c.status() == M.MOT_ERR_TIMEOUT
        M.mot_debug_set(c.h, False)
        for _ in range(2):
            _, out = _attend(c, [0], [new], q=q)
            assert c.status() == M.MOT_OK
            assert torch.equal(out, want)
