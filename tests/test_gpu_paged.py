"""The paged cache on the GPU through the C ABI: its pages against lists, the append and the
attention against their formulas in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import _paged as P   # noqa: E402
M = P.M
i32 = P.i32


# ---------------------------------------------------------------- pages

@pytest.mark.parametrize("page,dtype,d", [(16, "bf16", 64), (32, "fp32", 64), (64, "bf16", 128), (128, "fp32", 128)])
def test_pages_over_a_random_run(page, dtype, d):
    """Reserve, fork, free, compact, store and load in a random order: the bookkeeping as lists have it,
    and every sequence's positions hold what was stored, whatever moves and is shared around them."""
    rng = np.random.default_rng(page + d)
    c = P.Cache(layers=3, kv_heads=3, q_heads=3, d=d, page=page, n_pages=23, max_seqs=7, max_pages=6, dtype=dtype)
    want = [None] * c.max_seqs   # a slot's keys and values, [2][layers][heads][len][d]
    S = c.max_pages * page

    def load(slots):
        flat = [torch.full((c.L, len(slots), c.H, S, d), 7.0, dtype=P.DT[dtype], device="cuda") for _ in range(2)]
        M.mot_paged_load(c.h, c.c, i32(slots), len(slots), *flat)
        return flat

    for step in range(60):
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
            # the grown sequences get new contents as a whole where they hold their pages alone
            alone = [s for s in seqs if all(c.r[p] == 1 for p in c.t[s])]
            if alone:
                flat = [c.normal(c.L, len(alone) + 1, c.H, S, d) for _ in range(2)]
                M.mot_paged_store(c.h, c.c, i32(alone), len(alone), *flat)
                for i, s in enumerate(alone):
                    want[s] = torch.stack([x[:, i, :, :c.n[s]] for x in flat])
            for s in set(seqs) - set(alone):   # stale contents behind the old length
                want[s] = torch.stack([x[:, c.t[s]].permute(0, 2, 1, 3, 4).reshape(c.L, c.H, -1, d)[:, :, :c.n[s]]
                                       for x in (c.k, c.v)])
        elif op == "fork" and used and empty:
            k = int(rng.integers(1, len(empty) + 1))
            src, dst = [int(rng.choice(used)) for _ in range(k)], empty[:k]
            if sum(c.n[s] % page != 0 for s in src) > free:
                continue
            before = [x.clone() for x in (c.k, c.v)]
            for a, b, part in c.fork(src, dst):
                for x in before:
                    x[:, b, :, :part] = x[:, a, :, :part]
            for a, b in zip(src, dst):
                want[b] = want[a]
            for x, y in zip(before, (c.k, c.v)):   # nothing else of the pools changes
                assert torch.equal(x, y)
        elif op == "free" and used:
            c.free([int(s) for s in rng.permutation(used)[:rng.integers(1, len(used) + 1)]])
        elif op == "compact":
            live = i32([-1])
            before = [x.clone() for x in (c.k, c.v)]
            moves = c.compact(live)
            assert int(live) == sum(x > 0 for x in c.r)
            for x, y in zip(before, (c.k, c.v)):
                for a, b in moves:
                    x[:, b] = x[:, a]
                assert torch.equal(x, y)
        c.check(f"step {step} {op}")
        used = [s for s in range(c.max_seqs) if c.n[s]]
        if used:
            flat = load(used)
            for i, s in enumerate(used):
                for x, y in zip(flat, want[s]):
                    assert torch.equal(x[:, i, :, :c.n[s]], y), (step, op, s)
                    assert bool((x[:, i, :, c.n[s]:] == 7.0).all())   # other positions are left
    assert c.status() == M.MOT_OK


def test_refused_changes_change_nothing_until_the_status_is_read():
    c = P.Cache(n_pages=8, max_seqs=5, max_pages=4, page=16)
    c.reserve([0, 1], [40, 16])   # 3 + 1 pages
    c.check()

    def refuse(call):
        call()
        c.check()
        c.free([0], ok=False)   # nothing moves behind a refused change
        M.mot_paged_compact(c.h, c.c)
        c.check("behind a refused change")
        assert c.status() == M.MOT_ERR_PAGES
        assert c.status() == M.MOT_OK   # read and cleared

    refuse(lambda: c.reserve([2, 2], [1, 1], ok=False))            # a slot twice
    refuse(lambda: c.reserve([2, 5], [1, 1], ok=False))            # outside the table
    refuse(lambda: c.reserve([-1], [1], ok=False))
    refuse(lambda: c.reserve([1], [49], ok=False))                 # beyond max_pages P
    refuse(lambda: c.reserve([2, 3], [16, 64], ok=False))          # 5 pages of 4
    refuse(lambda: M.mot_paged_reserve(c.h, c.c, M.paged_batch(i32([2, 3]), i32([0, 4, 2]), 2, 4)))   # starts fall
    refuse(lambda: c.fork([0], [1], ok=False))                     # not empty
    refuse(lambda: c.fork([0, 0], [2, 2], ok=False))               # a destination twice
    refuse(lambda: c.fork([0, 3], [3, 2], ok=False))               # a source that is a destination
    refuse(lambda: c.fork([5], [2], ok=False))
    refuse(lambda: c.fork([0], [-2], ok=False))
    refuse(lambda: c.free([1, 1], ok=False))
    refuse(lambda: c.free([7], ok=False))
    c.reserve([2], [64])          # the last four pages
    refuse(lambda: c.fork([0], [3], ok=False))                     # no page for the copy
    c.fork([1], [3])              # a full last page needs none
    c.reserve([], [])
    c.fork([], [])
    c.free([])
    c.reserve([2, 4], [0, 0])
    c.fork([4], [4])              # an empty slot onto itself stays empty
    c.check()
    assert c.status() == M.MOT_ERR_PAGES   # that one is a source and a destination: refused as well


def test_reserve_refuses_starts_outside_its_rows():
    """starts below 0 or beyond the batch's rows, in the first entry, a middle one and the last."""
    c = P.Cache(n_pages=20, max_seqs=5, max_pages=4, page=16)
    c.reserve([0], [5])
    for starts, rows in (([0, 4, 9], 8), ([-1, 2, 3], 8), ([0, 9, 9], 8), ([9, 9, 12], 8), ([3, 5, 4], 8)):
        M.mot_paged_reserve(c.h, c.c, M.paged_batch(i32([1, 2]), i32(starts), 2, rows))
        c.check(f"{starts}")
        assert c.status() == M.MOT_ERR_PAGES, starts
    c.reserve([1, 2], [4, 4])
    c.check()
    assert c.status() == M.MOT_OK


def test_compaction_of_very_wide_pages():
    """A page of one layer has 2^31 bytes."""
    H = 32768
    c = P.Cache(q_heads=H, kv_heads=H, d=128, page=128, n_pages=2, max_seqs=2, max_pages=1, dtype="fp32")
    c.reserve([0, 1], [128, 100])
    c.free([0])
    before = [x[0, 1].clone() for x in (c.k, c.v)]
    c.compact()
    c.check()
    assert c.t[1] == [0]
    for x, y in zip((c.k, c.v), before):
        assert torch.equal(x[0, 0], y)
    assert c.status() == M.MOT_OK


def test_store_and_append_do_nothing_behind_a_refused_change():
    c = P.Cache(n_pages=4, max_pages=4, page=16)
    c.reserve([0], [20])
    before = [x.clone() for x in (c.k, c.v)]
    c.reserve([1], [64], ok=False)
    flat = [c.normal(1, 1, c.H, 32, c.d) for _ in range(2)]
    M.mot_paged_store(c.h, c.c, i32([0]), 1, *flat)
    x = c.normal(3, c.Hq + 2 * c.H, c.d)
    out = torch.zeros((3, c.Hq, c.d), dtype=torch.bfloat16, device="cuda")
    M.mot_paged_append(c.h, 0, c.c, c.batch([0], [3]), x[:, :c.Hq], x[:, c.Hq:c.Hq + c.H], x[:, c.Hq + c.H:], out)
    assert c.status() == M.MOT_ERR_PAGES
    assert torch.equal(before[0], c.k) and torch.equal(before[1], c.v)
    M.mot_paged_store(c.h, c.c, i32([0]), 1, *flat)
    assert c.status() == M.MOT_OK
    assert torch.equal(c.rows(0)[0], flat[0][0, 0, :, :20].double())


def test_store_and_load_of_some_layers():
    c = P.Cache(layers=5, page=32, n_pages=11)
    c.reserve([4, 1], [33, 64])
    flat = [c.normal(2, 3, c.H, 64, c.d) for _ in range(2)]
    before = [x.clone() for x in (c.k, c.v)]
    M.mot_paged_store(c.h, c.c, i32([4, 1]), 2, *flat, first_layer=2)
    torch.cuda.synchronize()
    for x, y, f in zip(before, (c.k, c.v), flat):
        for i, s in enumerate((4, 1)):
            for j, p in enumerate(c.t[s]):
                m = min(32, c.n[s] - 32 * j)
                x[2:4, p, :, :m] = f[:, i, :, 32 * j:32 * j + m]
        assert torch.equal(x, y)
    # a contiguous cache that is shorter than a sequence takes what it holds, and says so
    short = [torch.zeros((2, 1, c.H, 40, c.d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    M.mot_paged_load(c.h, c.c, i32([1]), 1, *short, first_layer=2)
    assert c.status() == M.MOT_ERR_PAGES
    assert torch.equal(short[0][:, 0], flat[0][:, 1, :, :40])


def test_many_pages_and_slots():
    """Bookkeeping over several pieces of a scan: 20,000 pages, 3,000 slots."""
    n, seqs = 20000, 3000
    c = P.Cache(n_pages=n, max_seqs=seqs, max_pages=8, page=16, kv_heads=1, q_heads=1)
    rng = np.random.default_rng(3)
    new = [int(x) for x in rng.integers(0, 100, size=seqs)]
    order = [int(x) for x in rng.permutation(seqs)]
    c.reserve(order, new)
    c.check()
    gone = [int(x) for x in rng.permutation(seqs)[:1500]]
    c.free(gone)
    c.check()
    live = [s for s in range(seqs) if c.n[s]]
    empty = [s for s in range(seqs) if not c.n[s]]
    c.fork([int(rng.choice(live)) for _ in empty[:1200]], empty[:1200])
    c.check()
    c.free(live[:700])
    c.compact()
    c.check()
    assert c.status() == M.MOT_OK


# ---------------------------------------------------------------- append

def _turned(x, pos, rot, pairs, base):
    """x [rows][heads][d] in 64 bits, rotated by its positions."""
    y = x.clone()
    if not rot:
        return y
    t = pos.double()[:, None, None] * base ** (-2 * torch.arange(rot // 2, device=x.device, dtype=torch.float64) / rot)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * t.cos() - b * t.sin(), b * t.cos() + a * t.sin()
    if pairs:
        y[..., 0:rot:2], y[..., 1:rot:2] = u, v
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = u, v
    return y


APPEND = [
    # dtype, q heads, kv heads, d, page, rot, pairs, norm
    ("bf16", 12, 2, 128, 16, 128, False, False),
    ("bf16", 5, 5, 64, 32, 64, True, True),
    ("bf16", 14, 2, 64, 64, 32, False, True),
    ("bf16", 16, 1, 128, 128, 0, False, True),
    ("bf16", 3, 1, 128, 16, 48, True, False),
    ("bf16", 12, 12, 64, 16, 0, False, False),
    ("fp32", 4, 2, 128, 16, 128, True, True),
    ("fp32", 7, 1, 64, 32, 16, False, True),
    ("fp32", 12, 2, 128, 64, 64, False, False),
]


@pytest.mark.parametrize("dtype,hq,h,d,page,rot,pairs,norm", APPEND)
def test_append_matches_the_formula(dtype, hq, h, d, page, rot, pairs, norm):
    base, eps = 1e6, 1e-5
    c = P.Cache(layers=2, q_heads=hq, kv_heads=h, d=d, page=page, n_pages=60, max_pages=20, dtype=dtype,
                rot_dim=rot, rot_pairs=pairs, rot_base=base, norm_eps=eps)
    c.reserve([3, 0, 5, 2], [page + 3, 2, 19, 1])
    new = [5, 2, 0, 1]
    seqs = [3, 0, 5, 2]
    rows = sum(new)
    # the columns of a fused projection, with rows that belong to no entry at either end
    x = c.normal(rows + 3, hq + 2 * h, d) * 3
    w = [(1 + 0.2 * c.normal(d)).to(P.DT[dtype]) for _ in range(2)] if norm else [None, None]
    starts = [1 + sum(new[:i]) for i in range(5)]
    b = M.paged_batch(i32(seqs), i32(starts), 4, rows + 3, 5)
    out = torch.full((rows + 3, hq, d), 9.0, dtype=P.DT[dtype], device="cuda")
    before = [t.clone() for t in (c.k, c.v)]
    M.mot_paged_append(c.h, 1, c.c, b, x[:, :hq], x[:, hq:hq + h], x[:, hq + h:], out, *w)
    assert c.status() == M.MOT_OK
    pos = torch.cat([torch.arange(c.n[s] - m, c.n[s]) for s, m in zip(seqs, new)]).cuda()
    y = x[1:1 + rows].double()
    half = P.HALF[dtype]

    def expect(z, weight):
        if weight is not None:
            z = z * (z.square().mean(2, keepdim=True) + eps).rsqrt() * weight.double()
        # fp32 on the way: 2^-20 of the pair's size covers the norm's sum of d squares ((d + 8) / 2 roundings
        # of 2^-24), the angle (2^-23 of a half turn), and the products
        return _turned(z, pos, rot, pairs, base), 2.0 ** -20 * z.abs().amax(2, keepdim=True)

    want, slop = expect(y[:, :hq], w[0])
    if not (norm or rot):
        half, slop = 0, 0 * slop
    P.assert_close(out[1:1 + rows], want, half * want.abs() + slop, "q")
    assert bool((out[0] == 9).all()) and bool((out[1 + rows:] == 9).all())
    wk, slop = expect(y[:, hq:hq + h], w[1])
    at = 0
    for s, m in zip(seqs, new):
        for j in range(c.n[s] - m, c.n[s]):
            p, r = c.t[s][j // page], j % page
            P.assert_close(c.k[1, p, :, r], wk[at], half * wk[at].abs() + slop[at] * (1 if half else 0), "k")
            assert torch.equal(c.v[1, p, :, r], x[1 + at, hq + h:])
            before[0][1, p, :, r], before[1][1, p, :, r] = c.k[1, p, :, r], c.v[1, p, :, r]
            at += 1
    for a, e in zip(before, (c.k, c.v)):   # nothing else of the pools changes
        assert torch.equal(a, e)


@pytest.mark.parametrize("pos", [1, 4095, 131071, 1000003])
def test_append_angles_at_far_positions(pos):
    """The rotation by a position far out, to 32-bit accuracy: cos and sin of pos * base^(-2 i / rot)."""
    page = 128
    c = P.Cache(q_heads=1, kv_heads=1, d=128, page=page, n_pages=2, max_seqs=1, max_pages=8192, dtype="fp32",
                rot_dim=128, rot_base=1e4)
    c.lens[0] = pos + 1
    c.table[0, pos // page] = 1
    x = torch.zeros((1, 3, 128), device="cuda")
    x[..., :64] = 1.0   # pairs (1, 0) become (cos, sin)
    out = torch.zeros((1, 1, 128), device="cuda")
    M.mot_paged_append(c.h, 0, c.c, M.paged_batch(i32([0]), i32([0, 1]), 1, 1), x[:, :1], x[:, 1:2], x[:, 2:], out)
    assert c.status() == M.MOT_OK
    t = pos * 1e4 ** (-2 * torch.arange(64, dtype=torch.float64) / 128)
    want = torch.cat([t.cos(), t.sin()])
    # the angle is rounded to 2^-24 of at most pi, cos and sin to two steps of 2^-23 more
    assert float((out[0, 0].double().cpu() - want).abs().max()) <= math.pi * 2.0 ** -24 + 2.0 ** -22
    assert torch.equal(c.k[0, 1, 0, pos % page], out[0, 0])


def test_append_in_place_and_many_rows():
    """q_out may be q; more rows than one pass of the grid; many entries, some without rows."""
    n = 700
    c = P.Cache(q_heads=2, kv_heads=1, d=64, page=16, n_pages=n, max_seqs=n, max_pages=2, rot_dim=64)
    new = [(i * 7) % 15 for i in range(n)]
    c.reserve(list(range(n)), new)
    rows = sum(new)
    q, k, v = c.normal(rows, 2, 64), c.normal(rows, 1, 64), c.normal(rows, 1, 64)
    keep = q.clone()
    M.mot_paged_append(c.h, 0, c.c, c.batch(list(range(n)), new), q, k, v, q)
    assert c.status() == M.MOT_OK
    pos = torch.cat([torch.arange(m) for m in new]).cuda()
    want = _turned(keep.double(), pos, 64, False, 1e4)
    P.assert_close(q, want, 2.0 ** -8 * want.abs() + 2.0 ** -20 * keep.double().abs().amax(2, keepdim=True))
    at = 0
    for s in range(0, n, 41):
        at = sum(new[:s])
        assert torch.equal(c.v[0, c.t[s][0], :, :new[s]].transpose(0, 1), v[at:at + new[s]]) if new[s] else True


# ---------------------------------------------------------------- attention

def _filled(lens, new, **kw):
    """A cache whose slots 0 .. hold sequences of these lengths, in pages without order."""
    kw.setdefault("page", 16)
    need = sum(-(-n // kw["page"]) for n in lens)
    c = P.Cache(n_pages=need + 5, max_seqs=len(lens) + 1, max_pages=max(2, max(-(-n // kw["page"]) for n in lens)), **kw)
    order = np.random.default_rng(len(lens)).permutation(need + 5).tolist()
    for s, n in enumerate(lens):
        c.n[s] = n
        c.t[s] = [order.pop() for _ in range(-(-n // c.P))]
        for p in c.t[s]:
            c.r[p] = 1
        if n:
            c.table[s, :len(c.t[s])] = i32(c.t[s])
    c.lens.copy_(i32(c.n))
    c.refs.copy_(i32(c.r))
    return c


def _attend(c, seqs, new, q=None, layer=0, spare=2):
    """The call with `spare` rows of no entry behind; checked against the formula. Returns q, out."""
    rows = sum(new)
    if q is None:
        q = c.normal(rows + spare, c.Hq, c.d)
    out = torch.full_like(q, 9.0)
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    b = M.paged_batch(i32(seqs), i32(starts), len(seqs), rows + spare, max(new, default=0))
    M.mot_paged_attention(c.h, layer, c.c, b, q, out)
    assert c.status() == M.MOT_OK
    P.check_attention(c, seqs, new, q, out, layer)
    assert bool((out[rows:] == 9).all())
    return q, out


TYPES = ["bf16", "fp32"]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,h,d,page", [(4, 2, 64, 16), (12, 2, 128, 64), (14, 2, 64, 32), (7, 1, 128, 128), (16, 1, 64, 16),
                                         (3, 3, 128, 32), (11, 1, 128, 16)])
def test_attention_of_single_rows(dtype, hq, h, d, page):
    lens = [1, 2, page - 1, page, page + 1, 200, 513]
    c = _filled(lens, None, q_heads=hq, kv_heads=h, d=d, page=page, dtype=dtype, seed=hq)
    _attend(c, list(range(7)), [1] * 7)
    _attend(c, [5], [1], spare=0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,h,d,page", [(4, 2, 64, 16), (12, 2, 128, 64), (14, 2, 64, 128), (7, 1, 128, 32), (16, 1, 128, 16), (3, 3, 64, 32)])
def test_attention_of_chunks(dtype, hq, h, d, page):
    """Prompts as long as their sequences and on top of a context, single rows and none among them."""
    lens = [1, 64, 65, 300, 129, 40, 260]
    new = [1, 64, 2, 131, 129, 0, 1]
    c = _filled(lens, new, q_heads=hq, kv_heads=h, d=d, page=page, dtype=dtype, seed=hq + d)
    _attend(c, [2, 0, 1, 6, 3, 5, 4], [new[s] for s in (2, 0, 1, 6, 3, 5, 4)])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [1, 2, 3, 5, 8, 9, 16, 17, 33])
def test_attention_of_every_small_chunk(dtype, new):
    """Row counts around the sizes of the row tiles: 3 heads of a group make 3 to 99 rows."""
    c = _filled([new, 150, 97 + new], None, q_heads=6, kv_heads=2, d=64, dtype=dtype, seed=new)
    _attend(c, [0, 1, 2], [new, new, 1])


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_a_long_context(dtype):
    """One row over 20,011 positions: many CTAs share each head's keys. Twice: the same bits."""
    c = _filled([20011], None, q_heads=6, kv_heads=2, d=128, page=32, dtype=dtype)
    q, out = _attend(c, [0], [1])
    again = torch.zeros_like(out)
    M.mot_paged_attention(c.h, 0, c.c, M.paged_batch(i32([0]), i32([0, 1]), 1, 1), q, again)
    assert torch.equal(again[:1], out[:1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new,n", [(1, 3000), (1, 9001), (20, 3000), (20, 20011), (70, 8200)])
def test_attention_of_few_rows_in_many_pieces(dtype, new, n):
    """Items that up to eight, up to 64 and more CTAs share: joins in one level and in two."""
    c = _filled([n, 40], None, q_heads=4, kv_heads=2, d=64, page=128, dtype=dtype, seed=n)
    q, out = _attend(c, [0, 1], [new, 1])
    again = torch.zeros_like(out)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0, 1], [new, 1]), q, again)
    assert torch.equal(again[:new + 1], out[:new + 1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [33, 500])
def test_attention_of_many_chunks(dtype, n):
    """More entries than a warp has lanes, and than a CTA has threads, with chunks of several sizes."""
    lens = [(i * 53) % 150 for i in range(n)]
    new = [min(x, (i * 11) % 31) for i, x in enumerate(lens)]
    c = _filled(lens, None, q_heads=4, kv_heads=2, d=64, dtype=dtype, seed=n)
    seqs = np.random.default_rng(n).permutation(n).tolist()
    _attend(c, seqs, [new[s] for s in seqs])


@pytest.mark.parametrize("dtype", TYPES)
def test_max_chunk_is_only_a_hint(dtype):
    """Entries with more rows than max_chunk says are computed all the same."""
    c = _filled([300, 90, 64], None, q_heads=6, kv_heads=2, d=128, page=32, dtype=dtype)
    q = c.normal(150 + 3 + 64, 6, 128)
    for hint in (0, 1, 10 ** 6):
        out = torch.full_like(q, 9.0)
        b = M.paged_batch(i32([0, 1, 2]), i32([0, 150, 153, 217]), 3, 217, hint)
        M.mot_paged_attention(c.h, 0, c.c, b, q, out)
        assert c.status() == M.MOT_OK
        P.check_attention(c, [0, 1, 2], [150, 3, 64], q, out)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_a_long_chunk(dtype):
    """A chunk of 700 on 1,600 positions, checked at some rows; every layer of the pool is its own."""
    c = _filled([2300], None, layers=3, q_heads=4, kv_heads=2, d=64, page=64, dtype=dtype)
    q = c.normal(700, 4, 64)
    for layer in (0, 2):
        out = torch.empty_like(q)
        M.mot_paged_attention(c.h, layer, c.c, c.batch([0], [700]), q, out)
        assert c.status() == M.MOT_OK
        K, V = c.rows(0, layer)
        for r in (0, 1, 63, 64, 127, 128, 350, 698, 699):
            n = 1600 + r + 1
            ref, absv, slop = P.attention(q[r:r + 1], K[:, :n], V[:, :n])
            half = P.HALF[dtype]
            P.assert_close(out[r:r + 1], ref, half * (ref.abs() + (absv if dtype == "bf16" else 0)) + slop, f"row {r}")


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_many_entries(dtype):
    """More entries than a CTA has threads, many without rows."""
    n = 900
    lens = [(i * 37) % 50 for i in range(n)]
    c = _filled(lens, None, q_heads=2, kv_heads=1, d=64, dtype=dtype)
    new = [1 if x and i % 3 else 0 for i, x in enumerate(lens)]
    _attend(c, list(range(n)), new)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_before_position_zero_are_zeros(dtype):
    """More rows than positions: the rows without any key are written as zeros."""
    c = _filled([3, 0, 20], None, q_heads=4, kv_heads=2, d=64, dtype=dtype)
    q = c.normal(5 + 2 + 30, 4, 64)
    out = torch.full_like(q, 9.0)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0, 1, 2], [5, 2, 30]), q, out)
    assert c.status() == M.MOT_OK
    P.check_attention(c, [0, 1, 2], [5, 2, 30], q, out)
    assert not bool(out[:2].any()) and not bool(out[5:7].any()) and not bool(out[7:17].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("new", [1, 4, 40, 150])
def test_masked_positions_add_nothing_whatever_they_hold(dtype, poison, new):
    """Free pages, positions behind the end and keys behind a row's position are NaN or infinite."""
    c = _filled([70 + new, 33], None, q_heads=6, kv_heads=2, d=64, page=32, dtype=dtype)
    q = c.normal(new + 1, 6, 64)
    b = c.batch([0, 1], [new, 1])
    held = torch.zeros((c.n_pages, c.P), dtype=torch.bool, device="cuda")
    for s in (0, 1):
        for j in range(c.n[s]):
            held[c.t[s][j // c.P], j % c.P] = True
    for x in (c.k, c.v):
        x[0] = torch.where(held[:, None, :, None], x[0], poison)
    out = torch.zeros_like(q)
    M.mot_paged_attention(c.h, 0, c.c, b, q, out)
    P.check_attention(c, [0, 1], [new, 1], q, out)
    # and the last position itself: only its own row sees it
    last = c.n[0] - 1
    for x in (c.k, c.v):
        x[0, c.t[0][last // c.P], :, last % c.P] = poison
    M.mot_paged_attention(c.h, 0, c.c, b, q, out)
    n = c.n[0]
    K, V = c.rows(0)
    ref, absv, slop = P.attention(q[:new], K[:, :n].nan_to_num(0, 0, 0), V[:, :n].nan_to_num(0, 0, 0))
    half = P.HALF[dtype]
    tol = half * (ref.abs() + (absv if dtype == "bf16" else 0)) + slop
    P.assert_close(out[:new - 1], ref[:new - 1], tol[:new - 1], "rows before the poisoned one")
    assert not bool(torch.isfinite(out[new - 1]).all())
    P.check_attention(c, [1], [1], q[new:], out[new:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [1, 60])
def test_an_infinite_value_that_is_seen(dtype, new):
    """An infinite value with weight gives an infinite result in its column, and only there."""
    c = _filled([300], None, q_heads=4, kv_heads=2, d=64, dtype=dtype)
    c.v[0, c.t[0][2], 1, 5, 7] = math.inf
    q = c.normal(new, 4, 64)
    out = torch.zeros_like(q)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0], [new]), q, out)
    inf = torch.isinf(out)
    assert bool(inf[:, 2:, 7].all()) and int(inf.sum()) == 2 * new and not bool(torch.isnan(out).any())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 2, 3])
def test_infinite_values_that_are_seen_by_few_rows(d, new):
    """The same at many positions: whatever a weight's two bf16 parts are (the second one may be 0 or
    negative), they give the infinity and no NaN; a NaN and both infinities in a column give NaN."""
    c = _filled([600], None, q_heads=8, kv_heads=2, d=d, page=32)
    q = c.normal(new, 8, d)
    b, clean = c.batch([0], [new]), c.v.clone()
    out = torch.zeros_like(q)
    for j in range(0, 600 - new, 13):
        sign = -1 if j % 2 else 1
        c.v.copy_(clean)
        page, at = c.t[0][j // 32], j % 32
        c.v[0, page, 0, at, 9] = sign * math.inf
        c.v[0, page, 1, at, 3] = math.nan
        c.v[0, page, 1, at, 40] = math.inf
        c.v[0, c.t[0][0], 1, 31, 40] = -math.inf
        M.mot_paged_attention(c.h, 0, c.c, b, q, out)
        odd = torch.zeros_like(out, dtype=torch.bool)
        odd[:, :4, 9] = True
        odd[:, 4:, 3] = odd[:, 4:, 40] = True
        assert bool((out[:, :4, 9] == sign * math.inf).all()), j
        assert bool(torch.isnan(out[:, 4:, 3]).all()) and bool(torch.isnan(out[:, 4:, 40]).all()), j
        assert bool(torch.isfinite(out[~odd]).all()), j


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [1, 40])
def test_rows_whose_scores_are_all_minus_infinity_are_zeros(dtype, new):
    c = _filled([90], None, q_heads=4, kv_heads=2, d=64, dtype=dtype)
    c.k[0, c.t[0], 1] = -math.inf   # the second key/value head's keys, all positions
    q = c.normal(new, 4, 64).abs() + 0.5
    out = torch.full_like(q, math.nan)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0], [new]), q, out)
    assert not bool(out[:, 2:].any()) and bool(torch.isfinite(out).all())
    K, V = c.rows(0)
    ref, absv, slop = P.attention(q[:, :2], K[:1], V[:1])
    half = P.HALF[dtype]
    P.assert_close(out[:, :2], ref, half * (ref.abs() + (absv if dtype == "bf16" else 0)) + slop, "the other head")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gain", [0.05, 2.0, -2.0])
@pytest.mark.parametrize("new", [1, 50])
def test_scores_that_rise_or_fall_along_the_context(dtype, gain, new):
    """Scores that grow by `gain` (base 2) from key to key: the running maximum moves all the time."""
    c = _filled([777], None, q_heads=4, kv_heads=2, d=128, page=64, dtype=dtype)
    j = torch.arange(777, device="cuda", dtype=torch.float64)
    for s in (0,):
        for p0, page in enumerate(c.t[0]):
            pos = p0 * 64 + torch.arange(64, device="cuda", dtype=torch.float64)
            c.k[0, page] = (0.25 * c.k[0, page].double() + gain * (pos % 1024)[None, :, None] / 16).to(c.k.dtype)
    q = (0.25 * c.normal(new, 4, 128).float() + 1).to(P.DT[dtype])
    _attend(c, [0], [new], q=q, spare=0)


@pytest.mark.parametrize("dtype", TYPES)
def test_lowest_values_in_the_cache(dtype):
    """Keys of the type's lowest value: their scores are -inf or huge, their weight 0 or 1, never NaN
    beside others."""
    c = _filled([100], None, q_heads=2, kv_heads=1, d=64, dtype=dtype)
    low = torch.finfo(P.DT[dtype]).min
    for j in (3, 50, 98):
        c.k[0, c.t[0][j // 16], 0, j % 16] = low
    q = c.normal(40, 2, 64).abs() + 0.5   # every score of those keys is -inf
    out = torch.zeros_like(q)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0], [40]), q, out)
    K, V = c.rows(0)
    keep = [j for j in range(100) if j not in (3, 50, 98)]
    for r in (0, 10, 39):
        rows = [j for j in keep if j <= 60 + r]
        ref, absv, slop = P.attention(q[r:r + 1], K[:, rows], V[:, rows])
        half = P.HALF[dtype]
        P.assert_close(out[r:r + 1], ref, half * (ref.abs() + (absv if dtype == "bf16" else 0)) + slop, f"row {r}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [1, 30])
def test_table_entries_out_of_range_are_reported(dtype, new):
    """They are held inside the pool: the call ends, the others' rows are right, the status tells."""
    c = _filled([200, 90], None, q_heads=4, kv_heads=2, d=64, dtype=dtype)
    c.table[0, 3] = c.n_pages
    c.table[0, 5] = -7
    q = c.normal(new + 1, 4, 64)
    out = torch.zeros_like(q)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0, 1], [new, 1]), q, out)
    assert c.status() == M.MOT_ERR_PAGES
    P.check_attention(c, [1], [1], q[new:], out[new:])
    # slots, lengths and starts out of their ranges
    for seqs, starts in (([99, 1], [0, new, new + 1]), ([-3, 1], [0, new, new + 1]), ([0, 1], [0, 1 << 30, new + 1])):
        M.mot_paged_attention(c.h, 0, c.c, M.paged_batch(i32(seqs), i32(starts), 2, new + 1, new), q, out)
        assert c.status() == M.MOT_ERR_PAGES
    c.lens[0] = 1 << 29
    M.mot_paged_attention(c.h, 0, c.c, c.batch([1], [1]), q, out)
    assert c.status() == M.MOT_OK


@pytest.mark.parametrize("new", [1, 200])
def test_offsets_beyond_32_bits(new):
    """A pool of 9 GB a side, its sequence in the last pages: element offsets pass 2^32."""
    page, H, d = 128, 4, 128
    n_pages = (1 << 32) // (page * H * d) + 600
    c = P.Cache.__new__(P.Cache)
    c.L, c.Hq, c.H, c.d, c.P, c.n_pages, c.max_seqs, c.max_pages, c.dtype = 1, 8, H, d, page, n_pages, 1, 8, "bf16"
    c.gen = torch.Generator(device="cuda").manual_seed(5)
    c.k, c.v = (torch.empty((1, n_pages, H, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.t, c.n = [[n_pages - 1 - 90 * i for i in range(6)]], [700]
    for x in (c.k, c.v):
        x[0, c.t[0]] = c.normal(6, H, page, d)
    c.table = torch.full((1, 8), -1, dtype=torch.int32, device="cuda")
    c.table[0, :6] = i32(c.t[0])
    c.lens, c.refs = i32([700]), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    c.c = M.paged_cache(c.k, c.v, c.table, c.lens, c.refs)
    c.h = M.mot_create_paged(M.make_paged_config(1, 8, H, d, page, n_pages, 1, 8))
    _attend(c, [0], [new])
    # the append, the copies and a compaction reach there too
    x = c.normal(new, 8 + 2 * H, d)
    q = torch.zeros((new, 8, d), dtype=torch.bfloat16, device="cuda")
    M.mot_paged_append(c.h, 0, c.c, c.batch([0], [new]), x[:, :8], x[:, 8:8 + H], x[:, 8 + H:], q)
    flat = [torch.zeros((1, 1, H, 700, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    M.mot_paged_load(c.h, c.c, i32([0]), 1, *flat)
    assert c.status() == M.MOT_OK
    for f, stored, k in zip(flat, c.rows(0), (x[:, 8:8 + H], x[:, 8 + H:])):
        assert torch.equal(f[0, 0, :, 700 - new:].transpose(0, 1), k)
        assert torch.equal(f[0, 0].double(), stored)
    M.mot_paged_store(c.h, c.c, i32([0]), 1, flat[1], flat[0])
    c.refs[c.t[0]] = 1
    M.mot_paged_compact(c.h, c.c)
    assert c.status() == M.MOT_OK
    c.t[0] = c.table[0, :6].tolist()
    assert sorted(c.t[0]) == list(range(6))
    for f, stored in zip((flat[1], flat[0]), c.rows(0)):
        assert torch.equal(f[0, 0].double(), stored)


def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right():
    """The first CTA loads nothing (test hook) under a limit of about 10 ms: the call ends with
    MOT_ERR_TIMEOUT. Its split items' arrivals are settled, so the next call joins them rightly."""
    c = _filled([3000, 900], None, q_heads=8, kv_heads=2, d=128, page=32)
    q = c.normal(200, 8, 128)
    out = torch.zeros_like(q)
    b = c.batch([0, 1], [120, 80])
    for _ in range(2):
        M.mot_debug_set(c.h, True, 20_000_000)
        M.mot_paged_attention(c.h, 0, c.c, b, q, out)
        assert c.status() == M.MOT_ERR_TIMEOUT
        M.mot_debug_set(c.h, False)
        M.mot_paged_attention(c.h, 0, c.c, b, q, out)
        assert c.status() == M.MOT_OK
        P.check_attention(c, [0, 1], [120, 80], q, out)


# ---------------------------------------------------------------- streams, graphs, the whole run

def test_a_step_is_captured_and_replayed_on_another_stream():
    """Reserve, append and attention of one decoding step in a graph: each replay is the next step."""
    c = P.Cache(layers=1, q_heads=6, kv_heads=2, d=64, page=16, n_pages=30, max_pages=12, rot_dim=64)
    c.reserve([0, 1], [60, 17])
    x = torch.zeros((2, 10, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((2, 6, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    b = c.batch([0, 1], [1, 1])

    def step():
        M.mot_paged_reserve(c.h, c.c, b)
        M.mot_paged_append(c.h, 0, c.c, b, x[:, :6], x[:, 6:8], x[:, 8:], q)
        M.mot_paged_attention(c.h, 0, c.c, b, q, out)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(20):
        x.copy_(c.normal(2, 10, 64))
        graph.replay()
        torch.cuda.synchronize()
        for s in (0, 1):
            c.t[s] += c.take(c.pages(c.n[s] + 1) - c.pages(c.n[s]))
            c.n[s] += 1
        c.check()
        P.check_attention(c, [0, 1], [1, 1], q, out)
    assert c.status() == M.MOT_OK


def test_forks_compaction_and_chunks_are_captured_and_replayed():
    """A turn of an agents' loop in a graph: branches end, the pool is compacted, new branches start and
    take a prompt. Every replay is another turn."""
    c = P.Cache(layers=2, q_heads=6, kv_heads=2, d=64, page=16, n_pages=40, max_pages=12, rot_dim=64)
    c.reserve([0, 1], [70, 33])
    c.fork([0, 1, 0], [2, 3, 4])
    rows, new = 60, [40, 15, 5]
    x = c.normal(rows, 10, 64)
    q, out = (torch.zeros((rows, 6, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dst, src, b = i32([2, 3, 4]), i32([0, 1, 0]), c.batch([2, 3, 4], new)

    def turn():
        M.mot_paged_free(c.h, c.c, dst, 3)
        M.mot_paged_compact(c.h, c.c)
        M.mot_paged_fork(c.h, c.c, src, dst, 3)
        M.mot_paged_reserve(c.h, c.c, b)
        M.mot_paged_append(c.h, 1, c.c, b, x[:, :6], x[:, 6:8], x[:, 8:], q)
        M.mot_paged_attention(c.h, 1, c.c, b, q, out)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        turn()
    for _ in range(4):
        x.copy_(c.normal(rows, 10, 64))
        graph.replay()
        torch.cuda.synchronize()
        for s in (2, 3, 4):   # the same on the lists
            for p in c.t[s]:
                c.r[p] -= 1
            c.t[s], c.n[s] = [], 0
        used = sum(r > 0 for r in c.r)
        to = dict(zip([p for p in range(used, c.n_pages) if c.r[p]], [p for p in range(used) if not c.r[p]]))
        for a, e in to.items():
            c.r[e], c.r[a] = c.r[a], 0
        c.t = [[to.get(p, p) for p in row] for row in c.t]
        for s, e in ((0, 2), (1, 3), (0, 4)):
            full, part = divmod(c.n[s], 16)
            c.t[e], c.n[e] = c.t[s][:full], c.n[s]
            for p in c.t[e]:
                c.r[p] += 1
            if part:
                c.t[e] = c.t[e] + c.take(1)
        for s, m in zip((2, 3, 4), new):
            c.t[s] = c.t[s] + c.take(c.pages(c.n[s] + m) - c.pages(c.n[s]))
            c.n[s] += m
        c.check()
        P.check_attention(c, [2, 3, 4], new, q, out, 1)
    assert c.status() == M.MOT_OK


def test_two_handles_at_once():
    """Two handles have workspaces of their own: their calls may run side by side on two streams."""
    caches = [_filled([6000, 500], None, q_heads=4, kv_heads=2, d=64, page=64, seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in caches]
    qs = [c.normal(33, 4, 64) for c in caches]
    outs = [torch.zeros_like(q) for q in qs]
    batches = [(c.batch([0, 1], [32, 1]), c.batch([0, 1], [1, 1])) for c in caches]
    torch.cuda.synchronize()
    for _ in range(30):
        for c, st, q, o, (chunk, step) in zip(caches, streams, qs, outs, batches):
            M.mot_paged_attention(c.h, 0, c.c, chunk, q, o, stream=st)
            M.mot_paged_attention(c.h, 0, c.c, step, q[31:], o[31:], stream=st)
            M.mot_paged_attention(c.h, 0, c.c, chunk, q, o, stream=st)
    torch.cuda.synchronize()
    for c, q, o in zip(caches, qs, outs):
        assert c.status() == M.MOT_OK
        P.check_attention(c, [0, 1], [32, 1], q, o)


def test_calls_follow_the_given_stream():
    c = _filled([500], None, q_heads=4, kv_heads=2, d=64)
    q = c.normal(1, 4, 64)
    out = torch.zeros_like(q)
    side, b = torch.cuda.Stream(), c.batch([0], [1])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        big = torch.randn((4096, 4096), device="cuda")
        for _ in range(20):
            big = big @ big / 4096
        q.mul_(2)   # behind the products: the call has to wait for it
    M.mot_paged_attention(c.h, 0, c.c, b, q, out, stream=side)
    assert M.mot_get_device_status(c.h, side) == M.MOT_OK
    P.check_attention(c, [0], [1], q, out)


def test_from_translation_to_many_branches():
    """The whole run: a context is translated, stored into pages and forked; the branches take prompts
    and decode; one ends, the pool is compacted, and the others go on; a branch is loaded back."""
    import synth
    wl = synth.Workload("paged_run", 3, 2, 64, 4, 2, 128, 2, 256, 2, 150, "bf16", (150, 83), layer_map=(0, 1, 2, 2))
    run = P.G.Run(wl, synth.gen_cache(wl, 0), synth.gen_cache(wl, 1), synth.gen_weights(wl))
    assert run.translate() == M.MOT_OK
    L, Hq, H, d = 4, 12, 2, 128
    c = P.Cache(layers=L, q_heads=Hq, kv_heads=H, d=d, page=32, n_pages=30, max_seqs=8, max_pages=8, rot_dim=128, rot_base=1e6)
    c.reserve([0, 1], [150, 83])
    M.mot_paged_store(c.h, c.c, i32([0, 1]), 2, run.dk, run.dv)
    c.fork([0, 0, 1], [2, 3, 4])
    c.check()
    text = {s: [[run.dk[l, b, :, :n].clone(), run.dv[l, b, :, :n].clone()] for l in range(L)]
            for s, b, n in ((0, 0, 150), (1, 1, 83), (2, 0, 150), (3, 0, 150), (4, 1, 83))}

    def step(seqs, new):
        c.reserve(seqs, new)
        b = c.batch(seqs, new)
        rows = sum(new)
        for l in range(L):
            x = c.normal(rows, Hq + 2 * H, d)
            q = torch.empty((rows, Hq, d), dtype=torch.bfloat16, device="cuda")
            out = torch.empty_like(q)
            M.mot_paged_append(c.h, l, c.c, b, x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], q)
            M.mot_paged_attention(c.h, l, c.c, b, q, out)
            assert c.status() == M.MOT_OK
            at = 0
            for s, m in zip(seqs, new):
                pos = torch.arange(c.n[s] - m, c.n[s], device="cuda")
                k = _turned(x[at:at + m, Hq:Hq + H].double(), pos, 128, False, 1e6).to(torch.bfloat16)
                got = c.rows(s, l)[0][:, -m:]
                P.assert_close(got, k.double().transpose(0, 1), 2.0 ** -7 * k.double().transpose(0, 1).abs() + 2e-5, "keys")
                text[s][l][0] = torch.cat([text[s][l][0], got.to(torch.bfloat16)], 1)
                text[s][l][1] = torch.cat([text[s][l][1], x[at:at + m, Hq + H:].transpose(0, 1)], 1)
                for mine, stored in zip(text[s][l], c.rows(s, l)):
                    assert torch.equal(mine.double(), stored)
                at += m
            P.check_attention(c, seqs, new, q, out, l)

    step([0, 2, 3, 4], [20, 7, 1, 45])      # prompts of several lengths
    for _ in range(3):
        step([0, 1, 2, 3, 4], [1] * 5)      # decoding
    c.free([0, 4])
    c.compact()
    c.check()
    step([3, 1, 2], [2, 1, 40])
    flat = [torch.zeros((L, 1, H, 256, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    M.mot_paged_load(c.h, c.c, i32([2]), 1, *flat)
    torch.cuda.synchronize()
    for l in range(L):
        for x, y in zip(flat, text[2][l]):
            assert torch.equal(x[l, 0, :, :c.n[2]], y)
    assert c.status() == M.MOT_OK


# ---------------------------------------------------------------- refusals on the host

def _refused(call, status=M.MOT_ERR_INVALID_ARG):
    with pytest.raises(M.MotError) as e:
        call()
    assert e.value.status == status


def test_host_refusals():
    c = _filled([40], None, layers=2, q_heads=4, kv_heads=2, d=64)
    q = c.normal(2, 4, 64)
    out = torch.zeros_like(q)
    b = c.batch([0], [2])
    _refused(lambda: M.mot_paged_attention(c.h, 2, c.c, b, q, out))
    _refused(lambda: M.mot_paged_attention(c.h, -1, c.c, b, q, out))
    _refused(lambda: M.mot_paged_attention(c.h, 0, c.c, b, q, q))
    _refused(lambda: M.mot_paged_attention(c.h, 0, c.c, b, q, c.k))
    _refused(lambda: M.mot_paged_attention(c.h, 0, c.c, b, None, out))
    _refused(lambda: M.mot_paged_attention(c.h, 0, c.c, b, q.data_ptr() + 2, out))
    _refused(lambda: M.mot_paged_attention(c.h, 0, c.c, M.paged_batch(b._keep[0], b._keep[1], c.max_seqs + 1, 2), q, out))
    _refused(lambda: M.mot_paged_attention(c.h, 0, c.c, M.paged_batch(b._keep[0], b._keep[1], 1, -1), q, out))
    _refused(lambda: M.mot_paged_attention(c.h, 0, c.c, M.paged_batch(b._keep[0], b._keep[1], 1, (1 << 26) + 1), q, out))
    _refused(lambda: M.mot_paged_attention(c.h, 0, c.c, M.paged_batch(None, b._keep[1], 1, 2), q, out))
    _refused(lambda: M.mot_paged_attention(c.h, 0, M.paged_cache(c.k, c.k, c.table, c.lens, c.refs), b, q, out))
    _refused(lambda: M.mot_paged_attention(c.h, 0, M.paged_cache(c.k, c.v, None, c.lens, c.refs), b, q, out))
    k = c.normal(2, 2, 64)
    _refused(lambda: M.mot_paged_append(c.h, 2, c.c, b, q, k, k, out))
    _refused(lambda: M.mot_paged_append(c.h, 0, c.c, b, q, k, k, k))
    _refused(lambda: M.mot_paged_append(c.h, 0, c.c, b, q, k, k, c.v))
    wide = c.normal(2, 5, 64)
    _refused(lambda: M.mot_paged_append(c.h, 0, c.c, b, wide[:, :4], k, k, wide))   # in place, rows apart
    odd = torch.zeros(2, 4 * 64 + 4, dtype=torch.bfloat16, device="cuda")
    _refused(lambda: M.mot_paged_append(c.h, 0, c.c, b, odd[:, :256].view(2, 4, 64), k, k, out))   # 8-byte rows
    with pytest.raises(ValueError):
        M.mot_paged_append(c.h, 0, c.c, b, q.transpose(0, 1), k, k, out)
    flat = [c.normal(2, 1, 2, 64, 64) for _ in range(2)]
    _refused(lambda: M.mot_paged_store(c.h, c.c, i32([0]), 1, *flat, first_layer=1))
    _refused(lambda: M.mot_paged_store(c.h, c.c, i32([0, 1]), 2, *flat))   # more slots than the batch holds
    _refused(lambda: M.mot_paged_load(c.h, c.c, i32([0]), 1, flat[0], flat[0]))
    _refused(lambda: M.mot_paged_fork(c.h, c.c, None, i32([1]), 1))
    _refused(lambda: M.mot_paged_free(c.h, c.c, i32([1]), -1))
    _refused(lambda: M.mot_paged_compact(c.h, c.c, c.lens.data_ptr() + 1))
    # handles of other kinds, both ways
    import synth
    other = M.mot_create_replay(M.mot_replay_config(4, 2, 64, 1, 64, 16, 1))
    _refused(lambda: M.mot_paged_attention(other, 0, c.c, b, q, out))
    _refused(lambda: M.mot_replay_attention(c.h, 0, q, k, k, None, i32([1]), 1, out))
    _refused(lambda: M.mot_translate(c.h, q, k, i32([1]), 1, out, out))
    _refused(lambda: M.mot_load_weights(c.h, np.zeros(1, dtype=np.uint16)))
    assert c.status() == M.MOT_OK
