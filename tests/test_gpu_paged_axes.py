"""Appends whose rotation goes by several positions of a row, on the GPU through the C ABI, against the
formula in 64 bits."""
import decimal
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import _paged as P   # noqa: E402
M = P.M
i32 = P.i32


def turned(x, angle, pairs):
    """x [rows][heads][d] in 64 bits, its first 2 n dimensions rotated by angle [rows][n]."""
    y, rot = x.clone(), 2 * angle.shape[1]
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * c - b * s, b * c + a * s
    if pairs:
        y[..., 0:rot:2], y[..., 1:rot:2] = u, v
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = u, v
    return y


def layout(kind, n):
    """The axis of each of n pairs, and its rate where it is not the base's."""
    if kind == "turns":
        return 3, [i % 3 for i in range(n)], None
    if kind == "one":
        return 1, [0] * n, None
    if kind == "unused":   # the second of four axes turns nothing
        return 4, [(0, 2, 3)[i % 3] for i in range(n)], None
    cut = [n // 4, n // 4 + n * 3 // 8]
    axis = [sum(i >= c for c in cut) for i in range(n)]
    return 3, axis, None if kind == "sections" else [(-1) ** i * 0.7 ** (i / 3) for i in range(n)]


CASES = [
    # dtype, q heads, kv heads, d, page, rot, pairs, norm, layout
    ("bf16", 12, 2, 128, 16, 128, False, True, "sections"),
    ("bf16", 5, 5, 64, 32, 64, True, False, "turns"),
    ("bf16", 14, 2, 64, 64, 32, False, False, "own"),
    ("bf16", 3, 1, 128, 128, 48, True, True, "unused"),
    ("fp32", 4, 2, 128, 16, 128, True, False, "sections"),
    ("fp32", 7, 1, 64, 32, 16, False, True, "one"),
    ("fp32", 12, 12, 64, 64, 64, False, True, "own"),
]


@pytest.mark.parametrize("dtype,hq,h,d,page,rot,pairs,norm,kind", CASES)
def test_append_at_matches_the_formula(dtype, hq, h, d, page, rot, pairs, norm, kind):
    base, eps = 1e5, 1e-5
    c = P.Cache(layers=2, q_heads=hq, kv_heads=h, d=d, page=page, n_pages=60, max_pages=20, dtype=dtype,
                rot_dim=rot, rot_pairs=pairs, rot_base=base, norm_eps=eps)
    axes, axis, rates = layout(kind, rot // 2)
    M.mot_paged_set_axes(c.h, axes, axis, rates)
    seqs, new = [3, 0, 5, 2], [7, 2, 0, 1]
    c.reserve(seqs, [page + 7, 2, 19, 1])
    rows = sum(new)
    x = c.normal(rows + 3, hq + 2 * h, d) * 3   # rows that belong to no entry at either end
    w = [(1 + 0.2 * c.normal(d)).to(P.DT[dtype]) for _ in range(2)] if norm else [None, None]
    at = torch.randint(-2 ** 20, 2 ** 20, (axes, rows + 3), generator=c.gen, device="cuda", dtype=torch.int32)
    at[:, 1] = 0
    starts = [1 + sum(new[:i]) for i in range(5)]
    b = M.paged_batch(i32(seqs), i32(starts), 4, rows + 3, 7)
    out = torch.full((rows + 3, hq, d), 9.0, dtype=P.DT[dtype], device="cuda")
    before = [t.clone() for t in (c.k, c.v)]
    M.mot_paged_append_at(c.h, 1, c.c, b, at, x[:, :hq], x[:, hq:hq + h], x[:, hq + h:], out, *w)
    assert c.status() == M.MOT_OK
    rate = torch.tensor(rates or [base ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device="cuda")
    angle = at[torch.tensor(axis, device="cuda")].T[1:1 + rows].double() * rate   # off by 2^20 2^-53 at most
    y, half = x[1:1 + rows].double(), P.HALF[dtype]

    def expect(z, weight):
        if weight is not None:
            z = z * (z.square().mean(2, keepdim=True) + eps).rsqrt() * weight.double()
        # fp32 on the way, as for a single position: the norm's sum of d squares ((d + 8) / 2 roundings of 2^-24),
        # the angle (2^-23 of a half turn) and the products stay below 2^-20 of the largest value
        return turned(z, angle, pairs), 2.0 ** -20 * z.abs().amax(2, keepdim=True)

    want, slop = expect(y[:, :hq], w[0])
    P.assert_close(out[1:1 + rows], want, half * want.abs() + slop, "q")
    assert bool((out[0] == 9).all()) and bool((out[1 + rows:] == 9).all())
    wk, slop = expect(y[:, hq:hq + h], w[1])
    r = 0
    for s, m in zip(seqs, new):
        for j in range(c.n[s] - m, c.n[s]):
            p, o = c.t[s][j // page], j % page
            P.assert_close(c.k[1, p, :, o], wk[r], half * wk[r].abs() + slop[r], "k")
            assert torch.equal(c.v[1, p, :, o], x[1 + r, hq + h:])
            before[0][1, p, :, o], before[1][1, p, :, o] = c.k[1, p, :, o], c.v[1, p, :, o]
            r += 1
    for a, e in zip(before, (c.k, c.v)):   # nothing else of the pools changes
        assert torch.equal(a, e)


def test_the_places_in_the_sequence_give_what_append_gives():
    """All axes at the row's place: bit for bit mot_paged_append, which the axes leave as it was."""
    new = [33, 1, 5]
    x = None
    got = []
    for way in ("plain", "set", "at"):
        c = P.Cache(q_heads=6, kv_heads=2, d=128, page=16, rot_dim=128, rot_base=1e6)
        c.reserve([0, 1, 2], [40, 17, 5])
        if x is None:
            x = c.normal(39, 10, 128)
        if way != "plain":
            M.mot_paged_set_axes(c.h, 3, [i % 3 for i in range(64)])
        c.k.zero_()
        out = torch.zeros((39, 6, 128), dtype=torch.bfloat16, device="cuda")
        args = x[:, :6], x[:, 6:8], x[:, 8:], out
        if way == "at":
            pos = torch.cat([torch.arange(c.n[s] - m, c.n[s]) for s, m in enumerate(new)]).to(torch.int32).cuda()
            M.mot_paged_append_at(c.h, 0, c.c, c.batch([0, 1, 2], new), pos.expand(3, -1).contiguous(), *args)
        else:
            M.mot_paged_append(c.h, 0, c.c, c.batch([0, 1, 2], new), *args)
        assert c.status() == M.MOT_OK
        got.append((out, c.k.clone()))
    for a, b in got[1:]:
        assert torch.equal(a, got[0][0]) and torch.equal(b, got[0][1])


@pytest.mark.parametrize("pos", [-1, 1000003, 2 ** 31 - 1, -2 ** 31])
def test_angles_at_far_and_negative_positions(pos):
    """cos and sin of pos times a rate, to 32-bit accuracy at the ends of the positions' range; rates of many
    turns a position and negative ones."""
    c = P.Cache(q_heads=1, kv_heads=1, d=64, page=16, n_pages=2, dtype="fp32", rot_dim=64)
    c.reserve([0], [1])
    rates = [(-1) ** i * 65536.0 * 0.5 ** i * (1 + i / 77) for i in range(32)]
    rates[0] = 65536.0
    M.mot_paged_set_axes(c.h, 2, [i % 2 for i in range(32)], rates)
    x = torch.zeros((1, 3, 64), device="cuda")
    x[..., :32] = 1.0   # pairs (1, 0) become (cos, sin)
    out = torch.zeros((1, 1, 64), device="cuda")
    M.mot_paged_append_at(c.h, 0, c.c, c.batch([0], [1]), i32([[pos], [pos // 2]]), x[:, :1], x[:, 1:2], x[:, 2:], out)
    assert c.status() == M.MOT_OK
    with decimal.localcontext() as ctx:
        ctx.prec = 60
        two_pi = 2 * decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
        t = [float((decimal.Decimal(pos if i % 2 == 0 else pos // 2) * decimal.Decimal(r)) % two_pi) for i, r in enumerate(rates)]
    want = torch.tensor([math.cos(a) for a in t] + [math.sin(a) for a in t], dtype=torch.float64)
    # a rate is held to 2^-64 turns and a position is below 2^31: 2^-33 turns, the next 2^-32 are cut off; the angle
    # is rounded to 2^-24 of at most pi, cos and sin to two steps of 2^-23 more
    tol = 2 * math.pi * (2.0 ** -33 + 2.0 ** -32) + math.pi * 2.0 ** -24 + 2.0 ** -22
    assert float((out[0, 0].double().cpu() - want).abs().max()) <= tol


def test_rows_without_a_place_give_nothing():
    """Rows before position 0 and an entry outside the table: reported, nothing written."""
    c = P.Cache(q_heads=2, kv_heads=2, d=64, page=16, rot_dim=64)
    c.reserve([0], [3])
    M.mot_paged_set_axes(c.h, 2, [0, 1] * 16)
    x = c.normal(6, 6, 64)
    out = torch.full((6, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    before = [t.clone() for t in (c.k, c.v)]
    b = M.paged_batch(i32([0, 77]), i32([0, 5, 6]), 2, 6)   # the first two rows lie before position 0
    M.mot_paged_append_at(c.h, 0, c.c, b, torch.ones((2, 6), dtype=torch.int32, device="cuda"), x[:, :2], x[:, 2:4], x[:, 4:], out)
    assert c.status() == M.MOT_ERR_PAGES
    assert bool((out[:2] == 9).all()) and bool((out[5] == 9).all()) and not bool((out[2:5] == 9).any())
    page = c.t[0][0]
    for a, e in zip(before, (c.k, c.v)):
        a[0, page, :, :3] = e[0, page, :, :3]
        assert torch.equal(a, e)


def test_a_captured_append_takes_the_positions_of_each_replay_and_the_axes_it_was_captured_with():
    c = P.Cache(q_heads=2, kv_heads=1, d=64, page=16, dtype="fp32", rot_dim=64)
    c.reserve([0], [4])
    M.mot_paged_set_axes(c.h, 2, [0] * 16 + [1] * 16)
    x = c.normal(4, 4, 64)
    at, out = torch.zeros((2, 4), dtype=torch.int32, device="cuda"), torch.zeros((4, 2, 64), device="cuda")
    b = c.batch([0], [4])
    args = x[:, :2], x[:, 2:3], x[:, 3:], out
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        M.mot_paged_append_at(c.h, 0, c.c, b, at, *args, stream=st)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        M.mot_paged_append_at(c.h, 0, c.c, b, at, *args, stream=torch.cuda.current_stream())
    M.mot_paged_set_axes(c.h, 2, [1] * 32)   # of the calls behind it
    rate = 1e4 ** (-2 * torch.arange(32, dtype=torch.float64, device="cuda") / 64)
    for step in range(3):
        at.copy_(torch.randint(-500, 500, (2, 4), dtype=torch.int32, device="cuda"))
        g.replay()
        assert c.status() == M.MOT_OK
        angle = torch.cat([at[0].double()[:, None] * rate[:16], at[1].double()[:, None] * rate[16:]], 1)
        want = turned(x[:, :2].double(), angle, False)
        P.assert_close(out, want, 2.0 ** -24 * want.abs() + 2.0 ** -20 * x.abs().amax().double(), f"replay {step}")


def test_refusals():
    c = P.Cache(q_heads=4, kv_heads=2, d=64, page=16, rot_dim=64)
    c.reserve([0], [2])
    b, q, k = c.batch([0], [2]), c.normal(2, 4, 64), c.normal(2, 2, 64)
    out, at = torch.zeros_like(q), torch.zeros((3, 2), dtype=torch.int32, device="cuda")

    def refused(call, status=M.MOT_ERR_INVALID_ARG):
        with pytest.raises(M.MotError) as e:
            call()
        assert e.value.status == status

    refused(lambda: M.mot_paged_append_at(c.h, 0, c.c, b, at, q, k, k, out))   # no axes yet
    for axes, axis, rates in ((0, [0] * 32, None), (5, [0] * 32, None), (2, [0, 2] * 16, None), (2, [0, -1] * 16, None),
                              (2, [0] * 31, None), (1, [0] * 32, [1.0] * 33), (1, [0] * 32, [math.nan] + [1.0] * 31),
                              (1, [0] * 32, [math.inf] + [1.0] * 31), (1, [0] * 32, [65537.0] * 32)):
        refused(lambda: M.mot_paged_set_axes(c.h, axes, axis, rates))
    M.mot_paged_set_axes(c.h, 3, [0, 1] * 16)
    refused(lambda: M.mot_paged_append_at(c.h, 0, c.c, b, None, q, k, k, out))
    refused(lambda: M.mot_paged_append_at(c.h, 0, c.c, b, at[:2].contiguous(), q, k, k, out))   # an axis short
    refused(lambda: M.mot_paged_append_at(c.h, 0, c.c, b, at.T.contiguous(), q, k, k, out))     # [rows][axes]
    refused(lambda: M.mot_paged_append_at(c.h, 0, c.c, b, at.long(), q, k, k, out))
    refused(lambda: M.mot_paged_append_at(c.h, 0, c.c, b, at.cpu(), q, k, k, out))
    refused(lambda: M.mot_paged_append_at(c.h, 0, c.c, b, at.data_ptr() + 2, q, k, k, out))
    refused(lambda: M.mot_paged_append_at(c.h, 0, c.c, b, out.data_ptr(), q, k, k, out))        # what it writes
    refused(lambda: M.mot_paged_append_at(c.h, 0, c.c, b, c.k.data_ptr(), q, k, k, out))
    M.mot_paged_append_at(c.h, 0, c.c, b, at, q, k, k, out)
    assert c.status() == M.MOT_OK
    none = P.Cache(d=64, page=16)
    refused(lambda: M.mot_paged_set_axes(none.h, 1, []), M.MOT_ERR_UNSUPPORTED)
