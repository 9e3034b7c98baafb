"""Attention over 8-bit pages at the ends of its ranges: scores, queries, weights and scales far from one another."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import _paged as P   # noqa: E402
import _paged8 as P8   # noqa: E402
from test_gpu_paged8 import _attend   # noqa: E402
M = P.M
i32 = P.i32


def _one_dimension(c, s, keys):
    """The keys of slot s: `keys` (8-bit values, one a position) in dimension 0 of every head, 0 elsewhere, scales 1."""
    c.k.zero_()
    c.ks[0, c.t[s]] = 1.0
    for j, p in enumerate(c.t[s]):
        x = keys[j * c.P:(j + 1) * c.P].to(P8.F8)
        c.k.view(torch.uint8)[0, p, :, :len(x), 0] = x.view(torch.uint8)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 9, 250])
@pytest.mark.parametrize("size", [2.0 ** 20, -(2.0 ** 20), 2.0 ** 27, 2.0 ** 60, -(2.0 ** 100)])
def test_scores_far_from_zero(size, new, d):
    """Scores up to 2^107, which fp32 holds in steps of whole powers of two: no two of them are near one another (2^8
    apart at least), so a row's result is the value of the best key that it sees."""
    c = P8.Cache(q_heads=4, kv_heads=2, d=d, page=16, n_pages=20, max_pages=16)
    c.reserve([0], [250])
    all8 = torch.arange(256, dtype=torch.uint8, device="cuda")
    all8 = all8[(all8 != 127) & (all8 != 255) & (all8 != 128)]   # every 8-bit value but NaN, 0 once
    keys = all8.view(P8.F8).float()[torch.randperm(len(all8), generator=c.gen, device="cuda")[:250]]
    _one_dimension(c, 0, keys)
    q = torch.zeros((new, 4, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = size
    _, out = _attend(c, [0], [new], q=q)
    assert c.status() == M.MOT_OK
    V = c.rows(0)[1].repeat_interleave(2, 0)
    for r in range(new):
        best = int((keys[:250 - new + r + 1].double() * size).argmax())
        assert torch.equal(out[r].double(), V[:, best]), r


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 9, 140])
@pytest.mark.parametrize("eq,ek", [(-58, 59), (-64, 65), (-66, 66), (-100, 66), (52, -52), (30, -29)])
def test_queries_and_keys_that_meet_from_far(eq, ek, new, d):
    """Queries of about 2^eq against keys of about 2^ek, whose products are scores of some size: every element counts."""
    c = P8.Cache(q_heads=8, kv_heads=2, d=d, page=32, n_pages=12, max_pages=8)
    c.reserve([0], [200])
    c.ks[0, c.t[0]] = torch.exp2(torch.tensor([ek - 6.0, ek - 7.0, ek - 6.0, ek - 8.0, ek - 6.0, ek - 5.0, ek - 6.0], device="cuda")
                                 .clamp(-60, 60))[:, None].expand(-1, 2)
    q = c.normal(new, 8, d) * 2.0 ** eq
    _, out = _attend(c, [0], [new], q=q)
    assert c.status() == M.MOT_OK
    P8.check_attention(c, [0], [new], q, out, label=f"{eq} {ek}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 9, 140])
@pytest.mark.parametrize("size,ek", [(2.0 ** 127, 60), (1.99 * 2.0 ** 127, -60), (2.0 ** 100, 60), (2.0 ** -130, -60), (2.0 ** -133, 60)])
def test_queries_at_the_ends_of_bf16_that_no_key_meets(size, ek, new, d):
    """One element of each query at an end of bf16, keys that are 0 there and of any scale elsewhere: scores of 0, and
    the mean of the values that are seen."""
    c = P8.Cache(q_heads=4, kv_heads=2, d=d, page=16, n_pages=20, max_pages=16)
    c.reserve([0], [200])
    c.k.view(torch.uint8)[..., 3] = 0
    c.ks[0, c.t[0]] = 2.0 ** ek
    c.ks[0, c.t[0][3]] = 2.0 ** -ek
    q = torch.zeros((new, 4, d), dtype=torch.bfloat16, device="cuda")
    q[..., 3] = size
    _, out = _attend(c, [0], [new], q=q)
    assert c.status() == M.MOT_OK
    V = c.rows(0)[1].repeat_interleave(2, 0)
    for r in range(new):
        seen = V[:, :200 - new + r + 1]
        # weights that are powers of two, exact in fp16; sums of n values in fp32; the result rounded once
        P.assert_close(out[r], seen.mean(1), 2.0 ** -8 * seen.mean(1).abs() + 210 * 2.0 ** -24 * seen.abs().mean(1), f"row {r}")


@pytest.mark.parametrize("new", [1, 9, 140])
def test_scores_that_fp32_does_not_hold(new):
    """A score above 2^128 makes the rows that see it NaN, one below -2^128 counts for nothing beside others. Value scales
    of 1: another's exponent would be added to scores of 2^97, whose steps in fp32 are larger."""
    c = P8.Cache(q_heads=4, kv_heads=2, d=64, page=16, n_pages=20, max_pages=16)
    c.reserve([0], [200])
    c.vs.fill_(1.0)
    keys = torch.full((200,), 1.0, device="cuda")
    keys[[3, 70]] = -448.0
    _one_dimension(c, 0, keys)
    c.ks[0, c.t[0][70 // 16]] = c.ks[0, c.t[0][0]] = 2.0 ** 60
    c.k.view(torch.uint8)[0, c.t[0][70 // 16], :, :, 0] = c.k.view(torch.uint8)[0, c.t[0][0], :, :, 0] = 0
    for j in (3, 70):
        c.k[0, c.t[0][j // 16], :, j % 16, 0] = torch.tensor(-448.0, device="cuda").to(P8.F8)
    q = torch.zeros((new, 4, 64), dtype=torch.bfloat16, device="cuda")
    q[:, :2, 0], q[:, 2:, 0] = 2.0 ** 100, -(2.0 ** 100)
    _, out = _attend(c, [0], [new], q=q)
    assert c.status() == M.MOT_OK
    assert bool(out[:, 2:].isnan().all())
    V = c.rows(0)[1][0]
    best = [j for j in range(200) if keys[j] > 0 and j // 16 not in (0, 70 // 16)]   # scores of 2^97; the others 0 or less
    for r in range(new):
        ref = V[[j for j in best if j <= 200 - new + r]].mean(0)
        P.assert_close(out[r, 0], ref, 2.0 ** -8 * ref.abs() + 210 * 2.0 ** -24 * V.abs().mean(0), f"row {r}")


@pytest.mark.parametrize("where", ["first", "last"])
@pytest.mark.parametrize("new", [1, 9])
def test_many_small_weights_count_as_much_as_the_sum_says(new, where):
    """One key 25.4 powers of two ahead of 131,000 others, all values the same, and as many heads as keep an item's keys
    in one piece: what the others add to the sum of the weights (0.3% of it) they add to the result."""
    n, page, d = 131000, 128, 64
    heads = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    c = P8.Cache(q_heads=2 * heads, kv_heads=heads, d=d, page=page, n_pages=1024, max_pages=1024, max_seqs=1)
    c.reserve([0], [n])
    c.k.zero_()
    c.ks.fill_(1.0)
    c.v.view(torch.uint8).fill_(torch.tensor(1.875).to(P8.F8).view(torch.uint8).item())
    c.vs.fill_(0.25)
    at = 0 if where == "first" else n - new
    c.k.view(torch.uint8)[0, c.t[0][at // page], :, at % page, 0] = torch.tensor(16.0).to(P8.F8).view(torch.uint8).item()
    q = torch.zeros((new, 2 * heads, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 25.4 * math.log(2) * math.sqrt(d) / 16
    # the others' part of the sum is 131,000 2^-25.4 = 0.003. In fp16 it is off by 2^-7 of itself (2^-32 of the largest
    # for each); in fp32 sums beside the largest a step of 16 keys is off by a third of itself at most, 0.001 in all; the
    # border to the next bf16 is 2^-9 of the value away
    _, out = _attend(c, [0], [new], q=q)
    assert c.status() == M.MOT_OK
    assert bool((out == 1.875 / 4).all()), out.double().unique()


BAD = {3.0: 2.0, 0.0: 2.0 ** -60, -4.0: 4.0, math.nan: 2.0 ** 60, math.inf: 2.0 ** 60, -math.inf: 2.0 ** 60, 2.0 ** 61: 2.0 ** 60,
       2.0 ** -61: 2.0 ** -60, 1e-40: 2.0 ** -60, 0.75: 0.5}


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("bad", BAD, ids=str)
def test_a_scale_that_is_no_power_of_two_is_the_same_to_every_call_and_reported(bad, d, page):
    """Attention of few rows and of chunks, load, a store that cuts a page and appends to one: what they give for the
    power that the scale is taken as, and a status that says so; nothing for scales of pages that no call meets."""
    made = []
    for way in ("good", "bad"):
        got = []
        for which in ("ks", "vs"):
            c = P8.Cache(q_heads=6, kv_heads=2, d=d, page=page, n_pages=40, max_pages=12, seed=3)
            c.reserve([0, 1], [5 * page + 5, page + 3])
            scales = getattr(c, which)
            at = c.t[0][2], c.t[0][-1]   # a full page, and the last
            scales[0, [p for p in range(40) if p not in c.t[0] + c.t[1]]] = bad

            def put(p):
                scales[0, p, 1] = bad if way == "bad" else BAD[bad]

            def status(met=True):
                s = M.mot_get_device_status(c.h)
                assert s == (M.MOT_ERR_PAGES if way == "bad" and met else M.MOT_OK)
                if s != M.MOT_OK:
                    assert M.mot_paged_cause(c.h) == M.MOT_PAGES_HELD

            put(at[0])
            for new in (1, 40):
                q, out = _attend(c, [0], [new])
                got.append(out)
                status()
                got.append(_attend(c, [1], [new], q=q)[1])   # of the other sequence
                status(False)
            flat = [torch.zeros((1, 2, 2, 5 * page + 9, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            M.mot_paged_load(c.h, c.c, i32([0, 1]), 2, *flat)
            status()
            got += flat
            scales[0, at[0], 1] = 1.0
            x = c.normal(3, 10, d)
            q = torch.zeros((3, 6, d), dtype=torch.bfloat16, device="cuda")
            for new in ([2, 1], [1]):
                put(at[1])
                c.reserve([0, 1][:len(new)], new)
                M.mot_paged_append(c.h, 0, c.c, c.batch([0, 1][:len(new)], new), x[:, :6], x[:, 6:8], x[:, 8:], q)
                status()
                got += [q.clone()] + [t[0, c.t[0] + c.t[1]].clone() for t in c.bytes()[:2]]
                got.append(scales[0, at[1]].clone())
            put(at[1])
            M.mot_paged_store(c.h, c.c, i32([0]), 1, *[c.normal(1, 1, 2, 5 * page + 2, d) for _ in range(2)])
            assert M.mot_get_device_status(c.h) == M.MOT_ERR_PAGES   # it is shorter than the sequence, too
            got += [t[0, c.t[0]].clone() for t in c.bytes()[:2]] + [scales[0, at[1]].clone()]
        made.append(got)
    for k, (a, b) in enumerate(zip(*made)):
        assert P8.same(a.double(), b.double()), k


def _exponents(kind, n, gen):
    """Value scales' exponents of n pages of 16 positions, eight to a tile of 128 keys."""
    j = torch.arange(n, device="cuda")
    if kind == "rise":      # by 20 from tile to tile, within each by 14
        return (-60 + 20 * (j // 8 % 7) - 2 * (j % 8)).clamp(-60, 60)
    if kind == "fall":
        return (60 - 20 * (j // 8 % 7) + 2 * (j % 8)).clamp(-60, 60)
    if kind == "tiles":     # one tile's at the end, the next one's at the other
        return torch.where(j // 8 % 2 == 0, 55 + j % 6, -60 + j % 6)
    if kind == "pages":
        return torch.where(j % 2 == 0, 60, -60)
    if kind == "steps":     # spans of just about 60 in a tile
        return torch.where(j % 8 < 4, 30, -29 - j // 8 % 3)
    return torch.randint(-60, 61, (n,), generator=gen, device="cuda")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 9])
@pytest.mark.parametrize("kind", ["rise", "fall", "tiles", "pages", "steps", "any"])
def test_scales_far_apart_in_pieces_of_several_tiles(kind, new, d):
    """Value scales up to 2^120 apart from tile to tile and within one, where a CTA goes over many tiles of an item under a
    running maximum: 48 items of 11 to 17 tiles in pieces of about seven, of 34 to 48 in pieces or runs of five and more."""
    lens = [6100, 4300, 5700] if new == 1 else [2100, 1300, 1700]
    c = P8.Cache(q_heads=32, kv_heads=16, d=d, page=16, n_pages=1010, max_pages=400)
    c.reserve([0, 1, 2], lens)
    for s in range(3):
        for x in range(16):
            e = _exponents(kind, len(c.t[s]), c.gen)
            c.vs[0, c.t[s], x] = torch.exp2(e.float()) if x % 2 else torch.exp2(e.flip(0).float())
    q, out = _attend(c, [0, 1, 2], [new] * 3)
    assert c.status() == M.MOT_OK
    P8.check_attention(c, [0, 1, 2], [new] * 3, q, out, label=kind)
    # the keys of the small scales' pages have nearly all of the weight in half of the heads
    for s in range(3):
        small = [p for k, p in enumerate(c.t[s]) if k % 3 == 0]
        c.ks[0, small, :8] = 4.0
    _, out = _attend(c, [0, 1, 2], [new] * 3, q=q)
    assert c.status() == M.MOT_OK
    P8.check_attention(c, [0, 1, 2], [new] * 3, q, out, label=kind + " weighted")


@pytest.mark.parametrize("kind", ["tiles", "any"])
def test_scales_far_apart_in_chunks_of_two_streams(kind):
    c = P8.Cache(q_heads=8, kv_heads=1, d=128, page=16, n_pages=140, max_pages=140)
    c.reserve([0], [2100])
    c.vs[0, c.t[0], 0] = torch.exp2(_exponents(kind, len(c.t[0]), c.gen).float())
    for new in (40, 300):
        q, out = _attend(c, [0], [new])
        P8.check_attention(c, [0], [new], q, out, label=kind)
    assert c.status() == M.MOT_OK


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("kind", ["tiles", "pages", "any"])
def test_value_scales_far_apart_under_queries_far_from_their_keys(kind, new, d):
    """Both at once: rows whose scores are worked out first (queries of 2^-66 and keys of 2^66) beside rows of zeros, in
    tiles whose value scales lie further apart than a weight reaches."""
    c = P8.Cache(q_heads=4, kv_heads=2, d=d, page=16, n_pages=60, max_pages=40)
    c.reserve([0], [600])
    c.ks[0, c.t[0]] = 2.0 ** 60
    e = _exponents(kind, len(c.t[0]), c.gen).float()
    c.vs[0, c.t[0]] = torch.exp2(torch.stack([e, e.flip(0)], 1))
    q = c.normal(new, 4, d) * 2.0 ** -66
    q[:, 1::2][new // 2:] = 0.0
    _, out = _attend(c, [0], [new], q=q)
    assert c.status() == M.MOT_OK
    P8.check_attention(c, [0], [new], q, out, label=kind)
