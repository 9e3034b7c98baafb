"""The paged cache on the GPU in the states that a caller does not mean: refused batches, table entries
and lengths out of range, calls that find more than one thing wrong."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import _paged as P   # noqa: E402
M = P.M
i32 = P.i32


@pytest.mark.parametrize("wrong", ["twice", "outside"])
def test_a_refused_free_of_many_slots_changes_nothing(wrong):
    """More entries than CTAs, the last one named twice or outside the table, again and again beside
    work on another stream."""
    n = 2000
    c = P.Cache(n_pages=3 * n, max_seqs=n, max_pages=4, page=16, kv_heads=1, q_heads=1)
    c.reserve(list(range(n)), [1 + (7 * i) % 40 for i in range(n)])
    c.check()
    seqs = i32(list(range(n - 1)) + [17 if wrong == "twice" else n])
    side, big = torch.cuda.Stream(), torch.randn((2048, 2048), device="cuda")
    for _ in range(40):
        with torch.cuda.stream(side):
            big = big @ big / 2048
        M.mot_paged_free(c.h, c.c, seqs, n)
        assert c.status() == M.MOT_ERR_PAGES
        c.check()
    c.free(list(range(0, n, 3)))
    c.check()
    assert c.status() == M.MOT_OK


def _torn(dtype="bf16"):
    """Slot 0 holds pages 0 and 1, slot 1 pages 2 .. 5 with its entries 1 and 3 (the last, partly filled)
    out of range."""
    c = P.Cache(layers=2, kv_heads=2, q_heads=4, page=16, n_pages=12, max_seqs=4, max_pages=5, dtype=dtype)
    c.reserve([0, 1], [30, 55])
    c.check()
    c.t[1][1], c.t[1][3] = -1, c.n_pages
    c.table[1, 1], c.table[1, 3] = -1, c.n_pages
    return c


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_store_through_a_bad_table_entry_writes_no_page(dtype):
    c = _torn(dtype)
    want = [x.clone() for x in (c.k, c.v)]
    flat = [c.normal(c.L, 1, c.H, 64, c.d) for _ in range(2)]
    M.mot_paged_store(c.h, c.c, i32([1]), 1, *flat)
    assert c.status() == M.MOT_ERR_PAGES
    for x, y, f in zip(want, (c.k, c.v), flat):
        for j in (0, 2):   # the entries in range
            x[:, c.t[1][j]] = f[:, 0, :, 16 * j:16 * j + 16]
        assert torch.equal(x, y)
    # what a load finds there stays as it was
    out = [torch.full_like(f, 7.0) for f in flat]
    M.mot_paged_load(c.h, c.c, i32([1]), 1, *out)
    assert c.status() == M.MOT_ERR_PAGES
    for o, f in zip(out, flat):
        for j in (0, 2):
            assert torch.equal(o[:, 0, :, 16 * j:16 * j + 16], f[:, 0, :, 16 * j:16 * j + 16])
        assert bool((o[:, 0, :, 16:32] == 7).all()) and bool((o[:, 0, :, 48:] == 7).all())


def test_a_fork_of_a_bad_table_entry_counts_and_copies_no_page():
    c = _torn()
    want = [x.clone() for x in (c.k, c.v)]
    M.mot_paged_fork(c.h, c.c, i32([1, 0]), i32([2, 3]), 2)
    assert c.status() == M.MOT_ERR_PAGES
    last = [c.take(1)[0] for _ in range(2)]
    c.t[2], c.n[2] = [c.t[1][0], -1, c.t[1][2], last[0]], 55
    c.t[3], c.n[3] = [c.t[0][0], last[1]], 30
    for p in (c.t[1][0], c.t[1][2], c.t[0][0]):
        c.r[p] += 1
    c.check()
    for x, y in zip(want, (c.k, c.v)):
        x[:, last[1], :, :14] = x[:, c.t[0][1], :, :14]
        assert torch.equal(x, y)


def test_a_refusal_is_still_reported_behind_a_timeout():
    """A step whose reserve is refused and whose attention runs out of time (its first CTA loads nothing,
    under a limit of some 10 ms) reports both, one a call, and changes are held back until both are read."""
    c = P.Cache(q_heads=8, kv_heads=2, d=128, page=32, n_pages=40, max_seqs=3, max_pages=39)
    c.reserve([0], [1100])
    before = [x.clone() for x in (c.k, c.v)]
    q = c.normal(100, 8, 128)
    out, k = torch.zeros_like(q), c.normal(100, 2, 128)
    b = c.batch([0], [100])
    c.reserve([1], [500], ok=False)   # 16 pages of the 5 that are left
    M.mot_debug_set(c.h, True, 20_000_000)
    M.mot_paged_attention(c.h, 0, c.c, b, q, out)
    M.mot_debug_set(c.h, False)
    assert c.status() == M.MOT_ERR_TIMEOUT
    M.mot_paged_append(c.h, 0, c.c, b, q, k, k, out)
    c.reserve([1], [5], ok=False)
    c.check("behind the refused reserve")
    assert c.status() == M.MOT_ERR_PAGES
    for x, y in zip(before, (c.k, c.v)):
        assert torch.equal(x, y)
    assert c.status() == M.MOT_OK
    c.reserve([1], [5])
    c.check()
    assert c.status() == M.MOT_OK


def test_a_refused_change_and_a_value_held_in_range_are_told_apart():
    c = _torn()
    flat = [c.normal(c.L, 1, c.H, 64, c.d) for _ in range(2)]

    def load():
        M.mot_paged_load(c.h, c.c, i32([1]), 1, *flat)

    def refused():
        c.free([0, 0], ok=False)

    for calls, cause in (((), 0), ((load,), M.MOT_PAGES_HELD), ((refused,), M.MOT_PAGES_REFUSED),
                         ((refused, load), M.MOT_PAGES_REFUSED | M.MOT_PAGES_HELD), ((), 0)):
        for call in calls:
            call()
        assert c.status() == (M.MOT_ERR_PAGES if calls else M.MOT_OK)
        assert M.mot_paged_cause(c.h) == cause
    c.check()
    other = M.mot_create_replay(M.mot_replay_config(4, 2, 64, 1, 64, 16, 1))
    with pytest.raises(M.MotError) as e:
        M.mot_paged_cause(other)
    assert e.value.status == M.MOT_ERR_INVALID_ARG


@pytest.mark.parametrize("length", [-1, -2 ** 31, 4 * 16 + 1, 2 ** 30, 2 ** 31 - 1])
def test_changes_of_a_sequence_with_a_length_out_of_range_are_refused(length):
    """A stored length that the table cannot hold: reserve, fork and free of that slot change nothing,
    alone or among others, and the slot is as it was when its length is put right."""
    c = P.Cache(n_pages=20, max_seqs=6, max_pages=4, page=16)
    c.reserve([0, 1, 2], [20, 40, 5])
    c.check()
    c.n[1] = c.lens[1] = length
    for call in (lambda: c.reserve([1], [1], ok=False), lambda: c.reserve([0, 1], [3, 0], ok=False),
                 lambda: c.fork([1], [3], ok=False), lambda: c.fork([0, 1, 2], [3, 4, 5], ok=False),
                 lambda: c.fork([0], [1], ok=False), lambda: c.free([1], ok=False), lambda: c.free([0, 2, 1], ok=False)):
        call()
        c.check()
        assert c.status() == M.MOT_ERR_PAGES
        assert M.mot_paged_cause(c.h) == M.MOT_PAGES_REFUSED
    c.n[1] = c.lens[1] = 40
    c.reserve([1, 0], [24, 1])
    c.free([1])
    c.check()
    assert c.status() == M.MOT_OK


@pytest.mark.parametrize("length", [None, -3, 2 ** 30])
def test_a_compaction_reports_what_it_finds_out_of_range(length):
    """Bad table entries, and lengths that the table cannot hold; the good entries follow their pages."""
    c = _torn()
    c.reserve([2], [20])   # pages 6 and 7
    if length is not None:
        c.t[1][1], c.t[1][3] = 3, 5   # the entries are good, the length of slot 2 is not
        c.table[1, :4] = i32(c.t[1])
        c.lens[2] = length
    c.free([0])
    c.compact()   # six pages are in use: 6 and 7 move to 0 and 1
    if length is not None:   # a row of no length is not read; one that is too long has its entries up to the table's end
        c.n[2] = length
        if length < 0:
            c.t[2] = [6, 7]
    c.check()
    assert c.status() == M.MOT_ERR_PAGES
    assert M.mot_paged_cause(c.h) == M.MOT_PAGES_HELD


def _with_keys(n, first, dtype, d=64):
    """A sequence of n positions whose keys are `first` [n] in their first dimension and 0 in the others,
    and queries [..][4][d] of ones there: scores of first / sqrt(d)."""
    c = P.Cache(q_heads=4, kv_heads=2, d=d, page=32, n_pages=-(-n // 32), max_seqs=1, max_pages=-(-n // 32), dtype=dtype)
    c.reserve([0], [n])
    flat = [torch.zeros((1, 1, 2, n, d), dtype=P.DT[dtype], device="cuda"), c.normal(1, 1, 2, n, d)]
    flat[0][0, 0, :, :, 0] = first.to(P.DT[dtype])
    return c, flat


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 4, 60, 300])
@pytest.mark.parametrize("n", [640, 20000])
def test_infinite_values_of_small_and_of_no_weight(n, new, dtype):
    """The header's sentences: an infinite value comes out as itself while its weight is 2^-90 of the row's
    largest, and as no finite number where its weight is none in 32 bits; other columns are finite. The
    keys lie in tiles that every row sees as a whole, in the same CTA's keys as the largest and in others."""
    c, flat = _with_keys(n, torch.zeros(n, device="cuda"), dtype)
    small, none = [30, 200], [40, 250]   # in the tiles before the last 300 positions
    unit = 8 / 1.4426950408889634        # a base-2 step of the scores
    flat[0][0, 0, :, small, 0] = -90 * unit
    flat[0][0, 0, :, none, 0] = -400 * unit
    flat[1][0, 0, :, 30, 3], flat[1][0, 0, :, 200, 5] = float("inf"), float("-inf")
    flat[1][0, 0, :, 40, 7], flat[1][0, 0, :, 250, 9] = float("inf"), float("-inf")
    M.mot_paged_store(c.h, c.c, i32([0]), 1, *flat)
    q = torch.zeros((new, 4, 64), dtype=P.DT[dtype], device="cuda")
    q[..., 0] = 1
    out = torch.zeros_like(q)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0], [new]), q, out)
    assert c.status() == M.MOT_OK
    assert bool((out[..., 3] == float("inf")).all()) and bool((out[..., 5] == float("-inf")).all())
    assert not bool(torch.isfinite(out[..., [7, 9]]).any())
    rest = [i for i in range(64) if i not in (3, 5, 7, 9)]
    assert bool(torch.isfinite(out[..., rest]).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 4, 60])
def test_rows_without_weights_are_zeros_whatever_the_values_are(new, dtype):
    c, flat = _with_keys(640, torch.full((640,), float("-inf"), device="cuda"), dtype)
    flat[1][0, 0, :, 30, 3], flat[1][0, 0, :, 500, 5], flat[1][0, 0, :, 200, 7] = float("inf"), float("nan"), float("-inf")
    flat[0][0, 0, :, :, 1:] = float("-inf")
    q = torch.ones((new, 4, 64), dtype=P.DT[dtype], device="cuda")
    M.mot_paged_store(c.h, c.c, i32([0]), 1, *flat)
    out = torch.zeros_like(q)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0], [new]), q, out)
    assert c.status() == M.MOT_OK
    assert bool((out == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 4, 60])
def test_infinite_values_beside_keys_of_no_weight_at_all(new, dtype):
    """Long stretches of keys whose scores are -inf, each with an infinite value, so that whole CTAs see no
    weight; the other keys weigh alike. The values' columns are not finite, the others are as the keys with
    weight have them."""
    n = 20000
    first = torch.zeros(n, device="cuda")
    first[1000:9000] = first[12000:12100] = first[19500:19900] = float("-inf")
    c, flat = _with_keys(n, first, dtype)
    for j, col in ((1500, 3), (8000, 5), (12050, 7), (19600, 9)):
        flat[1][0, 0, :, j, col] = float("inf")
    flat[1][..., 20] = 3.0
    M.mot_paged_store(c.h, c.c, i32([0]), 1, *flat)
    q = torch.zeros((new, 4, 64), dtype=P.DT[dtype], device="cuda")
    q[..., 0] = 1
    out = torch.zeros_like(q)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0], [new]), q, out)
    assert c.status() == M.MOT_OK
    assert not bool(torch.isfinite(out[..., [3, 5, 7, 9]]).any())
    assert bool(torch.isfinite(out[..., [i for i in range(64) if i not in (3, 5, 7, 9)]]).all())
    # 12,000 equal weights: sums of n terms are off by n 2^-24 at most on either side
    P.assert_close(out[..., 20], torch.full((new, 4), 3.0, dtype=torch.float64, device="cuda"),
                   P.HALF[dtype] * 3 + 2 * n * 2.0 ** -24 * 3)


def test_buffers_that_overlap_are_refused():
    """What a call writes meets nothing else that it reads, and the cache's arrays do not meet: each pair,
    by a tensor that holds both."""
    n_pages, S, W, H, d = 24, 4, 6, 2, 64
    ints = torch.zeros(4096, dtype=torch.int32, device="cuda")
    table, lens, refs = ints[:S * W].view(S, W), ints[32:32 + S], ints[64:64 + n_pages]
    table.fill_(-1)
    pools = torch.zeros((2, 1, n_pages, H, 16, d), dtype=torch.bfloat16, device="cuda")
    k, v = pools
    cfg = M.make_paged_config(1, 4, H, d, 16, n_pages, S, W)
    h = M.mot_create_paged(cfg)
    seqs, starts = ints[128:130], ints[160:163]
    seqs.copy_(i32([0, 1]))
    starts.copy_(i32([0, 1, 2]))
    c = M.paged_cache(k, v, table, lens, refs)
    b = M.paged_batch(seqs, starts, 2, 2)
    q, kn = torch.zeros((2, 4, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, H, d), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(1024, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    before = ints.clone()

    def refused(call):
        with pytest.raises(M.MotError) as e:
            call()
        assert e.value.status == M.MOT_ERR_INVALID_ARG

    # the cache's own arrays
    for bad in (M.paged_cache(k, v, table, table.view(-1)[4:4 + S], refs), M.paged_cache(k, v, table, lens, ints[20:20 + n_pages]),
                M.paged_cache(k, v, table, lens, ints[33:33 + n_pages]), M.paged_cache(k, k, table, lens, refs),
                M.paged_cache(k, v, table, k.view(torch.int32).view(-1)[:S], refs)):
        refused(lambda: M.mot_paged_reserve(h, bad, b))
    # what a batch and a list of slots lie in
    for x in (lens, table.view(-1), refs):
        refused(lambda: M.mot_paged_reserve(h, c, M.paged_batch(x[:2], starts, 2, 2)))
        refused(lambda: M.mot_paged_reserve(h, c, M.paged_batch(seqs, x[1:4], 2, 2)))
        refused(lambda: M.mot_paged_free(h, c, x[:2], 2))
        refused(lambda: M.mot_paged_fork(h, c, x[:1], seqs, 1))
        refused(lambda: M.mot_paged_fork(h, c, seqs, x[:1], 1))
        refused(lambda: M.mot_paged_compact(h, c, x[2:3]))
    # outputs over the cache's arrays and the batch's (addresses: the tensors are of other types)
    base = ints.data_ptr()
    for at in (0, 128, 256, 512, 640):   # table, lens, refs, seqs, starts
        refused(lambda: M.mot_paged_attention(h, 0, c, b, q, base + at))
        refused(lambda: M.mot_paged_append(h, 0, c, b, q, kn, kn, base + at))
    flat = torch.zeros((2, 1, 1, H, 16, d), dtype=torch.bfloat16, device="cuda")
    for x in (ints[:1024].view(torch.bfloat16).view(1, 1, H, 16, d), pools[0, :, :1].view(1, 1, H, 16, d)):
        refused(lambda: M.mot_paged_load(h, c, seqs[:1], 1, x, flat[0]))
        refused(lambda: M.mot_paged_load(h, c, seqs[:1], 1, flat[0], x))
    # norm weights under the output
    refused(lambda: M.mot_paged_append(h, 0, c, b, q, kn, kn, w[:512].view(2, 4, d), q_norm=w[448:512]))
    refused(lambda: M.mot_paged_append(h, 0, c, b, q, kn, kn, w[:512].view(2, 4, d), k_norm=w[:64]))
    assert M.mot_get_device_status(h) == M.MOT_OK
    assert torch.equal(ints, before)
    # and none of it where they only stand side by side
    M.mot_paged_reserve(h, c, b)
    M.mot_paged_append(h, 0, c, b, q, kn, kn, w[:512].view(2, 4, d), q_norm=w[512:576], k_norm=w[576:640])
    M.mot_paged_attention(h, 0, c, b, q, out)
    M.mot_paged_load(h, c, seqs[:1], 1, flat[0], flat[1])
    M.mot_paged_compact(h, c, ints[31:32])
    assert M.mot_get_device_status(h) == M.MOT_OK
    assert int(ints[31]) == 2


def test_a_paged_handle_takes_no_calls_of_other_kinds():
    """Each call with arguments that are good for a handle of its own kind, or would pass as such."""
    import ctypes
    c = P.Cache()
    L, h, n = M._lib, c.h.ptr, ctypes.c_int32(7)
    x = torch.zeros(4096, dtype=torch.int32, device="cuda").data_ptr()
    out = (ctypes.c_int32 * 4)()
    bad = M.MOT_ERR_INVALID_ARG
    assert L.mot_load_weights(h, x, 0) == bad
    assert L.mot_translate(h, x, x, x, 0, x, x, None) == bad
    assert L.mot_translate_host(h, x, x, x, 0, x, x, None) == bad
    assert L.mot_translate_h(h, x, x, 0, x, x, None) == bad
    assert L.mot_translate_bt(h, x, x, x, 0, x, x, None) == bad
    assert L.mot_replay_attention(h, 0, x, x, x, x, x, 0, x, None) == bad
    assert L.mot_replay_select(h, x, x, 0, x, None) == bad
    assert L.mot_get_layer_map(h, out, 0) == bad
    assert L.mot_get_path(h, ctypes.byref(n)) == bad
    assert L.mot_set_schedule(h, 0) == bad and L.mot_get_schedule(h, ctypes.byref(n)) == bad
    assert L.mot_set_routing(h, 0) == bad and L.mot_get_routing(h, ctypes.byref(n)) == bad
    assert L.mot_get_expert_counts(h, out, 0, None) == bad
    assert L.mot_debug_fixed_gate(h, None) == bad
    assert n.value == 7
    # and those that it does
    count = ctypes.c_int64()
    assert L.mot_get_launch_count(h, ctypes.byref(count)) == M.MOT_OK
    assert L.mot_debug_set(h, 0, 0) == M.MOT_OK
    assert L.mot_profile_enable(h, 1) == M.MOT_OK
    c.reserve([0], [5])
    stats = (M.mot_kernel_stat * 4)()
    assert L.mot_profile_read(h, stats, 4, ctypes.byref(n)) == M.MOT_OK and n.value == 1
    assert stats[0].name == b"paged_reserve" and stats[0].launches == 1
    assert L.mot_profile_enable(h, 0) == M.MOT_OK
    assert c.status() == M.MOT_OK
