"""Calls on a paged cache whose launches may begin before what is in front of them in the stream has ended: kernels of one
and two streams, copies and memory sets, eager, captured, and with a wait between the calls."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import _paged as P   # noqa: E402
import _paged8 as P8   # noqa: E402
M = P.M
i32 = P.i32


def _replayed(make, step, outputs, rounds=10):
    """`step(state, k)` over states that `make` makes: eager, eager with a wait behind every call, and a graph; their
    outputs are equal round by round."""
    eager, waiting, graph = make(), make(), make()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        step(graph, lambda: None)
    for k in range(rounds):
        step(eager, lambda: None)
        step(waiting, torch.cuda.synchronize)
        g.replay()
        torch.cuda.synchronize()
        for n, (a, b, c) in enumerate(zip(*(outputs(s) for s in (eager, waiting, graph)))):
            assert torch.equal(a, b) and torch.equal(a, c), (k, n)


def _kind(kind, **shape):
    return P8.Cache(**shape) if kind == "8" else P.Cache(dtype=kind, **shape)


@pytest.mark.parametrize("kind", ["bf16", "fp32", "8"])
@pytest.mark.parametrize("new", [[1, 1, 1], [150, 3, 40]])
@pytest.mark.parametrize("axes", [False, True])
def test_appends_behind_work_of_two_streams(kind, new, axes):
    """A step of a serving loop: rows and positions that another stream has just made, sequences that the call before has
    made longer, pages that the append before has written and the attention reads."""
    H, Hq, d = 2, 6, 128
    seqs, rows = [0, 1, 2], sum(new)
    side = torch.cuda.Stream()

    def make():
        c = _kind(kind, q_heads=Hq, kv_heads=H, d=d, page=32, n_pages=400, max_pages=100, rot_dim=d, seed=7)
        c.reserve(seqs, [300, 33, 700])
        if axes:
            M.mot_paged_set_axes(c.h, 2, [i % 2 for i in range(d // 2)])
        x, src = c.normal(rows, Hq + 2 * H, d), c.normal(rows, Hq + 2 * H, d)
        at, count = torch.zeros((2, rows), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        q, out = torch.zeros_like(x[:, :Hq].contiguous()), torch.zeros_like(x[:, :Hq].contiguous())
        return c, x, src, at, count, q, out, c.batch(seqs, new)

    def step(s, wait):
        c, x, src, at, count, q, out, b = s
        st = torch.cuda.current_stream()
        side.wait_stream(st)
        with torch.cuda.stream(side):
            count.add_(37)
            at.copy_(count.expand(2, rows)).mul_(3)
        x.copy_(src).mul_(0.5)
        wait()
        M.mot_paged_reserve(c.h, c.c, b)
        st.wait_stream(side)
        wait()
        call = (lambda *a: M.mot_paged_append_at(c.h, 0, c.c, b, at, *a)) if axes else (lambda *a: M.mot_paged_append(c.h, 0, c.c, b, *a))
        call(x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], q)
        wait()
        M.mot_paged_attention(c.h, 0, c.c, b, q, out)
        wait()
        src[:, :Hq].add_(out)   # behind the calls: a kernel that overlaps nothing
        src.mul_(0.9)

    def outputs(s):
        assert s[0].status() == M.MOT_OK
        assert bool(s[6].isfinite().all())
        c = s[0]
        return [s[2], s[5], s[6], c.lens] + (c.bytes() if kind == "8" else [c.k, c.v])

    _replayed(make, step, outputs)


@pytest.mark.parametrize("kind", ["bf16", "fp32", "8"])
@pytest.mark.parametrize("new", [[1, 1], [90, 20]])
def test_a_copy_or_a_memory_set_right_in_front_of_a_call(kind, new):
    """What a call reads is written by a copy, or a memory set, that the stream holds right before it: appends, attention,
    and the copies between pages and a contiguous cache."""
    H, Hq, d = 2, 4, 64
    rows = sum(new)

    def make():
        c = _kind(kind, q_heads=Hq, kv_heads=H, d=d, page=16, n_pages=200, max_pages=100, seed=3)
        c.reserve([0, 1, 2], [300, 500, 1500])
        x, src = [[c.normal(rows, n, d) for n in (Hq, H, H)] for _ in range(2)]   # contiguous: plain copies and memory sets
        flat, kv = [[c.normal(1, 1, H, 1500, d) for _ in range(2)] for _ in range(2)]
        q = torch.zeros((rows, Hq, d), dtype=x[0].dtype, device="cuda")
        outs = [torch.zeros_like(q) for _ in range(4)]
        return c, x, src, flat, kv, q, outs, c.batch([0, 1], new), i32([2])

    def step(s, wait):
        c, x, src, flat, kv, q, outs, b, slot = s
        x[0].zero_()
        x[2].copy_(src[2])
        x[1].copy_(src[1])   # a device copy right in front of the append
        wait()
        M.mot_paged_append(c.h, 0, c.c, b, *x, outs[0])
        wait()
        q.copy_(src[0])
        wait()
        M.mot_paged_attention(c.h, 0, c.c, b, q, outs[1])
        wait()
        x[1].zero_()         # a memory set
        wait()
        M.mot_paged_append(c.h, 0, c.c, b, *x, outs[0])
        wait()
        q.zero_()
        wait()
        M.mot_paged_attention(c.h, 0, c.c, b, q, outs[2])
        wait()
        flat[0].zero_()
        flat[1].copy_(kv[1])
        wait()
        M.mot_paged_store(c.h, c.c, slot, 1, *flat)
        wait()
        for f in flat:
            f.fill_(0)
        wait()
        M.mot_paged_load(c.h, c.c, slot, 1, *flat)
        wait()
        src[0].copy_(outs[1])
        kv[1].mul_(0.75)

    def outputs(s):
        c = s[0]
        assert c.status() == M.MOT_OK
        return [s[3][0], s[3][1], s[6][0], s[6][1], s[6][2], s[2][0]] + (c.bytes() if kind == "8" else [c.k, c.v])

    _replayed(make, step, outputs)
