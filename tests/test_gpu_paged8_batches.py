"""Appends to 8-bit pages of batches that mix single rows, prompts and entries without rows: the pages are dealt out by the
row or by the entry as the counts go, and what they hold is the same."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import _paged as P   # noqa: E402
import _paged8 as P8   # noqa: E402
from test_gpu_paged8 import _check_pages, _turned   # noqa: E402
M = P.M
i32 = P.i32


def _append(c, calls, new, x, starts, hint):
    """The rows of all entries in one call, or in several of some entries each."""
    out = torch.zeros((x.shape[0], 4, c.d), dtype=torch.bfloat16, device="cuda")
    for part in calls:
        at = [0]
        for i in part:
            at.append(at[-1] + new[i])
        rows = torch.cat([torch.arange(starts[i], starts[i + 1]) for i in part]).cuda()
        y, q = x[rows], torch.zeros((len(rows), 4, c.d), dtype=torch.bfloat16, device="cuda")
        M.mot_paged_append(c.h, 0, c.c, M.paged_batch(i32(part), i32(at), len(part), at[-1], hint), y[:, :4], y[:, 4:6], y[:, 6:], q)
        out[rows] = q
    assert c.status() == M.MOT_OK
    return out


@pytest.mark.parametrize("page,d", [(16, 64), (64, 128)])
@pytest.mark.parametrize("name,new", [
    ("single rows and a prompt", [1] * 200 + [333] + [1] * 150),                        # by the row
    ("rows beside entries without any", [0, 0, 40] * 30 + [0] * 2000 + [17, 1, 0]),     # by the row
    ("threes", [3] * 300),                                                              # by the entry
    ("two a sequence", [2] * 150 + [1] * 10),                                           # by the row
    ("a border", [2] * 150 + [3]),                                                      # one row above it
    ("a prompt alone", [700]),
])
def test_a_batch_gives_what_its_parts_give(name, new, page, d):
    n = len(new)
    starts = [sum(new[:i]) for i in range(n + 1)]
    by_size = [[i for i in range(n) if new[i] <= 1], [i for i in range(n) if new[i] > 1]]
    ways = [list(range(n))], [p for p in by_size if p], [list(range(0, n, 2)), list(range(1, n, 2))][:1 + (n > 1)]
    got, x = [], None
    for k, calls in enumerate(ways):
        c = P8.Cache(q_heads=4, kv_heads=2, d=d, page=page, n_pages=2600, max_seqs=2200, max_pages=64, rot_dim=d, seed=5)
        c.reserve(list(range(n)), [m + i % 9 if m else 0 for i, m in enumerate(new)])
        before = [t.double() for t in (c.k, c.v, c.ks, c.vs)]
        x = c.normal(starts[-1], 8, d) if x is None else x
        got.append([_append(c, calls, new, x, starts, (1, 5000, max(new))[k])] + c.bytes())
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
    y = x.double()
    pos = torch.cat([torch.arange(c.n[s] - m, c.n[s]) for s, m in enumerate(new)]).cuda()
    keys = _turned(y[:, 4:6], pos.double()[:, None] * 1e4 ** (-2 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d), False)
    _check_pages(c, before, 0, list(range(n)), new, keys, 2.0 ** -20 * keys.abs().amax(2), y[:, 6:])
