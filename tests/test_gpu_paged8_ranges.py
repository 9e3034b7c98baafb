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
