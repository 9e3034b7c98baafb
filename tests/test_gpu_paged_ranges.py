"""Attention over 16- and 32-bit pages with scores far from zero."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import _paged as P   # noqa: E402
M = P.M


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 9, 250])
@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 27, -(2.0 ** 30), 2.0 ** 34, -(2.0 ** 60), 2.0 ** 100])
def test_scores_far_from_zero(size, new, d, dtype):
    """Scores whose steps in fp32 are whole powers of two, no two of them near one another (2^16 apart at least): a row's
    result is the value of the best key that it sees."""
    c = P.Cache(q_heads=4, kv_heads=2, d=d, page=16, n_pages=20, max_pages=16, dtype=dtype)
    c.reserve([0], [250])
    keys = torch.randperm(250, generator=c.gen, device="cuda").float() - 125   # exact in bf16
    c.k.zero_()
    for j, p in enumerate(c.t[0]):
        x = keys[16 * j:16 * j + 16]
        c.k[0, p, :, :len(x), 0] = x.to(c.k.dtype)
    q = torch.zeros((new, 4, d), dtype=P.DT[dtype], device="cuda")
    q[..., 0] = size
    out = torch.zeros_like(q)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0], [new]), q, out)
    assert c.status() == M.MOT_OK
    V = c.rows(0)[1].repeat_interleave(2, 0)
    for r in range(new):
        best = int((keys[:250 - new + r + 1].double() * size).argmax())
        # weights of 1 and of 0, whatever 2^x of an x that is off by some steps of the score may be
        P.assert_close(out[r], V[:, best], 2.0 ** -23 * V[:, best].abs(), f"row {r}")
