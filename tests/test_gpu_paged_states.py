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
