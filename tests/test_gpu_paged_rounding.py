"""What the attention's roundings may do to its results: bounds that are tighter than those of the general
tests, each where it holds."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import _paged as P   # noqa: E402
M = P.M
i32 = P.i32
LOG2E = 1.4426950408889634


def _one_sequence(n, scores, values, d, dtype):
    """A cache of one sequence of n positions whose key j has the product scores[j] with a query of ones in
    its first dimension, and whose values are `values` [d] at every position."""
    page = 32
    pages = -(-n // page)
    c = P.Cache(q_heads=4, kv_heads=2, d=d, page=page, n_pages=pages + 1, max_seqs=1, max_pages=pages, dtype=dtype)
    c.reserve([0], [n])
    flat = [torch.zeros((1, 1, 2, n, d), dtype=P.DT[dtype], device="cuda") for _ in range(2)]
    flat[0][0, 0, :, :, 0] = scores.to(P.DT[dtype])
    flat[1][:] = values.to(P.DT[dtype])
    M.mot_paged_store(c.h, c.c, i32([0]), 1, *flat)
    return c


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 4, 300])
def test_a_mean_of_equal_values_is_that_value(new, d, dtype):
    """Every position has the same values, so whatever the weights are their mean is those values. The
    weights are rounded, but as numerator and denominator take them alike: what is left are 32-bit sums, n
    additions of 2^-24 on either side and a handful of roundings, less than half of a step of bf16 above
    any value. One key outweighs the others by 2^6 to 2^7.9, so no average hides a rounding, and it lies
    two tiles behind the next heaviest, in one CTA's keys, so that its weight is not 1."""
    n = 20000
    scores = torch.full((n,), -60.0, device="cuda")
    scores[8 * 128 + 5], scores[10 * 128 + 44] = 0.0, 5.0
    values = 1 + torch.arange(d, device="cuda") / 128.0   # steps of bf16: each is a bf16 value
    c = _one_sequence(n, scores, values, d, dtype)
    q = torch.zeros((new, 4, d), dtype=P.DT[dtype], device="cuda")
    # base-2 scores of the heavy key: 6.0 .. 7.9
    rows = torch.linspace(6.0, 7.9, new * 4, device="cuda").view(new, 4)
    q[..., 0] = (rows / LOG2E * math.sqrt(d) / 5.0).to(q.dtype)
    out = torch.zeros_like(q)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0], [new]), q, out)
    assert c.status() == M.MOT_OK
    want = values.double().expand(new, 4, d)
    P.assert_close(out, want, 0 * want if dtype == "bf16" else (2 * n + 16) * 2.0 ** -24 * want)


@pytest.mark.parametrize("hq,h,d,new", [(8, 2, 64, 1), (8, 2, 64, 4), (14, 2, 64, 2), (7, 1, 128, 1), (16, 2, 128, 2), (3, 3, 128, 16)])
def test_few_rows_hold_their_weights_to_17_bits(hq, h, d, new):
    """Up to 16 rows per key/value head in bf16: the weights enter in two bf16 parts. The first is off by half a
    step, 2^-8 of the weight's power of two; what is left lies a binade lower or is that tie, which is exact, so
    the second is off by 2^-17. The result's own rounding and the 32-bit terms of the general bound are all
    that comes on top. The oracle with the second part left out breaks this bound, so the test can tell."""
    lens = [777, 130 + new, 61 + new]
    c = P.Cache(q_heads=hq, kv_heads=h, d=d, page=32, n_pages=40, max_seqs=3, max_pages=25, seed=hq + new)
    c.reserve([0, 1, 2], lens)
    q = c.normal(3 * new, hq, d)
    out = torch.zeros_like(q)
    M.mot_paged_attention(c.h, 0, c.c, c.batch([0, 1, 2], [new] * 3), q, out)
    assert c.status() == M.MOT_OK
    told = 0
    for i, n in enumerate(lens):
        K, V = c.rows(i)
        rows = slice(i * new, (i + 1) * new)
        ref, absv, slop = P.attention(q[rows], K, V)
        tol = 2.0 ** -8 * ref.abs() + 2.0 ** -17 * absv + slop
        P.assert_close(out[rows], ref, tol, f"slot {i}")
        for r in range(new):   # the mistake, in the oracle
            p = n - new + r + 1
            Kr, Vr = (x[:, :p].repeat_interleave(hq // h, 0) for x in (K, V))
            s = torch.einsum("hd,hnd->hn", q[i * new + r].double(), Kr) / math.sqrt(d)
            w = torch.exp(s - s.amax(1, keepdim=True))
            one = torch.einsum("hn,hnd->hd", w.to(torch.bfloat16).double(), Vr) / w.sum(1, keepdim=True)
            told += int(((one.to(torch.bfloat16).double() - ref[r]).abs() > tol[r]).sum())
    assert told > 0.02 * out.numel(), told
