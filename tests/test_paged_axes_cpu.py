"""Appends by several positions of a row, what is refused before any CUDA call."""
import ctypes

import pytest

from paper_2607_28979_gb300 import build as mot_build

mot_build.build()
import paper_2607_28979_gb300.mot as M   # noqa: E402
from test_paged_binding_cpu import GOOD, H, D, T, _batch, _cache, _handle, _reaches_the_library, _refused   # noqa: E402

I32 = dict(dtype="torch.int32")
KV = T(3, H, D)


def _with_axes(n):
    h = _handle()
    h.axes = n
    return h


def test_null_handles_and_arguments():
    lib, bad = M._lib, M.MOT_ERR_INVALID_ARG
    c, b = ctypes.byref(M.paged_cache(64, 128, 64, 64, 64)), ctypes.byref(M.paged_batch(64, 64, 1, 1))
    axis = (ctypes.c_int32 * 64)()
    assert lib.mot_paged_set_axes(None, 1, axis, None) == bad
    assert lib.mot_paged_append_at(None, 0, c, b, 64, 64, 64, 64, 64, 64, 64, None, None, 64, None) == bad


@pytest.mark.parametrize("match, at", [
    ("positions is not a CUDA tensor", T(3, 3, is_cuda=False, **I32)),
    ("positions is of type torch.int64", T(3, 3, dtype="torch.int64")),
    ("positions is not contiguous", T(3, 3, stride=(6, 1), **I32)),
    ("positions has 6 elements, 9 are", T(2, 3, **I32)),
    (r"positions is \(3, 4\)", T(3, 4, **I32)),
    ("positions is on another device", T(3, 3, device=1, **I32)),
])
def test_positions_are_checked(match, at):
    _refused(match, lambda: M.mot_paged_append_at(_with_axes(3), 0, _cache(), _batch(), at, GOOD, KV, KV, GOOD, stream=0))


def test_good_positions_reach_the_library():
    _reaches_the_library(lambda: M.mot_paged_append_at(_with_axes(3), 0, _cache(), _batch(), T(3, 3, **I32), GOOD, KV, KV, GOOD,
                                                       stream=0))


def test_the_axes_are_one_for_each_pair():
    h = _handle()
    h.paged.rot_dim = 16
    for axis, rates in (([0] * 7, None), ([0] * 9, None), ([0] * 8, [1.0] * 7)):
        _refused("8 pairs are rotated", lambda: M.mot_paged_set_axes(h, 1, axis, rates))
    _reaches_the_library(lambda: M.mot_paged_set_axes(h, 1, [0] * 8, [1.0] * 8))
