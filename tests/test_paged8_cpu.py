"""The paged cache in 8 bits without a GPU: bad configs and NULL handles are refused before any CUDA call, and what
the Python calls refuse before the library sees it."""
import ctypes

import pytest

from paper_2607_28979_gb300 import build as mot_build

mot_build.build()
import paper_2607_28979_gb300.mot as M   # noqa: E402
from test_paged_binding_cpu import GOOD, HQ, H, D, L, N, P, S, T, W, _batch, _reaches_the_library, _refused   # noqa: E402
from test_paged_cpu import GOOD as CONFIG   # noqa: E402

I32, F32, F8 = dict(dtype="torch.int32"), dict(dtype="torch.float32"), dict(dtype="torch.float8_e4m3fn")
ROWS = T(3, H, D)


def _handle():
    h = M.Handle(None, 0)   # the library refuses it: nothing is launched
    h.paged, h.bits8, h.device = M.make_paged_config(L, HQ, H, D, P, N, S, W), True, 0
    return h


def _cache(**change):
    a = dict(k=T(L, N, H, P, D, **F8), v=T(L, N, H, P, D, **F8), table=T(S, W, **I32), lens=T(S, **I32), refs=T(N, **I32),
             k_scale=T(L, N, H, **F32), v_scale=T(L, N, H, **F32))
    a.update(change)
    return M.paged_cache(**a)


@pytest.mark.parametrize("change, expect", [
    (dict(dtype="fp32"), "MOT_ERR_UNSUPPORTED"), (dict(kv_heads=5), "MOT_ERR_INVALID_ARG"),
    (dict(page=8), "MOT_ERR_UNSUPPORTED"), (dict(head_dim=96, rot_dim=96), "MOT_ERR_UNSUPPORTED"),
    (dict(n_pages=0), "MOT_ERR_INVALID_ARG"), (dict(max_seqs=32769), "MOT_ERR_UNSUPPORTED"),
])
def test_create_refuses_bad_configs_before_cuda(change, expect):
    cfg = M.make_paged_config(**dict(CONFIG, **change))
    out = ctypes.c_void_p(1)
    assert M._lib.mot_create_paged8(ctypes.byref(cfg), ctypes.byref(out)) == getattr(M, expect)
    assert not out.value


def test_null_arguments():
    assert M._lib.mot_create_paged8(None, None) == M.MOT_ERR_INVALID_ARG
    assert M._lib.mot_create_paged8(None, ctypes.byref(ctypes.c_void_p())) == M.MOT_ERR_INVALID_ARG


def _calls():
    one = T(1, **I32)
    return (lambda c: M.mot_paged_attention(_handle(), 0, c, _batch(), GOOD, GOOD, stream=0),
            lambda c: M.mot_paged_append(_handle(), 0, c, _batch(), GOOD, ROWS, ROWS, GOOD, stream=0),
            lambda c: M.mot_paged_free(_handle(), c, one, 1, stream=0),
            lambda c: M.mot_paged_fork(_handle(), c, one, one, 1, stream=0),
            lambda c: M.mot_paged_compact(_handle(), c, stream=0),
            lambda c: M.mot_paged_reserve(_handle(), c, _batch(), stream=0),
            lambda c: M.mot_paged_store(_handle(), c, one, 1, T(L, 1, H, 9, D), T(L, 1, H, 9, D), stream=0),
            lambda c: M.mot_paged_load(_handle(), c, one, 1, T(L, 1, H, 9, D), T(L, 1, H, 9, D), stream=0))


@pytest.mark.parametrize("match, change", [
    ("k is of type torch.bfloat16", dict(k=T(L, N, H, P, D))),
    ("v is of type torch.float32", dict(v=T(L, N, H, P, D, **F32))),
    (r"v is \(2, 100, 2, 32, 128\)", dict(v=T(L, N, H, 32, D, **F8))),
    ("k_scale is of type torch.bfloat16", dict(k_scale=T(L, N, H))),
    ("v_scale has 396 elements, 400", dict(v_scale=T(L, N - 1, H, **F32))),
    ("v_scale is not contiguous", dict(v_scale=T(L, N, H, stride=(2 * N * H, H, 1), **F32))),
    ("k_scale is on another device", dict(k_scale=T(L, N, H, device=1, **F32))),
    ("k_scale is not a CUDA tensor", dict(k_scale=T(L, N, H, is_cuda=False, **F32))),
])
def test_caches_of_another_form(match, change):
    for call in _calls():
        _refused(match, lambda: call(_cache(**change)))
        _reaches_the_library(lambda: call(_cache()))


def test_bytes_stand_for_the_values():
    raw = T(L, N, H, P, D, dtype="torch.uint8")
    for call in _calls():
        _reaches_the_library(lambda: call(_cache(k=raw, v=raw)))


def test_a_cache_of_16_bits_takes_no_8_bit_pools():
    h = M.Handle(None, 0)
    h.paged, h.device = M.make_paged_config(L, HQ, H, D, P, N, S, W), 0
    _refused("k is of type torch.float8_e4m3fn", lambda: M.mot_paged_free(h, _cache(), T(1, **I32), 1, stream=0))
