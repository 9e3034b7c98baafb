"""The paged cache's entry points without a GPU: bad configs and NULL handles are refused before any
CUDA call; the kernels that start under their predecessor, read from the sources."""
import ctypes
import os
import re

import pytest

from paper_2607_28979_gb300 import build as mot_build

mot_build.build()
import paper_2607_28979_gb300.mot as M   # noqa: E402

GOOD = dict(n_layers=2, q_heads=12, kv_heads=2, head_dim=128, page=64, n_pages=100, max_seqs=8, max_pages=32,
            rot_dim=128, rot_base=1e6, norm_eps=1e-6)


@pytest.mark.parametrize("change, expect", [
    *[({k: 0}, "MOT_ERR_INVALID_ARG") for k in ("n_layers", "q_heads", "kv_heads", "head_dim", "page", "n_pages",
                                               "max_seqs", "max_pages")],
    (dict(n_pages=-4), "MOT_ERR_INVALID_ARG"),
    (dict(kv_heads=5), "MOT_ERR_INVALID_ARG"),              # 12 heads on 5
    (dict(rot_dim=-16), "MOT_ERR_INVALID_ARG"),
    (dict(rot_dim=144), "MOT_ERR_INVALID_ARG"),             # more than a head has
    (dict(rot_base=0.5), "MOT_ERR_INVALID_ARG"),
    (dict(rot_base=float("nan")), "MOT_ERR_INVALID_ARG"),
    (dict(rot_base=float("inf")), "MOT_ERR_INVALID_ARG"),
    (dict(norm_eps=-1.0), "MOT_ERR_INVALID_ARG"),
    (dict(norm_eps=float("nan")), "MOT_ERR_INVALID_ARG"),
    (dict(head_dim=96, rot_dim=96), "MOT_ERR_UNSUPPORTED"),
    (dict(page=8), "MOT_ERR_UNSUPPORTED"),
    (dict(page=48), "MOT_ERR_UNSUPPORTED"),
    (dict(page=256), "MOT_ERR_UNSUPPORTED"),
    (dict(q_heads=34, kv_heads=2), "MOT_ERR_UNSUPPORTED"),  # 17 heads share one
    (dict(rot_dim=24), "MOT_ERR_UNSUPPORTED"),
    (dict(max_seqs=32769), "MOT_ERR_UNSUPPORTED"),
    (dict(n_pages=(1 << 30) // 128 + 1), "MOT_ERR_UNSUPPORTED"),
])
def test_create_refuses_bad_configs_before_cuda(change, expect):
    cfg = M.make_paged_config(**dict(GOOD, **change))
    out = ctypes.c_void_p(1)
    assert M._lib.mot_create_paged(ctypes.byref(cfg), ctypes.byref(out)) == getattr(M, expect)
    assert not out.value


@pytest.mark.parametrize("field, value", [("dtype", 2), ("rot_pairs", 2), ("rot_pairs", -1)])
def test_create_refuses_bad_choices(field, value):
    cfg = M.make_paged_config(**GOOD)
    setattr(cfg, field, value)
    out = ctypes.c_void_p(1)
    assert M._lib.mot_create_paged(ctypes.byref(cfg), ctypes.byref(out)) == M.MOT_ERR_INVALID_ARG


def test_a_good_config_without_a_gpu_is_a_cuda_error():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(M.MotError) as e:
        M.mot_create_paged(M.make_paged_config(**GOOD))
    assert e.value.status == M.MOT_ERR_CUDA


def test_null_handles_and_arguments():
    L, bad = M._lib, M.MOT_ERR_INVALID_ARG
    c, b = M.paged_cache(64, 128, 64, 64, 64), M.paged_batch(64, 64, 1, 1)
    c, b = ctypes.byref(c), ctypes.byref(b)
    assert L.mot_create_paged(None, None) == bad
    assert L.mot_create_paged(None, ctypes.byref(ctypes.c_void_p())) == bad
    assert L.mot_paged_reserve(None, c, b, None) == bad
    assert L.mot_paged_fork(None, c, 64, 64, 1, None) == bad
    assert L.mot_paged_free(None, c, 64, 1, None) == bad
    assert L.mot_paged_compact(None, c, None, None) == bad
    assert L.mot_paged_store(None, c, 0, 1, 64, 1, 1, 1, 64, 64, None) == bad
    assert L.mot_paged_load(None, c, 0, 1, 64, 1, 1, 1, 64, 64, None) == bad
    assert L.mot_paged_append(None, 0, c, b, 64, 64, 64, 64, 64, 64, None, None, 64, None) == bad
    assert L.mot_paged_attention(None, 0, c, b, 64, 64, None) == bad
    assert M.mot_status_string(M.MOT_ERR_PAGES) == "MOT_ERR_PAGES"


def test_overlapped_kernels_wait_before_they_read_or_leave():
    """The second kernels of a fork and of a compaction start while the plan before them runs: each
    waits for it first of all."""
    src = open(os.path.join(os.path.dirname(mot_build.__file__), "csrc", "paged.cu")).read()
    names = re.findall(r"launch_kernel\(overlap, (\w+)", src)
    assert sorted(names) == ["paged_compact_kernel", "paged_fork_kernel"]
    for name in names:
        body = src[src.index("{", src.index(name + "(")):]
        assert body[1:].lstrip().startswith("pdl_enter();"), name
