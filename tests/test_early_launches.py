"""Kernels that begin a call and may start before the kernel in front of them has finished: every thread waits for it
first, read from the sources. Before the wait they touch their own shared memory alone; one that lets the next kernel
start early as well does so behind its tensor memory, which that one could otherwise take and hold."""
import glob
import os
import re

import pytest

from test_overlapped_launches import CSRC, _kernels

FILES = sorted(os.path.basename(path) for path in glob.glob(os.path.join(CSRC, "*.cu"))
               if re.search(r"launch_kernel\(\w\.early", open(path).read()))


def test_the_files():
    assert FILES == ["paged8.cu", "paged8_decode.cu", "paged8_fmha.cu", "paged_append.cu"]


def _of(name):
    src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    return {k: v for k, v in _kernels().items() if re.search(r"\b%s\(" % k, src) and "__global__" in src}, src


@pytest.mark.parametrize("name", FILES)
def test_every_thread_waits_first(name):
    kernels, src = _of(name)
    assert kernels and all(x.startswith(("launch_kernel(a.early", "launch_kernel(p.early"))
                           for x in re.findall(r"launch_kernel\([^,]*", src))
    for kernel, body in kernels.items():
        wait = body.find("\n  pdl_wait();")   # in the kernel's outermost block
        assert wait >= 0 and body.count("pdl_wait();") == 1, kernel
        head = body[:wait]
        assert not re.search(r"\breturn\b", head), kernel
        # no pointer of the call is followed, no other kernel's data read
        assert not re.search(r"\ba\.(q|out|k|v|ks|vs|table|lens|status|part|count|b)\b|\b[cpw]\.\w+|\bax\.|refused|tmem_alloc",
                             head), kernel
        trigger = body.find("pdl_trigger();")
        if trigger >= 0:
            between = body[body.find("tmem_alloc("):trigger]
            assert wait < body.find("tmem_alloc(") < trigger and "__syncthreads();" in between, kernel
