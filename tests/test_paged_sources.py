"""What no run shows reliably in the paged cache's kernels, read from the sources: decisions that a
whole CTA has to take alike, and the order of its writes to shared memory."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_28979_gb300", "csrc")


def _source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def _body(src, name):
    """The braces of the function that is defined as `name`(."""
    for m in re.finditer(r"\b%s\(" % name, src):
        i, depth = m.end(), 1
        while depth:
            depth += {"(": 1, ")": -1}.get(src[i], 0)
            i += 1
        rest = src[i:].lstrip()
        if not rest.startswith("{"):
            continue
        at = src.index("{", i)
        depth, i = 1, at + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(src[i], 0)
            i += 1
        return src[at:i]
    raise AssertionError(name)


def _kernels(src):
    return {m.group(1): _body(src, m.group(1)) for m in re.finditer(r"\b(paged_\w+_kernel)\(const PagedDims", src)}


def test_a_refusal_that_another_cta_may_set_is_read_by_the_cta_as_one():
    """A kernel of several CTAs that sets the refusal bit also meets it while it is being set: threads
    that read it one by one would disagree, and those that stay would act on a batch that is not checked."""
    src = _source("paged.cu")
    kernels = _kernels(src)
    sets = {name for name, body in kernels.items() if "kStatusPages)" in body}
    assert {"paged_reserve_kernel", "paged_free_kernel", "paged_fork_plan_kernel"} <= sets
    several = {name for name in sets if not re.search(r"launch_kernel\(\w+, %s, 1, " % name, src)}
    assert several == {"paged_free_kernel"}
    for name in several:
        reads = re.findall(r"[^;{}]*\brefused\([^;]*;", kernels[name])
        assert len(reads) == 1 and "if (__syncthreads_or(refused(w.status))) return;" in reads[0], (name, reads)


def test_a_share_is_cleared_before_another_thread_may_set_it():
    """Thread 0 clears st.work, the thread of the entry that the share lies in sets it: in both ways of
    dealing the work (by one warp, by the CTA) a barrier that orders memory stands between."""
    body = _body(_source("paged_common.cuh"), "paged_begin")
    cleared, found = body.index("st.work = 0;"), body.index("st.work = 1;")
    between = body[cleared:found]
    dealt = between[:between.index("shfl")]   # before anything that the warp does together
    assert "by_warp" in dealt and "__syncwarp();" in dealt and "__syncthreads();" in dealt


def test_the_status_word_is_cleared_before_its_reader_returns():
    """A fill of device memory, or a small copy from ordinary host memory, may still be under way when its
    call returns, and a kernel on a stream that does not wait for the default one would meet the old word
    (a refused change holds the changes behind it back) or lose what it writes. So the word is changed on
    the call's stream, and that is waited for."""
    src = _source("mot_api.cu")
    body = _body(src, "mot_get_device_status")
    assert not re.search(r"\bcuda(Memset|Memcpy)\(", body)
    changed = [m.end() for m in re.finditer(r"Async\(h->status", body)]
    assert changed and "cudaStreamSynchronize(st)" in body[changed[-1]:body.index("return MOT_ERR_TIMEOUT")]
    assert body.index("cudaSetDevice(h->device)") < body.index("Async(")


def test_a_short_wait_limit_leaves_time_for_copies_in_flight():
    """The limit of the waits bounds what drains copies and products behind a timeout too: a limit of a few
    cycles would let a CTA leave, and the next one start in its shared memory, with copies still to land."""
    body = _body(_source("mot_api.cu"), "mot_debug_set")
    least = int(re.search(r"kLeastWait = (\d+);", _source("mot_api.cu")).group(1))
    assert "std::max<int64_t>(wait_limit_cycles, kLeastWait)" in body and least >= 1_000_000
