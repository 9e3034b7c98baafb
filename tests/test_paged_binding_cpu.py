"""What the Python calls of the paged cache refuse before the library sees it: tensors that are not on the
GPU, not contiguous, of another type or shorter than the call reads, and caches of another handle's form."""
import pytest

from paper_2607_28979_gb300 import build as mot_build

mot_build.build()
import paper_2607_28979_gb300.mot as M   # noqa: E402


class T:
    """Stands for a CUDA tensor: shape, strides, type and device."""

    def __init__(self, *shape, dtype="torch.bfloat16", stride=None, device=0, is_cuda=True):
        dense = [1]
        for n in reversed(shape[1:]):
            dense.insert(0, dense[0] * n)
        self.shape, self._stride, self.dtype = shape, tuple(stride or dense), dtype
        self.is_cuda, self._device, self._dense = is_cuda, device, tuple(dense)

    def stride(self):
        return self._stride

    def dim(self):
        return len(self.shape)

    def size(self, i):
        return self.shape[i]

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def is_contiguous(self):
        return self._stride == self._dense

    def get_device(self):
        return self._device

    def data_ptr(self):
        return 4096


I32 = dict(dtype="torch.int32")
L, HQ, H, D, P, N, S, W = 2, 12, 2, 128, 64, 100, 8, 32


def _handle(dtype="bf16"):
    h = M.Handle(None, 0)   # the library refuses it: nothing is launched
    h.paged, h.device = M.make_paged_config(L, HQ, H, D, P, N, S, W, dtype=dtype), 0
    return h


def _cache(**change):
    a = dict(k=T(L, N, H, P, D), v=T(L, N, H, P, D), table=T(S, W, **I32), lens=T(S, **I32), refs=T(N, **I32))
    a.update(change)
    return M.paged_cache(**a)


def _batch(rows=3, seqs=None, starts=None, n=2):
    return M.paged_batch(seqs or T(2, **I32), starts or T(3, **I32), n, rows)


def _refused(match, call):
    with pytest.raises(M.MotError, match=match) as e:
        call()
    assert e.value.status == M.MOT_ERR_INVALID_ARG


def _reaches_the_library(call):
    with pytest.raises(M.MotError, match=r"^mot_paged_\w+: MOT_ERR_INVALID_ARG$"):
        call()


GOOD = T(3, HQ, D)


@pytest.mark.parametrize("match, q, out", [
    ("q is not contiguous", T(3, HQ, D, stride=((HQ + 2 * H) * D, D, 1)), GOOD),   # a slice of a fused projection
    ("out is not contiguous", GOOD, T(3, HQ, D, stride=(D, 3 * D, 1))),
    ("q is of type torch.float32", T(3, HQ, D, dtype="torch.float32"), GOOD),
    ("out is of type torch.float16", GOOD, T(3, HQ, D, dtype="torch.float16")),
    ("q is not a CUDA tensor", T(3, HQ, D, is_cuda=False), GOOD),
    ("q is on another device", T(3, HQ, D, device=1), GOOD),
    ("q has 1536 elements, 4608", T(1, HQ, D), GOOD),
    ("out has 2304 elements, 4608", GOOD, T(3, HQ, D // 2)),
])
def test_attention_tensors(match, q, out):
    _refused(match, lambda: M.mot_paged_attention(_handle(), 0, _cache(), _batch(), q, out, stream=0))


def test_attention_takes_what_it_reads():
    for q in (GOOD, T(5, HQ, D), T(3, HQ, D, dtype="torch.int16"), 4096, None):
        _reaches_the_library(lambda: M.mot_paged_attention(_handle(), 0, _cache(), _batch(), q, GOOD, stream=0))
    f = T(3, HQ, D, dtype="torch.float32")
    pools = dict(k=T(L, N, H, P, D, dtype="torch.float32"), v=T(L, N, H, P, D, dtype="torch.float32"))
    _reaches_the_library(lambda: M.mot_paged_attention(_handle("fp32"), 0, _cache(**pools), _batch(), f, f, stream=0))
    _reaches_the_library(lambda: M.mot_paged_attention(M.Handle(None, 0), 0, _cache(), _batch(), GOOD, GOOD, stream=0))


@pytest.mark.parametrize("match, change", [
    ("k is not contiguous", dict(k=T(L, N, H, P, D, stride=(N * H * P * D * 2, H * P * D, P * D, D, 1)))),
    ("v is not a CUDA tensor", dict(v=T(L, N, H, P, D, is_cuda=False))),
    ("v is of type torch.float32", dict(v=T(L, N, H, P, D, dtype="torch.float32"))),
    (r"k is \(2, 100, 2, 32, 128\)", dict(k=T(L, N, H, 32, D))),
    (r"k is \(2, 50, 2, 64, 128\)", dict(k=T(L, 50, H, P, D))),
    (r"v is \(1, 100, 2, 64, 128\)", dict(v=T(1, N, H, P, D))),
    ("table is of type torch.int64", dict(table=T(S, W, dtype="torch.int64"))),
    (r"table is \(8, 64\)", dict(table=T(S, 2 * W, **I32))),
    ("table has 224 elements, 256", dict(table=T(S - 1, W, **I32))),
    ("lens has 7 elements, 8", dict(lens=T(S - 1, **I32))),
    ("refs has 99 elements, 100", dict(refs=T(N - 1, **I32))),
    ("lens is on another device", dict(lens=T(S, device=1, **I32))),
])
def test_caches_of_another_form(match, change):
    calls = (lambda h, c: M.mot_paged_attention(h, 0, c, _batch(), GOOD, GOOD, stream=0),
             lambda h, c: M.mot_paged_reserve(h, c, _batch(), stream=0),
             lambda h, c: M.mot_paged_fork(h, c, T(1, **I32), T(1, **I32), 1, stream=0),
             lambda h, c: M.mot_paged_free(h, c, T(1, **I32), 1, stream=0),
             lambda h, c: M.mot_paged_compact(h, c, stream=0),
             lambda h, c: M.mot_paged_store(h, c, T(1, **I32), 1, T(L, 1, H, 9, D), T(L, 1, H, 9, D), stream=0),
             lambda h, c: M.mot_paged_load(h, c, T(1, **I32), 1, T(L, 1, H, 9, D), T(L, 1, H, 9, D), stream=0),
             lambda h, c: M.mot_paged_append(h, 0, c, _batch(), GOOD, T(3, H, D), T(3, H, D), GOOD, stream=0))
    for call in calls:
        _refused(match, lambda: call(_handle(), _cache(**change)))
        _reaches_the_library(lambda: call(_handle(), _cache()))


@pytest.mark.parametrize("match, batch", [
    ("seqs has 1 elements, 2", lambda: _batch(seqs=T(1, **I32))),
    ("starts has 2 elements, 3", lambda: _batch(starts=T(2, **I32))),
    ("starts is of type torch.int64", lambda: _batch(starts=T(3, dtype="torch.int64"))),
    ("seqs is not contiguous", lambda: _batch(seqs=T(2, stride=(2,), **I32))),
])
def test_batches(match, batch):
    _refused(match, lambda: M.mot_paged_reserve(_handle(), _cache(), batch(), stream=0))


def test_slots_and_counts():
    h, c = _handle(), _cache()
    _refused("src has 1 elements, 2", lambda: M.mot_paged_fork(h, c, T(1, **I32), T(2, **I32), 2, stream=0))
    _refused("dst is of type", lambda: M.mot_paged_fork(h, c, T(1, **I32), T(1, dtype="torch.int64"), 1, stream=0))
    _refused("seqs has 1 elements, 3", lambda: M.mot_paged_free(h, c, T(1, **I32), 3, stream=0))
    _refused("live is of type", lambda: M.mot_paged_compact(h, c, T(1, dtype="torch.int64"), stream=0))


@pytest.mark.parametrize("match, k, v", [
    ("4 heads of 64", T(L, 1, 4, 9, 64), T(L, 1, 4, 9, 64)),
    ("2 heads of 64", T(L, 1, H, 9, 64), T(L, 1, H, 9, 64)),
    ("K is of type torch.float32", T(L, 1, H, 9, D, dtype="torch.float32"), T(L, 1, H, 9, D, dtype="torch.float32")),
    ("V is not a CUDA tensor", T(L, 1, H, 9, D), T(L, 1, H, 9, D, is_cuda=False)),
])
def test_contiguous_caches(match, k, v):
    for call in (M.mot_paged_store, M.mot_paged_load):
        _refused(match, lambda: call(_handle(), _cache(), T(1, **I32), 1, k, v, stream=0))
        _refused("seqs has 1 elements, 2", lambda: call(_handle(), _cache(), T(1, **I32), 2, T(L, 2, H, 9, D),
                                                        T(L, 2, H, 9, D), stream=0))


ROW = (HQ + 2 * H) * D   # of a fused projection


@pytest.mark.parametrize("match, change", [
    (r"q is \(3, 14, 128\)", dict(q=T(3, 14, D))),
    (r"k is \(3, 2, 64\)", dict(k=T(3, H, 64))),
    (r"v is \(2, 2, 128\)", dict(v=T(2, H, D))),
    ("k is of type torch.float32", dict(k=T(3, H, D, dtype="torch.float32"))),
    ("q_out is not contiguous", dict(q_out=T(3, HQ, D, stride=(ROW, D, 1)))),
    ("q_out has 1536 elements", dict(q_out=T(1, HQ, D))),
    ("q_norm has 64 elements", dict(q_norm=T(64))),
    ("k_norm is of type torch.float32", dict(k_norm=T(D, dtype="torch.float32"))),
])
def test_append_tensors(match, change):
    a = dict(q=T(3, HQ, D, stride=(ROW, D, 1)), k=T(3, H, D, stride=(ROW, D, 1)), v=T(3, H, D, stride=(ROW, D, 1)),
             q_out=T(3, HQ, D), q_norm=T(D), k_norm=None)
    _reaches_the_library(lambda: M.mot_paged_append(_handle(), 0, _cache(), _batch(), stream=0, **a))
    a.update(change)
    _refused(match, lambda: M.mot_paged_append(_handle(), 0, _cache(), _batch(), stream=0, **a))


def test_row_strides():
    """One row's stride, and one head's, say nothing; what does is checked."""
    assert M._row_stride(T(3, HQ, D, stride=(ROW, D, 1)), "q") == ROW
    assert M._row_stride(T(1, HQ, D, stride=(ROW + 4, D, 1)), "q") == HQ * D
    assert M._row_stride(T(3, 1, D, stride=(D, 3 * D, 1)), "k") == D   # [1][rows][d] with its first two swapped
    for bad in (T(3, HQ, D, stride=(D, 3 * D, 1)), T(3, HQ, D, stride=(2 * HQ * D, 2 * D, 2)), T(3, HQ * D)):
        with pytest.raises(ValueError):
            M._row_stride(bad, "q")
