"""Python binding of ``libmot.so``: argument marshalling only.

Every step of the translation runs in the CUDA library (``csrc/``). This
module loads it with ctypes and exposes its C entry points under the same
names. There is no CPU fallback: if the library is missing, importing this
package raises ``ImportError`` (build it with ``python -m
paper_2607_28979_gb300.build`` or ``__graft_entry__.build()``).

Tensor arguments may be ``torch.Tensor`` objects (their ``data_ptr()`` is
passed) or plain integers holding device / host addresses. Streams may be a
``torch.cuda.Stream``, an integer handle, or ``None`` (the current torch
stream if torch is loaded, else the legacy default stream).
"""
from __future__ import annotations

import ctypes
import os
import sys
from typing import Optional, Sequence

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmot.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"libmot.so is not built ({LIB_PATH}); run "
                      "`python -m paper_2607_28979_gb300.build` first")

_lib = ctypes.CDLL(LIB_PATH)

# ---------------------------------------------------------------- C types

MOT_OK, MOT_ERR_INVALID_ARG, MOT_ERR_UNSUPPORTED, MOT_ERR_NO_WEIGHTS, MOT_ERR_WEIGHTS_SIZE, \
    MOT_ERR_OOM, MOT_ERR_CUDA, MOT_ERR_SEQ_LEN, MOT_ERR_TIMEOUT, MOT_ERR_PAGES = range(10)
MOT_BF16, MOT_FP32 = 0, 1
MOT_PAGES_REFUSED, MOT_PAGES_HELD = 1, 2


class mot_config(ctypes.Structure):
    _fields_ = [("n_layers_src", ctypes.c_int32), ("src_kv_heads", ctypes.c_int32),
                ("src_head_dim", ctypes.c_int32), ("n_layers_tgt", ctypes.c_int32),
                ("tgt_kv_heads", ctypes.c_int32), ("tgt_head_dim", ctypes.c_int32),
                ("n_translators", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("max_batch", ctypes.c_int32),
                ("max_seq", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("layer_map", ctypes.POINTER(ctypes.c_int32))]


class mot_h_config(ctypes.Structure):
    _fields_ = [("n_layers_src", ctypes.c_int32), ("src_act_dim", ctypes.c_int32),
                ("n_layers_tgt", ctypes.c_int32), ("tgt_act_dim", ctypes.c_int32),
                ("tgt_kv_heads", ctypes.c_int32), ("tgt_head_dim", ctypes.c_int32),
                ("n_translators", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("max_batch", ctypes.c_int32),
                ("max_seq", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("layer_map", ctypes.POINTER(ctypes.c_int32))]


class mot_bt_config(ctypes.Structure):
    _fields_ = [("win_start", ctypes.c_int32), ("win_len", ctypes.c_int32),
                ("width", ctypes.c_int32), ("heads", ctypes.c_int32), ("ffn", ctypes.c_int32)]


class mot_replay_config(ctypes.Structure):
    _fields_ = [("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("max_batch", ctypes.c_int32),
                ("max_seq", ctypes.c_int32), ("top_s", ctypes.c_int32), ("n_full", ctypes.c_int32)]


class mot_paged_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("max_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("rot_pairs", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("norm_eps", ctypes.c_float),
                ("rot_base", ctypes.c_double)]


class mot_paged_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class mot_paged_batch(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_void_p), ("starts", ctypes.c_void_p), ("n", ctypes.c_int32),
                ("rows", ctypes.c_int32), ("max_chunk", ctypes.c_int32)]


class mot_kernel_stat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int64),
                ("total_ms", ctypes.c_double)]


_H = ctypes.c_void_p
_P = ctypes.c_void_p
_S = ctypes.c_int
_I = ctypes.c_int32
_CACHE, _BATCH = ctypes.POINTER(mot_paged_cache), ctypes.POINTER(mot_paged_batch)

_SIGS = {
    "mot_create": [ctypes.POINTER(mot_config), ctypes.POINTER(ctypes.c_void_p)],
    "mot_load_weights": [_H, _P, ctypes.c_size_t],
    "mot_translate": [_H, _P, _P, _P, ctypes.c_int32, _P, _P, _P],
    "mot_translate_host": [_H, _P, _P, _P, ctypes.c_int32, _P, _P, _P],
    "mot_get_device_status": [_H, _P],
    "mot_destroy": [_H],
    "mot_get_layer_map": [_H, _P, ctypes.c_int32],
    "mot_get_path": [_H, ctypes.POINTER(ctypes.c_int32)],
    "mot_set_schedule": [_H, ctypes.c_int32],
    "mot_get_schedule": [_H, ctypes.POINTER(ctypes.c_int32)],
    "mot_profile_enable": [_H, ctypes.c_int32],
    "mot_profile_read": [_H, ctypes.POINTER(mot_kernel_stat), ctypes.c_int32,
                         ctypes.POINTER(ctypes.c_int32)],
    "mot_get_launch_count": [_H, ctypes.POINTER(ctypes.c_int64)],
    "mot_create_h": [ctypes.POINTER(mot_h_config), ctypes.POINTER(ctypes.c_void_p)],
    "mot_translate_h": [_H, _P, _P, ctypes.c_int32, _P, _P, _P],
    "mot_set_routing": [_H, ctypes.c_int32],
    "mot_get_routing": [_H, ctypes.POINTER(ctypes.c_int32)],
    "mot_get_expert_counts": [_H, _P, ctypes.c_int32, _P],
    "mot_expert_usage": [_P, ctypes.c_int32, _P, _P],
    "mot_debug_set": [_H, ctypes.c_int32, ctypes.c_int64],
    "mot_debug_gelu": [ctypes.c_int32, _P, _P, ctypes.c_int64, _P, _P],
    "mot_debug_fixed_gate": [_H, _P],
    "mot_translate_static": [ctypes.POINTER(mot_config), _P, _P, _P, _P, ctypes.c_int32, _P, _P,
                             _P],
    "mot_create_bt": [ctypes.POINTER(mot_config), ctypes.POINTER(mot_bt_config),
                      ctypes.POINTER(ctypes.c_void_p)],
    "mot_translate_bt": [_H, _P, _P, _P, ctypes.c_int32, _P, _P, _P],
    "mot_create_replay": [ctypes.POINTER(mot_replay_config), ctypes.POINTER(ctypes.c_void_p)],
    "mot_replay_attention": [_H, ctypes.c_int32, _P, _P, _P, _P, _P, ctypes.c_int32, _P, _P],
    "mot_replay_select": [_H, _P, _P, ctypes.c_int32, _P, _P],
    "mot_create_paged": [ctypes.POINTER(mot_paged_config), ctypes.POINTER(ctypes.c_void_p)],
    "mot_create_paged8": [ctypes.POINTER(mot_paged_config), ctypes.POINTER(ctypes.c_void_p)],
    "mot_paged_cause": [_H, ctypes.POINTER(ctypes.c_int32)],
    "mot_paged_reserve": [_H, _CACHE, _BATCH, _P],
    "mot_paged_fork": [_H, _CACHE, _P, _P, _I, _P],
    "mot_paged_free": [_H, _CACHE, _P, _I, _P],
    "mot_paged_compact": [_H, _CACHE, _P, _P],
    "mot_paged_store": [_H, _CACHE, _I, _I, _P, _I, _I, _I, _P, _P, _P],
    "mot_paged_load": [_H, _CACHE, _I, _I, _P, _I, _I, _I, _P, _P, _P],
    "mot_paged_append": [_H, _I, _CACHE, _BATCH, _P, ctypes.c_int64, _P, ctypes.c_int64, _P,
                         ctypes.c_int64, _P, _P, _P, _P],
    "mot_paged_set_axes": [_H, _I, _P, _P],
    "mot_paged_append_at": [_H, _I, _CACHE, _BATCH, _P, _P, ctypes.c_int64, _P, ctypes.c_int64, _P,
                         ctypes.c_int64, _P, _P, _P, _P],
    "mot_paged_attention": [_H, _I, _CACHE, _BATCH, _P, _P, _P],
}
for _name, _args in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = _S
_calls = {_name: getattr(_lib, _name) for _name in _SIGS}
_lib.mot_status_string.argtypes = [_S]
_lib.mot_status_string.restype = ctypes.c_char_p

# Names declared by include/mot.h, for the export check.
EXPORTED = sorted(list(_SIGS) + ["mot_status_string"])


class MotError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {mot_status_string(status)}")


def mot_status_string(status: int) -> str:
    return _lib.mot_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != MOT_OK:
        raise MotError(status, where)


def _addr(x) -> Optional[int]:
    if x is None or isinstance(x, int):
        return x
    at = getattr(x, "data_ptr", None)
    if at is not None:
        return at()
    if hasattr(x, "ctypes"):   # numpy array (host buffers)
        return x.ctypes.data
    raise TypeError(f"cannot take the address of {type(x)}")


_raw_stream = _get_device = None   # torch's, once CUDA is initialised: 0.4 us together, the Stream object 2.8


def _stream(s) -> Optional[int]:
    global _raw_stream, _get_device
    if s is None:
        if _raw_stream is not None:
            return _raw_stream(_get_device())
        torch = sys.modules.get("torch")
        if torch is not None and torch.cuda.is_initialized():
            raw, dev = (getattr(torch._C, x, None) for x in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
            if raw is not None and dev is not None:
                _raw_stream, _get_device = raw, dev
                return raw(dev())
            return torch.cuda.current_stream().cuda_stream
        return None
    if isinstance(s, int):
        return s
    return s.cuda_stream


# ---------------------------------------------------------------- entry points

class Handle:
    """Owns one ``mot_handle``; destroyed with ``mot_destroy`` or on GC."""

    paged = None    # the config of a paged handle
    bits8 = False   # its pages are in 8 bits
    axes = 0        # positions of a row, once its axes are set
    device = None   # its device, where torch had one when it was made

    def __init__(self, ptr: int, n_layers_tgt: int):
        self.ptr = ptr
        self.n_layers_tgt = n_layers_tgt

    def __del__(self):
        if getattr(self, "ptr", None):
            try:
                _lib.mot_destroy(self.ptr)
            except Exception:
                pass
            self.ptr = None


def make_config(n_layers_src, src_kv_heads, src_head_dim, n_layers_tgt, tgt_kv_heads,
                tgt_head_dim, n_translators, hidden, max_batch, max_seq, dtype="bf16", top_k=0,
                layer_map: Optional[Sequence[int]] = None):
    cfg = mot_config(n_layers_src, src_kv_heads, src_head_dim, n_layers_tgt, tgt_kv_heads,
                     tgt_head_dim, n_translators, top_k, hidden, max_batch, max_seq,
                     MOT_BF16 if dtype in ("bf16", MOT_BF16) else MOT_FP32, None)
    keep = None
    if layer_map is not None:
        keep = (ctypes.c_int32 * len(layer_map))(*layer_map)
        cfg.layer_map = ctypes.cast(keep, ctypes.POINTER(ctypes.c_int32))
    cfg._keep = keep   # keep the array alive as long as the struct
    return cfg


def config_from(wl):
    """mot_config for any object with the Workload field names."""
    return make_config(wl.n_layers_src, wl.src_kv_heads, wl.src_head_dim, wl.n_layers_tgt,
                       wl.tgt_kv_heads, wl.tgt_head_dim, wl.n_translators, wl.hidden,
                       wl.max_batch, wl.max_seq, wl.dtype, wl.top_k, wl.layer_map)


def h_config_from(wl):
    """mot_h_config (MoT-h) for a Workload with ``act_tgt`` > 0 (the source
    activation stored as a one-head cache of width ``src_head_dim``)."""
    cfg = mot_h_config(wl.n_layers_src, wl.src_head_dim, wl.n_layers_tgt, wl.act_tgt,
                       wl.tgt_kv_heads, wl.tgt_head_dim, wl.n_translators, wl.top_k, wl.hidden,
                       wl.max_batch, wl.max_seq, MOT_BF16 if wl.dtype == "bf16" else MOT_FP32)
    if wl.layer_map is not None:
        arr = (ctypes.c_int32 * len(wl.layer_map))(*wl.layer_map)
        cfg.layer_map = ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32))
        cfg._keep = arr
    return cfg


def mot_create_h(cfg: mot_h_config) -> Handle:
    out = ctypes.c_void_p()
    _check(_lib.mot_create_h(ctypes.byref(cfg), ctypes.byref(out)), "mot_create_h")
    return Handle(out.value, cfg.n_layers_tgt)


def mot_translate_h(h: Handle, src_act, seq_lens, batch: int, dst_k, dst_v, stream=None) -> None:
    _check(_lib.mot_translate_h(h.ptr, _addr(src_act), _addr(seq_lens), int(batch), _addr(dst_k),
                                _addr(dst_v), _stream(stream)), "mot_translate_h")


def bt_config_from(wl):
    """(mot_config, mot_bt_config) for a Workload with backbone translators (``bt``)."""
    return config_from(wl), mot_bt_config(*wl.bt)


def mot_create_bt(cfg: mot_config, bt: mot_bt_config) -> Handle:
    out = ctypes.c_void_p()
    _check(_lib.mot_create_bt(ctypes.byref(cfg), ctypes.byref(bt), ctypes.byref(out)),
           "mot_create_bt")
    return Handle(out.value, cfg.n_layers_tgt)


def mot_translate_bt(h: Handle, src_k, src_v, seq_lens, batch: int, dst_k, dst_v,
                     stream=None) -> None:
    _check(_lib.mot_translate_bt(h.ptr, _addr(src_k), _addr(src_v), _addr(seq_lens), int(batch),
                                 _addr(dst_k), _addr(dst_v), _stream(stream)), "mot_translate_bt")


def replay_config_from(wl):
    """mot_replay_config for a ``synth.ReplayWorkload``."""
    return mot_replay_config(wl.q_heads, wl.kv_heads, wl.head_dim, wl.max_batch, wl.max_seq,
                             wl.top_s, wl.n_full)


def mot_create_replay(cfg: mot_replay_config) -> Handle:
    out = ctypes.c_void_p()
    _check(_lib.mot_create_replay(ctypes.byref(cfg), ctypes.byref(out)), "mot_create_replay")
    return Handle(out.value, 0)


def mot_replay_attention(h: Handle, layer: int, q, k, v, guide, seq_lens, batch: int, out,
                         stream=None) -> None:
    _check(_lib.mot_replay_attention(h.ptr, int(layer), _addr(q), _addr(k), _addr(v),
                                     _addr(guide), _addr(seq_lens), int(batch), _addr(out),
                                     _stream(stream)), "mot_replay_attention")


def mot_replay_select(h: Handle, guide, seq_lens, batch: int, sel, stream=None) -> None:
    _check(_lib.mot_replay_select(h.ptr, _addr(guide), _addr(seq_lens), int(batch), _addr(sel),
                                  _stream(stream)), "mot_replay_select")


def make_paged_config(n_layers, q_heads, kv_heads, head_dim, page, n_pages, max_seqs, max_pages,
                      rot_dim=0, rot_pairs=False, rot_base=1e4, norm_eps=1e-6, dtype="bf16"):
    return mot_paged_config(n_layers, q_heads, kv_heads, head_dim, page, n_pages, max_seqs,
                            max_pages, rot_dim, int(bool(rot_pairs)),
                            MOT_BF16 if dtype in ("bf16", MOT_BF16) else MOT_FP32, norm_eps, rot_base)


# What the paged calls take as tensors is checked against the handle: contiguous device memory of its type and
# at least its sizes. Addresses (ints) and None go to the library as they are. A set of types holds their names,
# and the types themselves as they come.
_FLOATS = {MOT_BF16: {"torch.bfloat16", "torch.int16", "torch.uint16"},   # the values, or their bits
           MOT_FP32: {"torch.float32"}}
_EIGHT = {"torch.float8_e4m3fn", "torch.uint8", "torch.int8"}
_INT32, _FLOAT32 = {"torch.int32"}, {"torch.float32"}


def _bad(where: str, what: str) -> MotError:
    return MotError(MOT_ERR_INVALID_ARG, f"{where}, {what}")


def _typed(x, kinds, where: str, what: str, dev) -> None:
    """Raises unless x is on the GPU (``dev``, where it is known) and of one of the types."""
    if not getattr(x, "is_cuda", False):
        raise _bad(where, f"{what} is not a CUDA tensor")
    if x.dtype not in kinds:
        if str(x.dtype) not in kinds:
            raise _bad(where, f"{what} is of type {x.dtype}")
        kinds.add(x.dtype)
    if dev is not None and x.get_device() != dev:
        raise _bad(where, f"{what} is on another device than the handle")


def _whole(x, kinds, least: int, where: str, what: str, dev) -> Optional[int]:
    """The address of x: contiguous, ``least`` elements or more."""
    if x is None or isinstance(x, int):
        return x
    _typed(x, kinds, where, what, dev)
    if not x.is_contiguous():
        raise _bad(where, f"{what} is not contiguous")
    if x.numel() < least:
        raise _bad(where, f"{what} has {x.numel()} elements, {least} are read or written")
    return x.data_ptr()


def paged_cache(k, v, table, lens, refs, k_scale=None, v_scale=None) -> mot_paged_cache:
    """The arrays of a paged cache (contiguous device tensors): pools k, v
    [n_layers][n_pages][kv_heads][page][head_dim], int32 table [max_seqs][max_pages], lens
    [max_seqs] and refs [n_pages]; of one in 8 bits (pools of float8_e4m3fn) also the float32 scales
    [n_layers][n_pages][kv_heads]. The struct keeps the tensors; the calls check them."""
    keep = (k, v, table, lens, refs, k_scale, v_scale)
    c = mot_paged_cache(*[_addr(x) for x in keep])
    c._keep = keep
    return c


def paged_batch(seqs, starts, n: int, rows: int, max_chunk: Optional[int] = None) -> mot_paged_batch:
    """n slots (device int32 ``seqs`` [n]) with their new rows (device int32 ``starts`` [n + 1]);
    ``max_chunk``: the most rows of one (``rows`` where it is not known)."""
    b = mot_paged_batch(_addr(seqs), _addr(starts), int(n), int(rows),
                        int(rows if max_chunk is None else max_chunk))
    b._keep = (seqs, starts)
    return b


def mot_create_paged8(cfg: mot_paged_config) -> Handle:
    """mot_create_paged with pages in 8 bits; ``cfg.dtype`` is that of the calls, bf16."""
    h = mot_create_paged(cfg, "mot_create_paged8")
    h.bits8 = True
    return h


def mot_create_paged(cfg: mot_paged_config, _call: str = "mot_create_paged") -> Handle:
    out = ctypes.c_void_p()
    _check(getattr(_lib, _call)(ctypes.byref(cfg), ctypes.byref(out)), _call)
    h = Handle(out.value, 0)
    h.paged = mot_paged_config.from_buffer_copy(cfg)
    torch = sys.modules.get("torch")
    if torch is not None and torch.cuda.is_initialized():
        h.device = torch.cuda.current_device()
    return h


def _fits(h: Handle, cache: mot_paged_cache, where: str) -> Optional[mot_paged_config]:
    """The handle's config (None: no paged handle, which the library refuses); raises where the cache's
    tensors are not those of such a handle. A cache that fitted is not looked at again."""
    cfg = h.paged
    if cfg is None or getattr(cache, "_fitted", None) is cfg:
        return cfg
    keep = getattr(cache, "_keep", None)
    if keep is not None:
        c = cfg
        form = (c.n_pages, c.kv_heads, c.page, c.head_dim)
        for x, what in zip(keep, "kv"):
            _whole(x, _EIGHT if h.bits8 else _FLOATS[c.dtype], 0, where, what, h.device)
            if hasattr(x, "shape") and (tuple(x.shape[1:]) != form or x.shape[0] < c.n_layers):
                raise _bad(where, f"{what} is {tuple(x.shape)}, the handle's pools are {(c.n_layers,) + form}")
        table, lens, refs = keep[2:5]
        if h.bits8:
            for x, what in zip(keep[5:], ("k_scale", "v_scale")):
                _whole(x, _FLOAT32, c.n_layers * c.n_pages * c.kv_heads, where, what, h.device)
        _whole(table, _INT32, c.max_seqs * c.max_pages, where, "table", h.device)
        if hasattr(table, "shape") and table.shape[-1] != c.max_pages and table.dim() > 1:
            raise _bad(where, f"table is {tuple(table.shape)}, the handle's {(c.max_seqs, c.max_pages)}")
        _whole(lens, _INT32, c.max_seqs, where, "lens", h.device)
        _whole(refs, _INT32, c.n_pages, where, "refs", h.device)
    cache._fitted = cfg
    return cfg


def _batch_fits(h: Handle, batch: mot_paged_batch, where: str) -> int:
    """The batch's rows; raises where its tensors are shorter than its n says."""
    keep, n = getattr(batch, "_keep", None), batch.n
    if keep is not None and getattr(batch, "_fitted", None) != n:
        if 0 < n <= h.paged.max_seqs:   # else nothing is read, or the library refuses it
            dev = h.device
            _whole(keep[0], _INT32, n, where, "seqs", dev)
            _whole(keep[1], _INT32, n + 1, where, "starts", dev)
            batch._fitted = n
    return batch.rows


def mot_paged_cause(h: Handle) -> int:
    """MOT_PAGES_REFUSED and / or MOT_PAGES_HELD: what the last mot_get_device_status found."""
    out = ctypes.c_int32()
    _check(_lib.mot_paged_cause(h.ptr, ctypes.byref(out)), "mot_paged_cause")
    return out.value


def mot_paged_reserve(h: Handle, cache: mot_paged_cache, batch: mot_paged_batch, stream=None) -> None:
    where = "mot_paged_reserve"
    if _fits(h, cache, where) is not None:
        _batch_fits(h, batch, where)
    _check(_lib.mot_paged_reserve(h.ptr, ctypes.byref(cache), ctypes.byref(batch), _stream(stream)), where)


def mot_paged_fork(h: Handle, cache: mot_paged_cache, src, dst, n: int, stream=None) -> None:
    where = "mot_paged_fork"
    _fits(h, cache, where)
    _check(_lib.mot_paged_fork(h.ptr, ctypes.byref(cache), _whole(src, _INT32, n, where, "src", h.device),
                               _whole(dst, _INT32, n, where, "dst", h.device), int(n), _stream(stream)), where)


def mot_paged_free(h: Handle, cache: mot_paged_cache, seqs, n: int, stream=None) -> None:
    where = "mot_paged_free"
    _fits(h, cache, where)
    _check(_lib.mot_paged_free(h.ptr, ctypes.byref(cache), _whole(seqs, _INT32, n, where, "seqs", h.device), int(n),
                               _stream(stream)), where)


def mot_paged_compact(h: Handle, cache: mot_paged_cache, live=None, stream=None) -> None:
    where = "mot_paged_compact"
    _fits(h, cache, where)
    _check(_lib.mot_paged_compact(h.ptr, ctypes.byref(cache), _whole(live, _INT32, 1, where, "live", h.device),
                                  _stream(stream)), where)


def _contiguous_shape(h, k, v, where):
    """(n_layers, batch, max_seq) of contiguous caches [n_layers][batch][kv_heads][max_seq][head_dim]."""
    if tuple(k.shape) != tuple(v.shape) or len(k.shape) != 5:
        raise ValueError("contiguous caches are [n_layers][batch][kv_heads][max_seq][head_dim], K and V alike")
    for x in (k, v):
        if hasattr(x, "is_contiguous") and not x.is_contiguous():
            raise ValueError("contiguous caches are wanted")
    c = h.paged
    if c is not None:
        for x, what in ((k, "K"), (v, "V")):
            _typed(x, _FLOATS[c.dtype], where, what, h.device)
        if k.shape[2] != c.kv_heads or k.shape[4] != c.head_dim:
            raise _bad(where, f"{k.shape[2]} heads of {k.shape[4]}, the handle's are {c.kv_heads} of {c.head_dim}")
    return int(k.shape[0]), int(k.shape[1]), int(k.shape[3])


def mot_paged_store(h: Handle, cache: mot_paged_cache, seqs, n: int, src_k, src_v, first_layer: int = 0,
                    stream=None) -> None:
    """Tensors src_k, src_v [n_layers][batch][kv_heads][max_seq][head_dim] into the pages of the
    slots ``seqs``, layers first_layer ..."""
    where = "mot_paged_store"
    _fits(h, cache, where)
    layers, batch, max_seq = _contiguous_shape(h, src_k, src_v, where)
    _check(_lib.mot_paged_store(h.ptr, ctypes.byref(cache), int(first_layer), layers,
                                _whole(seqs, _INT32, n, where, "seqs", h.device), int(n), batch, max_seq,
                                _addr(src_k), _addr(src_v), _stream(stream)), where)


def mot_paged_load(h: Handle, cache: mot_paged_cache, seqs, n: int, dst_k, dst_v, first_layer: int = 0,
                   stream=None) -> None:
    """The pages of the slots ``seqs`` into tensors [n_layers][batch][kv_heads][max_seq][head_dim]."""
    where = "mot_paged_load"
    _fits(h, cache, where)
    layers, batch, max_seq = _contiguous_shape(h, dst_k, dst_v, where)
    _check(_lib.mot_paged_load(h.ptr, ctypes.byref(cache), int(first_layer), layers,
                               _whole(seqs, _INT32, n, where, "seqs", h.device), int(n), batch, max_seq,
                               _addr(dst_k), _addr(dst_v), _stream(stream)), where)


def _row_stride(x, what: str, least=None, where: str = "") -> int:
    """The stride of rows [heads][head_dim]; ``least``: (rows, heads, head_dim) that x has to hold."""
    shape = x.shape
    if len(shape) == 3:
        n, heads, d = shape
        row, head, last = x.stride()
        if last == 1 and (head == d or heads == 1):
            if least is not None and (n < least[0] or heads != least[1] or d != least[2]):
                raise _bad(where, f"{what} is {tuple(shape)}, the handle's is {least}")
            return row if n > 1 else heads * d   # the stride of a single row, or head, says nothing
    raise ValueError(f"{what}: [rows][heads][head_dim] with contiguous rows is wanted")


def _rows_at(x, what: str, least, kinds, where: str, dev):
    """Address and stride of rows x that have to hold ``least`` and to be of one of the types; what is refused is
    found out by the checks one by one."""
    shape = x.shape
    if len(shape) == 3 and shape[0] >= least[0] and shape[1] == least[1] and shape[2] == least[2] and x.dtype in kinds \
            and x.is_cuda and (dev is None or x.get_device() == dev):
        row, head, last = x.stride()
        if last == 1 and (head == least[2] or least[1] == 1):
            return x.data_ptr(), row if shape[0] > 1 else least[1] * least[2]
    stride = _row_stride(x, what, least, where)
    _typed(x, kinds, where, what, dev)
    return x.data_ptr(), stride


def _append(h: Handle, layer, cache, batch, q, k, v, q_out, q_norm, k_norm, stream, where, positions=()) -> None:
    c, dev = _fits(h, cache, where), h.device
    if c is None:
        (q, sq), (k, sk), (v, sv) = ((x.data_ptr(), _row_stride(x, what)) for x, what in ((q, "q"), (k, "k"), (v, "v")))
        positions = [_addr(x) for x in positions]
        q_out, q_norm, k_norm = _addr(q_out), _addr(q_norm), _addr(k_norm)
    else:
        rows, kinds, hq, d = _batch_fits(h, batch, where), _FLOATS[c.dtype], c.q_heads, c.head_dim
        kv = (rows, c.kv_heads, d)
        q, sq = _rows_at(q, "q", (rows, hq, d), kinds, where, dev)
        k, sk = _rows_at(k, "k", kv, kinds, where, dev)
        v, sv = _rows_at(v, "v", kv, kinds, where, dev)
        q_out = _whole(q_out, kinds, rows * hq * d, where, "q_out", dev)
        if q_norm is not None:
            q_norm = _whole(q_norm, kinds, d, where, "q_norm", dev)
        if k_norm is not None:
            k_norm = _whole(k_norm, kinds, d, where, "k_norm", dev)
        if positions:
            x, = positions
            if hasattr(x, "shape") and x.shape[-1] != rows:
                raise _bad(where, f"positions is {tuple(x.shape)}, {(h.axes, rows)} is wanted")
            positions = (_whole(x, _INT32, h.axes * rows, where, "positions", dev),)
    status = _calls[where](h.ptr, int(layer), ctypes.byref(cache), ctypes.byref(batch), *positions, q, sq, k, sk, v, sv, q_norm,
                           k_norm, q_out, _stream(stream))
    if status:
        _check(status, where)


def mot_paged_append(h: Handle, layer: int, cache: mot_paged_cache, batch: mot_paged_batch, q, k, v, q_out,
                     q_norm=None, k_norm=None, stream=None) -> None:
    """Tensors q, k, v [rows][heads][head_dim], whose rows may lie apart (columns of a fused
    projection); q_out [rows][q_heads][head_dim] contiguous."""
    _append(h, layer, cache, batch, q, k, v, q_out, q_norm, k_norm, stream, "mot_paged_append")


def mot_paged_set_axes(h: Handle, axes: int, axis, rates=None) -> None:
    """Pair i of a head turns by the position of axis ``axis[i]``, times ``rates[i]`` radians (None: the
    config's base). Host sequences of rot_dim / 2 numbers."""
    where = "mot_paged_set_axes"
    pairs = len(axis) if h.paged is None else h.paged.rot_dim // 2
    if len(axis) != pairs or (rates is not None and len(rates) != pairs):
        raise _bad(where, f"{pairs} pairs are rotated")
    _check(_lib.mot_paged_set_axes(h.ptr, int(axes), (ctypes.c_int32 * pairs)(*axis),
                                   None if rates is None else (ctypes.c_double * pairs)(*rates)), where)
    h.axes = int(axes)


def mot_paged_append_at(h: Handle, layer: int, cache: mot_paged_cache, batch: mot_paged_batch, positions, q, k, v, q_out,
                        q_norm=None, k_norm=None, stream=None) -> None:
    """mot_paged_append with an int32 tensor ``positions`` [axes][rows] that the rotation goes by."""
    _append(h, layer, cache, batch, q, k, v, q_out, q_norm, k_norm, stream, "mot_paged_append_at", (positions,))


def mot_paged_attention(h: Handle, layer: int, cache: mot_paged_cache, batch: mot_paged_batch, q, out,
                        stream=None) -> None:
    """Tensors q, out [rows][q_heads][head_dim], contiguous."""
    where = "mot_paged_attention"
    c, dev = _fits(h, cache, where), h.device
    if c is None:
        q, out = _addr(q), _addr(out)
    else:
        least, kinds = _batch_fits(h, batch, where) * c.q_heads * c.head_dim, _FLOATS[c.dtype]
        q, out = _whole(q, kinds, least, where, "q", dev), _whole(out, kinds, least, where, "out", dev)
    status = _calls[where](h.ptr, int(layer), ctypes.byref(cache), ctypes.byref(batch), q, out, _stream(stream))
    if status:
        _check(status, where)


def mot_create(cfg: mot_config) -> Handle:
    out = ctypes.c_void_p()
    _check(_lib.mot_create(ctypes.byref(cfg), ctypes.byref(out)), "mot_create")
    return Handle(out.value, cfg.n_layers_tgt)


def mot_load_weights(h: Handle, blob) -> None:
    """``blob``: host numpy array / bytes-like holding the packed weights."""
    if hasattr(blob, "ctypes"):
        ptr, nbytes = blob.ctypes.data, blob.nbytes
    else:
        buf = (ctypes.c_char * len(blob)).from_buffer_copy(blob)
        ptr, nbytes = ctypes.addressof(buf), len(blob)
    _check(_lib.mot_load_weights(h.ptr, ptr, nbytes), "mot_load_weights")


def mot_translate(h: Handle, src_k, src_v, seq_lens, batch: int, dst_k, dst_v, stream=None) -> None:
    _check(_lib.mot_translate(h.ptr, _addr(src_k), _addr(src_v), _addr(seq_lens), int(batch),
                              _addr(dst_k), _addr(dst_v), _stream(stream)), "mot_translate")


def mot_translate_host(h: Handle, src_k, src_v, seq_lens, batch: int, dst_k, dst_v,
                       stream=None) -> None:
    _check(_lib.mot_translate_host(h.ptr, _addr(src_k), _addr(src_v), _addr(seq_lens), int(batch),
                                   _addr(dst_k), _addr(dst_v), _stream(stream)),
           "mot_translate_host")


MOT_STATIC_SCRATCH_BYTES = 64 << 20


def mot_translate_static(cfg: mot_config, weights, src_k, src_v, seq_lens, batch: int, dst_k,
                         dst_v, stream=None) -> None:
    """Allocation-free translation: no handle, weights (packed blob) in device memory."""
    _check(_lib.mot_translate_static(ctypes.byref(cfg), _addr(weights), _addr(src_k),
                                     _addr(src_v), _addr(seq_lens), int(batch), _addr(dst_k),
                                     _addr(dst_v), _stream(stream)), "mot_translate_static")


def mot_debug_fixed_gate(h: Handle, gate) -> None:
    """Use the gate rows in `gate` (device float [G][max_batch][max_seq][E]) until
    cleared with None."""
    _check(_lib.mot_debug_fixed_gate(h.ptr, _addr(gate)), "mot_debug_fixed_gate")


GELU_FORM_MLP, GELU_FORM_BACKBONE, GELU_FORM_SIMT = 0, 1, 2


def mot_debug_gelu(form: int, u, gate, out, stream=None) -> None:
    """out = GELU(u) * gate with the device GELU form `form` (float32 device tensors)."""
    _check(_lib.mot_debug_gelu(int(form), _addr(u), _addr(gate), int(u.numel()), _addr(out),
                               _stream(stream)), "mot_debug_gelu")


def mot_get_device_status(h: Handle, stream=None) -> int:
    """Returns the status code (does not raise for device-reported errors)."""
    return _lib.mot_get_device_status(h.ptr, _stream(stream))


def mot_destroy(h: Handle) -> None:
    if h.ptr:
        ptr, h.ptr = h.ptr, None
        _check(_lib.mot_destroy(ptr), "mot_destroy")


def mot_get_layer_map(h: Handle) -> list:
    arr = (ctypes.c_int32 * h.n_layers_tgt)()
    _check(_lib.mot_get_layer_map(h.ptr, arr, h.n_layers_tgt), "mot_get_layer_map")
    return list(arr)


def mot_get_path(h: Handle) -> int:
    p = ctypes.c_int32()
    _check(_lib.mot_get_path(h.ptr, ctypes.byref(p)), "mot_get_path")
    return p.value


SCHEDULE_SPLIT, SCHEDULE_FUSED, SCHEDULE_PAIR, SCHEDULE_ONCHIP = 0, 1, 2, 3


def mot_set_schedule(h: Handle, schedule: int) -> None:
    _check(_lib.mot_set_schedule(h.ptr, int(schedule)), "mot_set_schedule")


def mot_get_schedule(h: Handle) -> int:
    v = ctypes.c_int32()
    _check(_lib.mot_get_schedule(h.ptr, ctypes.byref(v)), "mot_get_schedule")
    return v.value


def mot_debug_set(h: Handle, stall_test: bool, wait_limit_cycles: int = 0) -> None:
    _check(_lib.mot_debug_set(h.ptr, int(bool(stall_test)), int(wait_limit_cycles)), "mot_debug_set")


PROFILE_STAGES, PROFILE_AS_LAUNCHED = 1, 2


def mot_profile_enable(h: Handle, enable: int = True) -> None:
    """True (PROFILE_STAGES): backbone handles run stage by stage; PROFILE_AS_LAUNCHED: every
    handle's own launches."""
    level = PROFILE_AS_LAUNCHED if enable is not True and enable == PROFILE_AS_LAUNCHED else int(bool(enable))
    _check(_lib.mot_profile_enable(h.ptr, level), "mot_profile_enable")


def mot_profile_read(h: Handle) -> dict:
    """{kernel name: (launches, total_ms)} since the last read."""
    cap = 16
    arr = (mot_kernel_stat * cap)()
    n = ctypes.c_int32()
    _check(_lib.mot_profile_read(h.ptr, arr, cap, ctypes.byref(n)), "mot_profile_read")
    return {arr[i].name.decode(): (arr[i].launches, arr[i].total_ms) for i in range(n.value)}


def mot_get_launch_count(h: Handle) -> int:
    c = ctypes.c_int64()
    _check(_lib.mot_get_launch_count(h.ptr, ctypes.byref(c)), "mot_get_launch_count")
    return c.value


ROUTING_DENSE, ROUTING_SPARSE = 0, 1


def mot_set_routing(h: Handle, routing: int) -> None:
    _check(_lib.mot_set_routing(h.ptr, int(routing)), "mot_set_routing")


def mot_get_routing(h: Handle) -> int:
    v = ctypes.c_int32()
    _check(_lib.mot_get_routing(h.ptr, ctypes.byref(v)), "mot_get_routing")
    return v.value


def mot_get_expert_counts(h: Handle, n_groups: int, n_translators: int, stream=None):
    """Tokens routed to each translator of each (layer, K/V) group by the last
    translation: an int32 array [n_groups][n_translators]."""
    import numpy as np
    out = np.zeros((n_groups, n_translators), dtype=np.int32)
    _check(_lib.mot_get_expert_counts(h.ptr, out.ctypes.data, out.size, _stream(stream)),
           "mot_get_expert_counts")
    return out


def expert_usage(counts):
    """Translator usage statistics over selection counts I_e (Sec. 4.3), all
    groups pooled: (Var(I) / Mean(I)^2, -sum p_e ln p_e). Computed by the
    library's mot_expert_usage."""
    import numpy as np
    c = np.ascontiguousarray(np.asarray(counts).ravel(), dtype=np.int32)
    cv2, ent = ctypes.c_double(), ctypes.c_double()
    _check(_lib.mot_expert_usage(c.ctypes.data, int(c.size), ctypes.byref(cv2), ctypes.byref(ent)),
           "mot_expert_usage")
    return cv2.value, ent.value
