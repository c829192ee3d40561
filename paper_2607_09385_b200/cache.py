"""ctypes binding of the paged 4-bit key/value cache in ``include/steel_cache.h``.

Functions with the name and meaning of their C counterparts, and ``SteelCache``, which owns a cache's
device memory as torch tensors.  The library is the one that ``binding`` loads; there is no fallback.
"""
from __future__ import annotations

import ctypes
import struct

from . import binding
from .binding import STEEL_MASK_CAUSAL, STEEL_MASK_WINDOW, STEEL_OK, SteelError

STEEL_ERR_NO_PAGES = 6

EXPORTS = (
    "steel_cache_sizes", "steel_cache_create", "steel_cache_destroy", "steel_cache_reset", "steel_cache_extend",
    "steel_cache_append", "steel_cache_read", "steel_cache_attend", "steel_cache_attend_workspace", "steel_cache_fork",
    "steel_cache_free", "steel_cache_compact", "steel_cache_debug_wait", "steel_cache_last_status",
)

_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class CacheParams(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("layers", "pages", "page_tokens", "heads_kv", "head_dim", "slots", "max_pages")]


class CacheSizes(ctypes.Structure):
    _fields_ = [(n, _i64) for n in ("pool_bytes", "table_bytes", "lens_bytes", "refs_bytes", "status_bytes",
                                    "scratch_bytes", "unit_bytes", "page_bytes")]


class CacheMemory(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("pool", "table", "lens", "refs", "status", "scratch")]


class CacheTensor(ctypes.Structure):
    _fields_ = [("data", _vp), ("stride_batch", _i64), ("stride_head", _i64), ("stride_seq", _i64)]


class CacheAttend(ctypes.Structure):
    _fields_ = [("layer", _i32), ("batch", _i32), ("heads_q", _i32), ("seq_q", _i32), ("slots", _vp), ("counts", _vp),
                ("flags", ctypes.c_uint32), ("scale", ctypes.c_float), ("window", _i64), ("q", CacheTensor), ("o", _vp),
                ("lse", _vp), ("workspace", _vp), ("workspace_bytes", _i64)]


_lib = None


def load_library():
    """The library that ``binding`` loads, with the cache's functions declared."""
    global _lib
    if _lib is not None:
        return _lib
    lib = binding.load_library()
    ref = ctypes.POINTER
    lib.steel_cache_sizes.argtypes = [ref(CacheParams), ref(CacheSizes)]
    lib.steel_cache_create.argtypes = [ref(CacheParams), ref(CacheMemory), ref(_vp)]
    lib.steel_cache_destroy.argtypes = [_vp]
    lib.steel_cache_reset.argtypes = [_vp, _vp]
    lib.steel_cache_extend.argtypes = [_vp, _i32, _vp, _vp, _vp]
    # structures by address: a number costs 0.2 us less than an instance
    lib.steel_cache_append.argtypes = [_vp, _i32, _i32, _vp, _vp, _i32, _vp, _vp, _vp]
    lib.steel_cache_read.argtypes = [_vp, _i32, _i32, _vp, _vp, _i32, _vp, _vp, _vp]
    lib.steel_cache_attend.argtypes = [_vp, _vp, _vp]
    lib.steel_cache_attend_workspace.argtypes = [_vp, _i32, _i32, _i32]
    lib.steel_cache_fork.argtypes = [_vp, _i32, _vp, _vp, _vp]
    lib.steel_cache_free.argtypes = [_vp, _i32, _vp, _vp, _vp]
    lib.steel_cache_compact.argtypes = [_vp, _vp, _vp]
    lib.steel_cache_debug_wait.argtypes = [_vp, _i64]
    lib.steel_cache_last_status.argtypes = [_vp, _vp]
    for name in EXPORTS:
        getattr(lib, name).restype = ctypes.c_int
    lib.steel_cache_attend_workspace.restype = _i64
    _lib = lib
    return lib


def _check(status: int, where: str) -> None:
    if status != STEEL_OK:
        raise SteelError(status, where)


def steel_cache_sizes(params: CacheParams) -> dict:
    s = CacheSizes()
    _check(load_library().steel_cache_sizes(ctypes.byref(params), ctypes.byref(s)), "steel_cache_sizes")
    return {n: getattr(s, n) for n, _ in CacheSizes._fields_}


def steel_cache_create(params: CacheParams, memory: CacheMemory) -> int:
    handle = _vp()
    _check(load_library().steel_cache_create(ctypes.byref(params), ctypes.byref(memory), ctypes.byref(handle)),
           "steel_cache_create")
    return handle.value


def steel_cache_destroy(handle) -> None:
    _check(load_library().steel_cache_destroy(handle), "steel_cache_destroy")


def steel_cache_debug_wait(handle, cycles: int) -> None:
    """Test hook: the bound of attend's wait for other CTAs' parts (0: one look; < 0: the default)."""
    _check(load_library().steel_cache_debug_wait(handle, cycles), "steel_cache_debug_wait")


# The layouts of steel_cache_tensor_t and steel_cache_attend_t: one call fills a structure (field by field costs 1 us more)
_PACK_TENSOR = struct.Struct("Pqqq")
_PACK_ATTEND = struct.Struct("iiiiPPIfqPqqqPPPq")
assert _PACK_TENSOR.size == ctypes.sizeof(CacheTensor) and _PACK_ATTEND.size == ctypes.sizeof(CacheAttend)


class SteelCache:
    """Owner of one cache on a CUDA device (the current one by default).

    ``pool``, ``table``, ``lens`` and ``refs`` are torch tensors in the layout of the header; the methods enqueue
    their kernels on torch's current stream of that device, which has to be the current one (``torch.cuda.device``): they
    refuse with STEEL_ERR_INVALID_ARG otherwise.  Index arguments (``slots``, ``counts``, ``begin``,
    ``keep``, ``src``, ``dst``) are int32 CUDA tensors; what is wrong in them is found on the device and reported by
    ``last_status``.  Calls on one object from several host threads have to be serialised.  A step of a decoder:

        cache.extend(counts, slots)                       # once: room for the new tokens, in every layer
        for layer in ...:
            cache.append(layer, k, v, counts, slots)
            o, lse = cache.attend(layer, q, scale, counts, slots)
    """

    def __init__(self, layers, pages, page_tokens, heads_kv, head_dim, slots, max_pages, device=None):
        import torch
        self.params = CacheParams(layers, pages, page_tokens, heads_kv, head_dim, slots, max_pages)
        size = steel_cache_sizes(self.params)
        assert device is None or torch.device(device).type == "cuda", "device: a CUDA device"
        index = None if device is None else torch.device(device).index
        device = torch.device("cuda", torch.cuda.current_device() if index is None else index)
        self.device_index = device.index
        empty = lambda n, dtype: torch.empty(n, dtype=dtype, device=device)  # noqa: E731
        self.pool = empty(size["pool_bytes"], torch.uint8).view(layers, pages, heads_kv, page_tokens // 16, size["unit_bytes"])
        self.table = empty((slots, max_pages), torch.int32)
        self.lens, self.refs = empty(slots, torch.int32), empty(pages, torch.int32)
        self.status, self._scratch = empty(1, torch.int32), empty(size["scratch_bytes"], torch.uint8)
        self.live = torch.zeros(1, dtype=torch.int32, device=device)  # pages in use, as the last compact() found them
        self.heads_kv, self.head_dim, self.slots = heads_kv, head_dim, slots
        memory = CacheMemory(*(x.data_ptr() for x in (self.pool, self.table, self.lens, self.refs, self.status, self._scratch)))
        with torch.cuda.device(device):
            self.handle = steel_cache_create(self.params, memory)
            _check(load_library().steel_cache_reset(self.handle, binding._stream_getter()(device.index)), "steel_cache_reset")
        # what every call needs, looked up once: a decode step's calls are as short as this path (append of one token to 64
        # sequences: 6.9 us of host time before, of which 2.3 are the launch)
        self._lib, self._stream = load_library(), binding._stream_getter()
        self._args, self._k, self._v = CacheAttend(), CacheTensor(), CacheTensor()
        self._args_at, self._k_at, self._v_at = (ctypes.addressof(x) for x in (self._args, self._k, self._v))
        self._workspaces = {}  # bytes by (batch, heads_q, seq_q)
        self._empty, self._bf16, self._i32, self._f32 = torch.empty, torch.bfloat16, torch.int32, torch.float32
        self._device = device

    def _index(self, x, n, what):
        """Address of an index tensor of n entries (None: no tensor)."""
        if x is None:
            return None
        assert x.dtype is self._i32 and x.shape == (n,) and x.is_contiguous() and x.get_device() == self.device_index, \
            f"{what}: a contiguous int32 tensor of {n} entries on the cache's device"
        return x.data_ptr()

    def _rows(self, k, v):
        """Fill two CacheTensors from bf16 tensors [batch, heads_kv, seq, head_dim] whose last dimension is contiguous -> batch, seq."""
        shape, bf16, device = k.shape, self._bf16, self.device_index
        n, heads, seq, d = shape
        batch_k, head_k, seq_k, one_k = k.stride()
        batch_v, head_v, seq_v, one_v = v.stride()
        assert k.dtype is bf16 and v.dtype is bf16 and v.shape == shape and heads == self.heads_kv and d == self.head_dim \
            and one_k == 1 and one_v == 1 and k.get_device() == device and v.get_device() == device, \
            f"k, v: bf16 [batch, {self.heads_kv}, seq, {self.head_dim}] on the cache's device, channels side by side"
        _PACK_TENSOR.pack_into(self._k, 0, k.data_ptr(), batch_k, head_k, seq_k)
        _PACK_TENSOR.pack_into(self._v, 0, v.data_ptr(), batch_v, head_v, seq_v)
        return n, seq

    def reset(self) -> None:
        """Empty the cache."""
        _check(self._lib.steel_cache_reset(self.handle, self._stream(self.device_index)), "steel_cache_reset")

    def extend(self, counts, slots=None) -> None:
        """Room for ``counts[i]`` more tokens of each slot; a shared last page is copied first."""
        n = counts.shape[0]
        status = self._lib.steel_cache_extend(self.handle, n, self._index(slots, n, "slots"), self._index(counts, n, "counts"),
                                              self._stream(self.device_index))
        if status != STEEL_OK:
            raise SteelError(status, "steel_cache_extend")

    def append(self, layer, k, v, counts=None, slots=None) -> None:
        """Quantise the newest ``counts[i]`` tokens of each slot from k, v [batch, heads_kv, seq, head_dim] (any strides
        in multiples of 8).  Tokens on a page that another slot holds too are not written, and reported."""
        n, seq = self._rows(k, v)
        status = self._lib.steel_cache_append(self.handle, layer, n, self._index(slots, n, "slots"), self._index(counts, n, "counts"),
                                              seq, self._k_at, self._v_at, self._stream(self.device_index))
        if status != STEEL_OK:
            raise SteelError(status, "steel_cache_append")

    def read(self, layer, k, v, begin=None, slots=None):
        """Tokens ``begin[i]``, ... of each slot in bf16 into k, v [batch, heads_kv, seq, head_dim]; rows behind a slot's
        last token are left as they were."""
        n, seq = self._rows(k, v)
        status = self._lib.steel_cache_read(self.handle, layer, n, self._index(slots, n, "slots"), self._index(begin, n, "begin"),
                                            seq, self._k_at, self._v_at, self._stream(self.device_index))
        if status != STEEL_OK:
            raise SteelError(status, "steel_cache_read")
        return k, v

    def attend(self, layer, q, scale, counts=None, slots=None, flags=STEEL_MASK_CAUSAL, window=0, o=None, lse=None,
               want_lse: bool = True):
        """Attention of the newest tokens' queries [batch, heads_q, seq_q, head_dim] over the cache -> (o, lse).  Weights
        are fp16 numbers beside sums in 32 bits: ``include/steel_cache.h`` says what that costs."""
        shape = q.shape
        n, heads_q, seq, d = shape
        batch_stride, head_stride, seq_stride, one = q.stride()
        bf16, device = self._bf16, self.device_index
        assert q.dtype is bf16 and d == self.head_dim and one == 1 and q.get_device() == device, \
            f"q: bf16 [batch, heads, seq, {self.head_dim}] on the cache's device, channels side by side"
        if o is None:
            o = self._empty(shape, dtype=bf16, device=self._device)
        else:
            assert o.dtype is bf16 and o.shape == shape and o.is_contiguous() and o.get_device() == device, "o: as q, contiguous"
        if lse is None:
            if want_lse:
                lse = self._empty((n, heads_q, seq), dtype=self._f32, device=self._device)
        else:
            assert lse.dtype is self._f32 and lse.shape == (n, heads_q, seq) and lse.is_contiguous() and lse.get_device() == device, \
                "lse: float32 [batch, heads, seq], contiguous"
        need = self._workspaces.get((n, heads_q, seq))
        if need is None:
            need = self._lib.steel_cache_attend_workspace(self.handle, n, heads_q, seq)
            if need >= 0:
                self._workspaces[n, heads_q, seq] = need
        # of this call alone: calls on several streams, and graphs, do not share it.  (In 16-bit elements: new_empty takes the
        # device from q, which is 0.3 us shorter than naming it.)
        workspace = q.new_empty(max(need, 0) // 2)
        _PACK_ATTEND.pack_into(self._args, 0, layer, n, heads_q, seq, self._index(slots, n, "slots") or 0,
                               self._index(counts, n, "counts") or 0, flags, scale, window, q.data_ptr(), batch_stride,
                               head_stride, seq_stride, o.data_ptr(), 0 if lse is None else lse.data_ptr(),
                               workspace.data_ptr(), need)
        status = self._lib.steel_cache_attend(self.handle, self._args_at, self._stream(device))
        if status != STEEL_OK:
            raise SteelError(status, "steel_cache_attend")
        return o, lse

    def fork(self, src, dst) -> None:
        """Slot ``dst[i]`` takes over the pages that ``src[i]`` holds; what it held it gives up."""
        n = src.shape[0]
        status = self._lib.steel_cache_fork(self.handle, n, self._index(src, n, "src"), self._index(dst, n, "dst"),
                                            self._stream(self.device_index))
        if status != STEEL_OK:
            raise SteelError(status, "steel_cache_fork")

    def free(self, slots=None, keep=None) -> None:
        """Keep the first ``keep[i]`` tokens of each slot (None: none; slots None: all) and give the rest back."""
        n = self.slots if slots is None and keep is None else (keep if slots is None else slots).shape[0]
        status = self._lib.steel_cache_free(self.handle, n, self._index(slots, n, "slots"), self._index(keep, n, "keep"),
                                            self._stream(self.device_index))
        if status != STEEL_OK:
            raise SteelError(status, "steel_cache_free")

    def compact(self):
        """Move pages so that those in use have the lowest numbers -> their count, an int32 CUDA tensor [1]: ``live``, which the
        next call writes again."""
        _check(self._lib.steel_cache_compact(self.handle, self.live.data_ptr(), self._stream(self.device_index)),
               "steel_cache_compact")
        return self.live

    def last_status(self) -> int:
        """Wait for the current stream; the status word, which is cleared."""
        return self._lib.steel_cache_last_status(self.handle, self._stream(self.device_index))

    def close(self) -> None:
        if getattr(self, "handle", None):
            steel_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
