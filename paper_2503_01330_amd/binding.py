"""ctypes binding of libwkv (include/wkv.h): argument marshalling only.

Every step of the method runs inside the library's HIP kernels.  There is no
CPU or PyTorch fallback: if the shared library has not been built, importing
this module raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import numpy as np

# PyTorch ships its own copy of the HIP runtime.  The tensors handed to wkv_step live in that
# runtime's context, so it has to be the one libwkv binds to: load torch first, and the
# dynamic loader resolves libwkv's libamdhip64 dependency to the copy already in the process.
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libwkv.so")

WKV_FP32, WKV_FP16, WKV_BF16 = 0, 1, 2
WKV_OK, WKV_EINVAL, WKV_ENOMEM, WKV_EHIP, WKV_ESIZE = 0, -1, -2, -3, -4
WKV_MAX_BUDGET = 4095
WKV_MAX_PROMPT = 4096
WKV_SCORE_AVERAGE, WKV_SCORE_CUMULATIVE, WKV_SCORE_LAST = 0, 1, 2
WKV_MERGE_CONVEX, WKV_MERGE_NONE = 0, 1
WKV_LOADS_AUTO, WKV_LOADS_CACHED, WKV_LOADS_STREAMING = 0, 1, 2
(WKV_STEP, WKV_LEN, WKV_K, WKV_V, WKV_SCORE_SUM, WKV_COUNT, WKV_POS, WKV_NMERGED,
 WKV_EVICT_POS, WKV_EVICT_SLOT, WKV_STATUS) = range(11)

EXPORTS = ("wkv_create", "wkv_create_ex", "wkv_step", "wkv_prefill", "wkv_prefill_noalloc", "wkv_state", "wkv_load", "wkv_destroy",
           "wkv_last_error", "wkv_workspace_bytes", "wkv_step_bytes", "wkv_launch_shape", "wkv_probe_read", "wkv_paged_workspace_bytes",
           "wkv_paged_step", "wkv_paged_prefill", "wkv_paged_evict", "wkv_version")


class wkv_options(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("batch", "heads", "head_dim", "budget", "recent_window",
                                        "dtype", "n_sink", "score_mode", "merge_mode",
                                        "log_capacity", "threads", "split", "streaming", "max_prompt", "replayable")] + [("reserved", C.c_int * 1)]


class wkv_paged(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("k", "v")] + [(n, C.c_int64) for n in ("page_stride", "slot_stride", "head_stride")]
                + [("table", C.c_void_p), ("table_stride", C.c_int64), ("lens", C.c_void_p), ("scores", C.c_void_p), ("score_stride", C.c_int64)]
                + [(n, C.c_int) for n in ("batch", "heads", "kv_heads", "head_dim", "dtype", "page_size", "n_pages", "max_pages",
                                          "window", "n_sink")] + [("reserved", C.c_int * 4)])


class wkv_paged_rows(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("q", "k", "v", "out")]
                + [(n, C.c_int64) for n in ("q_stride", "q_head_stride", "k_stride", "k_head_stride", "v_stride", "v_head_stride",
                                            "out_stride", "out_head_stride")])


class WkvError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libwkv error {code}: {msg}")
        self.code = code


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it first (python -c "
                      "'import __graft_entry__ as g; g.build()'); there is no fallback path")

_lib = C.CDLL(LIB_PATH)
_lib.wkv_create.argtypes = [C.POINTER(C.c_void_p)] + [C.c_int] * 6
_lib.wkv_create_ex.argtypes = [C.POINTER(C.c_void_p), C.POINTER(wkv_options)]
_lib.wkv_step.argtypes = [C.c_void_p] * 6
_step = _lib.wkv_step
_lib.wkv_prefill.argtypes = [C.c_void_p] * 5 + [C.c_int, C.c_void_p]
_lib.wkv_prefill_noalloc.argtypes = [C.c_void_p] * 5 + [C.c_int, C.c_void_p]
_lib.wkv_state.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_size_t]
_lib.wkv_load.argtypes = [C.c_void_p, C.c_int64, C.c_int] + [C.c_void_p] * 4
_lib.wkv_destroy.argtypes = [C.c_void_p]
_lib.wkv_last_error.restype = C.c_char_p
_lib.wkv_workspace_bytes.restype = C.c_size_t
_lib.wkv_workspace_bytes.argtypes = [C.POINTER(wkv_options)]
_lib.wkv_step_bytes.restype = C.c_size_t
_lib.wkv_step_bytes.argtypes = [C.POINTER(wkv_options)]


_lib.wkv_paged_workspace_bytes.restype = C.c_size_t
_lib.wkv_paged_workspace_bytes.argtypes = [C.POINTER(wkv_paged), C.c_int, C.c_int]
_lib.wkv_paged_step.argtypes = [C.c_void_p] * 3 + [C.c_size_t, C.c_void_p]
_lib.wkv_paged_prefill.argtypes = [C.c_void_p] * 3 + [C.c_int, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
_lib.wkv_paged_evict.argtypes = [C.c_void_p, C.c_int, C.c_int] + [C.c_void_p] * 4 + [C.c_size_t, C.c_void_p]
_paged_step = _lib.wkv_paged_step
_lib.wkv_probe_read.argtypes = [C.c_void_p, C.c_size_t, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p]


def wkv_probe_read(src: int, nbytes: int, workgroups: int, threads: int, nontemporal: bool, sink: int = 0,
                   stream: int = 0) -> None:
    """Plain streaming read of device memory with a chosen launch shape (measurement aid)."""
    _check(_lib.wkv_probe_read(src, nbytes, workgroups, threads, int(nontemporal), sink or None, stream))


def wkv_last_error() -> str:
    return _lib.wkv_last_error().decode()


def _check(rc):
    if rc != WKV_OK:
        raise WkvError(rc, wkv_last_error())


def wkv_version() -> int:
    return _lib.wkv_version()


def make_options(batch, heads, head_dim, budget, recent_window, dtype, n_sink=0, score_mode=0,
                 merge_mode=0, log_capacity=0, threads=0, split=0, streaming=0, max_prompt=0,
                 replayable=0) -> wkv_options:
    return wkv_options(batch, heads, head_dim, budget, recent_window, dtype, n_sink, score_mode,
                       merge_mode, log_capacity, threads, split, streaming, max_prompt, replayable)


def wkv_create(batch, heads, head_dim, budget, recent_window, dtype):
    h = C.c_void_p()
    _check(_lib.wkv_create(C.byref(h), batch, heads, head_dim, budget, recent_window, dtype))
    return h


def wkv_create_ex(opt: wkv_options):
    h = C.c_void_p()
    _check(_lib.wkv_create_ex(C.byref(h), C.byref(opt)))
    return h


def wkv_step(h, q: int, k_new: int, v_new: int, out: int, stream: int = 0) -> None:
    """q, k_new, v_new, out: device addresses (tensor.data_ptr()); stream: hipStream_t as int."""
    _check(_lib.wkv_step(h, q, k_new, v_new, out, stream))


def wkv_prefill(h, q: int, k: int, v: int, out: int, n_tokens: int, stream: int = 0) -> None:
    """q, k, v, out: device addresses of [n_tokens, batch, heads, head_dim] arrays (out may be 0)."""
    _check(_lib.wkv_prefill(h, q, k, v, out or None, n_tokens, stream))


def wkv_prefill_noalloc(h, q: int, k: int, v: int, out: int, n_tokens: int, stream: int = 0) -> None:
    """wkv_prefill on the library's static scratch: no device allocation in the call."""
    _check(_lib.wkv_prefill_noalloc(h, q, k, v, out or None, n_tokens, stream))


def wkv_state_raw(h, what: int, dst: np.ndarray) -> None:
    _check(_lib.wkv_state(h, what, dst.ctypes.data_as(C.c_void_p), dst.nbytes))


def wkv_load(h, tokens: int, length: int, K: np.ndarray, V: np.ndarray, score_sum: np.ndarray,
             pos: np.ndarray) -> None:
    """Host arrays in token order, as wkv_state returns them."""
    K, V = np.ascontiguousarray(K), np.ascontiguousarray(V)
    score_sum = np.ascontiguousarray(score_sum, np.float64)
    pos = np.ascontiguousarray(pos, np.int32)
    _check(_lib.wkv_load(h, tokens, length, K.ctypes.data_as(C.c_void_p), V.ctypes.data_as(C.c_void_p),
                         score_sum.ctypes.data_as(C.c_void_p), pos.ctypes.data_as(C.c_void_p)))


def wkv_destroy(h) -> None:
    _check(_lib.wkv_destroy(h))


def wkv_workspace_bytes(opt: wkv_options) -> int:
    return _lib.wkv_workspace_bytes(C.byref(opt))


def wkv_step_bytes(opt: wkv_options) -> int:
    return _lib.wkv_step_bytes(C.byref(opt))


def wkv_launch_shape(opt: wkv_options):
    """(workgroups, threads per workgroup) of a wkv_step launch for these options."""
    g, t = C.c_int(), C.c_int()
    _check(_lib.wkv_launch_shape(C.byref(opt), C.byref(g), C.byref(t)))
    return g.value, t.value


# The calling thread's current stream as an address.  torch.cuda.current_stream() makes an object of it first, 2.7 us, which is
# more than the library takes to enqueue a small cache's step; torch has the address itself for its own launchers.
if hasattr(torch._C, "_cuda_getCurrentRawStream") and hasattr(torch._C, "_cuda_getDevice"):
    _current_device = torch._C._cuda_getDevice

    def _current_stream(_raw=torch._C._cuda_getCurrentRawStream, _device=torch._C._cuda_getDevice) -> int:
        return _raw(_device())
else:
    _current_device = torch.cuda.current_device

    def _current_stream() -> int:
        return torch.cuda.current_stream().cuda_stream


_NP_STORE = {WKV_FP32: np.float32, WKV_FP16: np.float16, WKV_BF16: np.uint16}


class Cache:
    """Owner of one handle; remembers the shape so readbacks can be sized."""

    def __init__(self, batch, heads, head_dim, budget, recent_window, dtype, **kw):
        self.opt = make_options(batch, heads, head_dim, budget, recent_window, dtype, **kw)
        self.units, self.d, self.dtype = batch * heads, head_dim, dtype
        self.h = wkv_create_ex(self.opt)

    def step(self, q, k_new, v_new, out, stream=None):
        """q, k_new, v_new, out: torch tensors on the GPU, contiguous [batch, heads, head_dim]."""
        # (no layer in between: a small cache's step takes the GPU 7 us, and this call is all the host does for it)
        rc = _step(self.h, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), out.data_ptr(),
                   _current_stream() if stream is None else stream)
        if rc:
            _check(rc)

    def prefill(self, q, k, v, out=None, stream=None, noalloc=False):
        """q, k, v (and out, if wanted): torch tensors on the GPU, contiguous [n_tokens, batch, heads, head_dim]
        (or [n_tokens, units, head_dim]); the cache must be empty.  noalloc: through wkv_prefill_noalloc."""
        if stream is None:
            stream = _current_stream()
        (wkv_prefill_noalloc if noalloc else wkv_prefill)(
            self.h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr() if out is not None else 0,
            q.shape[0], stream)

    def step_ptr(self, q, k_new, v_new, out, stream=0):
        wkv_step(self.h, q, k_new, v_new, out, stream)

    @property
    def tokens(self) -> int:
        t = np.zeros(1, np.int64)
        wkv_state_raw(self.h, WKV_STEP, t)
        return int(t[0])

    @property
    def length(self) -> int:
        l = np.zeros(1, np.int32)
        wkv_state_raw(self.h, WKV_LEN, l)
        return int(l[0])

    def state(self, what):
        """Slot arrays in token order; K/V in the storage dtype (bf16 as uint16 bit patterns)."""
        L = self.length
        if what in (WKV_K, WKV_V):
            dst = np.empty((self.units, L, self.d), _NP_STORE[self.dtype])
        elif what == WKV_SCORE_SUM:
            dst = np.empty((self.units, L), np.float64)
        elif what in (WKV_COUNT, WKV_POS, WKV_NMERGED):
            dst = np.empty((self.units, L), np.int32)
        elif what == WKV_STATUS:
            dst = np.empty(2, np.int32)
        else:
            raise ValueError("use evictions() / tokens / length for this item")
        if dst.size:
            wkv_state_raw(self.h, what, dst)
        return dst

    def evictions(self, n):
        """(evict_pos, evict_slot) of the last n steps, each int32 [n, units]."""
        pos = np.empty((n, self.units), np.int32)
        slot = np.empty((n, self.units), np.int32)
        if n:
            wkv_state_raw(self.h, WKV_EVICT_POS, pos)
            wkv_state_raw(self.h, WKV_EVICT_SLOT, slot)
        return pos, slot

    def load(self, tokens, K, V, score_sum, pos):
        wkv_load(self.h, tokens, pos.shape[1] if pos.ndim == 2 else 0, K, V, score_sum, pos)

    def step_bytes(self) -> int:
        return wkv_step_bytes(self.opt)

    def close(self):
        if self.h is not None:
            wkv_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_pack_rows = struct.Struct("@4P8q").pack_into       # (fields of a ctypes structure, one by one, take 2 us)
_TORCH_STORE = {torch.float32: WKV_FP32, torch.float16: WKV_FP16, torch.bfloat16: WKV_BF16}


def _refuse(message):
    raise WkvError(WKV_EINVAL, message)


def _ints(**kw):
    """(ctypes keeps the lowest 32 bits of a larger number)"""
    for name, x in kw.items():
        if not -2 ** 31 <= x < 2 ** 31:
            _refuse(f"{name}: {x} is no 32-bit number")


class PagedCache:
    """A wkv_paged over torch tensors that the caller owns, and a workspace of its own.

    k, v:   [n_pages, page_size, kv_heads, head_dim] on the GPU, any strides that are multiples of 16 bytes with the last one 1 (a
            pool laid out [page][head][slot] is handed over transposed); float32, float16 or bfloat16
    table:  int32 [batch, max_pages], lens: int32 [batch]
    scores: float32 [batch, kv_heads, n], n within the last page, or None
    The tensors are kept alive; what they hold is read when a call runs.  Calls on one object must not overlap in time
    (the workspace is one); another object over the same tensors has its own.

    A call runs on the current stream, or on `stream` (its address), whichever that is: the workspace's memory is given back when the streams
    that it was used on have got past it.  A stream that is no torch stream has to exist as long as the object, and the object as long as a
    HIP graph that has recorded its calls.
    """

    def __init__(self, k, v, table, lens, heads, window=0, n_sink=0, scores=None, max_tokens=0, max_new=0):
        _ints(heads=heads, window=window, n_sink=n_sink, max_tokens=max_tokens, max_new=max_new)
        if k.dim() != 4 or k.dtype not in _TORCH_STORE or v.shape != k.shape or v.dtype != k.dtype or v.stride() != k.stride():
            _refuse("k and v: [n_pages, page_size, kv_heads, head_dim] of one type and layout")
        if table.dim() != 2 or table.dtype != torch.int32 or lens.shape != table.shape[:1] or lens.dtype != torch.int32:
            _refuse("table: int32 [batch, max_pages], lens: int32 [batch]")
        if scores is not None and (scores.dtype != torch.float32 or scores.dim() != 3 or scores.shape[:2] != (table.shape[0], k.shape[2])):
            _refuse("scores: float32 [batch, kv_heads, slots]")
        for t in (k, table) + (() if scores is None else (scores,)):
            if t.stride(-1) != 1 and t.shape[-1] != 1:
                _refuse("the last dimension of pools, table and scores must be contiguous")
        if not lens.is_contiguous() or (scores is not None and not scores.is_contiguous()):
            _refuse("lens and scores must be contiguous")
        self._tensors = (k, v, table, lens, scores)
        if any(t is not None and t.device != k.device for t in self._tensors) or k.device.type != "cuda":
            _refuse("pools, table, lens and scores must be on one GPU")
        self.device, self.dtype, self.index = k.device, k.dtype, k.device.index
        self.batch, self.heads, self.kv_heads, self.head_dim = table.shape[0], heads, k.shape[2], k.shape[3]
        self.c = wkv_paged(k.data_ptr(), v.data_ptr(), *k.stride()[:3], table.data_ptr(), table.stride(0), lens.data_ptr(),
                           scores.data_ptr() if scores is not None else None, scores.shape[2] if scores is not None else 0,
                           self.batch, heads, self.kv_heads, self.head_dim, _TORCH_STORE[k.dtype], k.shape[1], k.shape[0], table.shape[1],
                           window, n_sink)
        self.rows = wkv_paged_rows()
        self._ref, self._rows_ref = C.addressof(self.c), C.addressof(self.rows)
        self._row, self._row_new = (heads, self.head_dim), (self.kv_heads, self.head_dim)
        self._kept = []
        self._work = None
        self._reserve(max_tokens, max_new)

    def _reserve(self, n_tokens, max_new, stream=None):
        need = _lib.wkv_paged_workspace_bytes(C.byref(self.c), n_tokens, max_new)
        if need == 0:
            _refuse("no workspace for these sizes: " + wkv_last_error())
        have = 0 if self._work is None else self._work.numel()
        if have < need:
            self._grow(max(need, have + have // 2), stream)          # (all that are kept: twice this one)
        self._at, self._bytes = self._work.data_ptr(), self._work.numel()

    def _grow(self, size, stream):
        home = torch.cuda.current_stream(self.device)
        for s in (home, *([] if stream is None else [torch.cuda.ExternalStream(stream, device=self.device)])):
            with torch.cuda.stream(s):
                if torch.cuda.is_current_stream_capturing():
                    _refuse("no workspace is taken while a graph is recorded: make a call of these sizes before, or an object with these max_tokens and max_new")
        work = torch.empty(size, dtype=torch.uint8, device=self.device)
        # What had the memory before may still run on the stream that it is taken on, which other streams do not wait for.
        home.synchronize()
        self._kept.append(self._work)                       # (work on another stream may still be using it, or a recorded graph)
        self._work, self._streams = work, {home.cuda_stream}

    def _used_on(self, stream):
        """The workspace's memory waits for this stream too before it is anyone else's."""
        self._work.record_stream(torch.cuda.ExternalStream(stream, device=self.device))
        self._streams.add(stream)

    def _fill(self, n, q, k, v, out):
        """The rows of a call, n tokens."""
        if (k is None) != (v is None):
            _refuse("k and v: both, or both None")
        x = []
        for t, shape in ((q, self._row), (k, self._row_new), (v, self._row_new), (out, self._row)):
            if t is None:
                x += (0, 0, 0)
                continue
            if t.dtype is not self.dtype or t.shape != (n, *shape) or t.get_device() != self.index:
                _refuse(f"rows of a call: {[n, *shape]} in the cache's type, on its GPU")
            s, h, e = t.stride()
            if e != 1:
                _refuse("the elements of a row must be next to each other")
            x += (t.data_ptr(), s, h)
        _pack_rows(self.rows, 0, x[0], x[3], x[6], x[9], x[1], x[2], x[4], x[5], x[7], x[8], x[10], x[11])

    def _stream(self, stream):
        if _current_device() != self.index:
            _refuse(f"the cache belongs to device {self.index}, which is not the current one")
        return _current_stream() if stream is None else stream

    def step(self, q, k_new, v_new, out, stream=None):
        """One token for every sequence: q, out [batch, heads, head_dim]; k_new, v_new [batch, kv_heads, head_dim], or both None
        (appended already).  Any strides that are multiples of 16 bytes.  lens counts the new tokens."""
        stream = self._stream(stream)
        self._fill(self.batch, q, k_new, v_new, out)
        if stream not in self._streams:
            self._used_on(stream)
        rc = _paged_step(self._ref, self._rows_ref, self._at, self._bytes, stream)
        if rc:
            _check(rc)

    def prefill(self, q, k, v, out, starts, max_new, stream=None):
        """A chunk of new tokens for every sequence, tokens starts[b] .. starts[b + 1] of q, out [n_tokens, heads, head_dim] and
        k, v [n_tokens, kv_heads, head_dim] (or both None); starts: int32 [batch + 1] on the GPU; max_new: the longest chunk.  The workspace
        grows here if it has to: a call recorded into a HIP graph follows one of the same sizes, or a constructor with these max_tokens and
        max_new."""
        stream = self._stream(stream)
        n = q.shape[0]
        self._fill(n, q, k, v, out)
        if starts.dtype != torch.int32 or starts.shape != (self.batch + 1,) or not starts.is_contiguous() or starts.get_device() != self.index:
            _refuse("starts: int32 [batch + 1] on the cache's GPU")
        if not 1 <= max_new <= n:
            _refuse(f"1 <= max_new <= n_tokens is wanted: {max_new}, {n}")
        self._reserve(n, max_new, stream)
        if stream not in self._streams:
            self._used_on(stream)
        _check(_lib.wkv_paged_prefill(self._ref, self._rows_ref, starts.data_ptr(), n, max_new, self._at, self._bytes, stream))

    def evict(self, budget, recent_window, new_lens, new_scores, kept=None, stream=None):
        """Cuts every sequence to `budget` slots: new_lens int32 [batch], new_scores like scores, kept int32 [batch, kv_heads, budget].
        new_lens and new_scores may be lens and scores themselves."""
        stream = self._stream(stream)
        _ints(budget=budget, recent_window=recent_window)
        scores = self._tensors[4]
        for t, like, what in ((new_lens, self._tensors[3], "new_lens"), (new_scores, scores, "new_scores")):
            if like is None:
                _refuse("eviction needs scores")
            if t.dtype != like.dtype or t.shape != like.shape or not t.is_contiguous() or t.device != self.device:
                _refuse(f"{what} must be like what it replaces")
        if kept is not None and (kept.dtype != torch.int32 or tuple(kept.shape) != (self.batch, self.kv_heads, budget)
                                 or not kept.is_contiguous() or kept.device != self.device):
            _refuse("kept: int32 [batch, kv_heads, budget]")
        if stream not in self._streams:
            self._used_on(stream)
        _check(_lib.wkv_paged_evict(self._ref, budget, recent_window, new_lens.data_ptr(), new_scores.data_ptr(),
                                    kept.data_ptr() if kept is not None else None, self._at, self._bytes, stream))
