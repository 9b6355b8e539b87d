"""Python binding of the backend operators (include/wwws_backend.h): argument marshalling only.

`Backend` is to the serving operators what `binding.Network` is to the simulator: it owns the device workspace (a torch
tensor), hands pointers and sizes to the C calls and raises `WwwsError` on a non-zero status.  Every operator runs in the
library's CUDA kernels; there is no fallback.

    b = Backend(n_heads=32, n_kv_heads=8, head_dim=128, page_tokens=64, n_pages=4096, max_seqs=64, max_tokens=8192, max_pages=256,
                max_rows=64, cache="e4m3")
    cache = b.new_cache()                                    # one per layer of a model
    batch = b.batch(q_start, kv_len, page_table, n_tokens=..., max_q_len=..., max_kv_len=...)
    b.append(cache, batch, k, v)                             # the new tokens' keys and values
    o = b.attend(cache, batch, q, window=4096, sinks=4)
    logits, token = b.shape_logits(logits, b.shaping(history=..., history_start=..., repetition=...))
    b.sync()                                                 # raises if a kernel met a bad id

Calls are enqueued on the stream that was current at creation (or the one given).  Tensors that a caller fills on another
stream must be ready before the call; the binding records the backend's stream on them, so that their memory is not
handed out again before the call has run.
"""
from __future__ import annotations

import ctypes as C

from .binding import WwwsError, load

EXPORTS = ("wwws_backend_workspace_bytes", "wwws_create_backend", "wwws_destroy_backend", "wwws_cache_append", "wwws_cache_read",
           "wwws_attend", "wwws_shape_logits", "wwws_backend_sync", "wwws_backend_last_error")
CACHES = {"16": 0, "int8": 1, "e4m3": 2}


class BackendConfig(C.Structure):
    _fields_ = [(k, C.c_uint32) for k in ("n_heads", "n_kv_heads", "head_dim", "page_tokens", "n_pages", "max_seqs", "max_tokens", "max_pages",
                                          "max_rows", "dtype", "cache")]


class KvPages(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("k", "v", "k_scale", "v_scale")]


class SeqBatch(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("q_start", "kv_len", "page_table")] + \
               [(k, C.c_uint32) for k in ("n_seqs", "n_tokens", "max_q_len", "max_kv_len")]


SHAPING_ARRAYS = ("history", "history_start", "prompt_len", "repetition", "presence", "frequency", "bias_id", "bias_value", "bias_start",
                  "mask", "mask_index")


class ShapingRecord(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in SHAPING_ARRAYS] + [("n_history", C.c_uint64), ("n_bias", C.c_uint64),
                                                            ("n_masks", C.c_uint32), ("mask_stride", C.c_uint32)]


_ready = False


def _lib():
    global _ready
    lib = load()
    if not _ready:
        vp, u64, u32 = C.c_void_p, C.c_uint64, C.c_uint32
        sig = {
            "wwws_backend_workspace_bytes": [C.POINTER(BackendConfig), C.POINTER(u64)],
            "wwws_create_backend": [C.POINTER(BackendConfig), vp, u64, vp, C.POINTER(vp)],
            "wwws_destroy_backend": [vp],
            "wwws_cache_append": [vp, vp, vp, vp, u64, vp, u64],
            "wwws_cache_read": [vp, vp, vp, vp, u64, vp, vp],
            "wwws_attend": [vp, vp, vp, vp, u64, vp, u64, C.c_float, u32, u32],
            "wwws_shape_logits": [vp, vp, u32, u32, u32, vp, u64, vp, u64, vp],
            "wwws_backend_sync": [vp],
        }
        for name, args in sig.items():
            f = getattr(lib, name)
            f.argtypes, f.restype = args, C.c_int
        lib.wwws_backend_last_error.argtypes, lib.wwws_backend_last_error.restype = [vp], C.c_char_p
        _ready = True
    return lib


class _Record:
    """A C record, its address, the tensors whose memory it names, and what of a backend's configuration their sizes follow."""
    __slots__ = ("c", "at", "tensors", "of", "extra")

    def __init__(self, c, tensors, of, extra=None):
        self.c, self.at, self.tensors, self.of, self.extra = c, C.addressof(c), tensors, of, extra


class Backend:
    """The operators of one serving backend on one GPU.  Methods are the C calls with the status checked."""

    def __init__(self, n_heads=0, n_kv_heads=0, head_dim=0, page_tokens=0, n_pages=0, max_seqs=0, max_tokens=0, max_pages=0, max_rows=0,
                 dtype=None, cache="16", device="cuda:0", stream=None):
        import torch
        self._torch = torch
        self._lib = _lib()
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.dtype = torch.bfloat16 if dtype is None else dtype
        self._codes = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
        if self.dtype not in self._codes or cache not in CACHES:
            raise ValueError("dtype must be torch.bfloat16 or torch.float16, cache one of " + ", ".join(CACHES))
        self.cache = cache
        self.n_heads, self.n_kv_heads, self.head_dim, self.page_tokens = n_heads, n_kv_heads, head_dim, page_tokens
        self.n_pages, self.max_pages = n_pages, max_pages
        self._scale = head_dim ** -0.5 if head_dim else 1.0
        self._elem = {"16": self.dtype, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}[cache]
        cfg = BackendConfig(n_heads, n_kv_heads, head_dim, page_tokens, n_pages, max_seqs, max_tokens, max_pages, max_rows,
                            self._codes[self.dtype], CACHES[cache])
        # records made by another backend fit where these are equal
        self._caches = ("cache", self.device, self._elem, n_pages, n_kv_heads, page_tokens, head_dim)
        self._batches, self._shapings = ("batch", self.device, max_pages), ("shaping", self.device)
        self._h = None
        nbytes = C.c_uint64()
        self._check(self._lib.wwws_backend_workspace_bytes(C.byref(cfg), C.byref(nbytes)))
        with torch.cuda.device(self.device):
            self._stream = stream if stream is not None else torch.cuda.current_stream(self.device)
            with torch.cuda.stream(self._stream):
                self._ws = torch.empty(nbytes.value, dtype=torch.uint8, device=self.device)
            self._index, self._raw, self._raw_current = self.device.index, self._stream.cuda_stream, torch._C._cuda_getCurrentRawStream
            h = C.c_void_p()
            self._check(self._lib.wwws_create_backend(C.byref(cfg), self._ws.data_ptr(), nbytes.value, self._stream.cuda_stream, C.byref(h)))
        self._h = h

    def _check(self, status):
        if status:
            raise WwwsError(status, self._lib.wwws_backend_last_error(self._h).decode())

    def close(self):
        if getattr(self, "_h", None):
            self._lib.wwws_destroy_backend(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _aside(self):
        """Whether another stream than the backend's is current (asked once per call: it costs as much as a small kernel)."""
        return self._raw_current(self._index) != self._raw

    def _used(self, *tensors):
        """Mark tensors of the current stream as used on the backend's."""
        for t in tensors:
            if t is not None:
                t.record_stream(self._stream)

    def _empty(self, shape, dtype, aside):
        if not aside:
            return self._torch.empty(shape, dtype=dtype, device=self.device)
        with self._torch.cuda.stream(self._stream):
            t = self._torch.empty(shape, dtype=dtype, device=self.device)
        t.record_stream(self._torch.cuda.current_stream(self.device))
        return t

    @staticmethod
    def _fits(record, of):
        if record.of is not of and record.of != of:
            raise ValueError(f"a {of[0]} of this backend's configuration is needed, got a {record.of[0]}" + (" of another's" if record.of[0] == of[0] else ""))

    def _array(self, t, dtype, name, dims=1):
        if t.dtype != dtype or t.dim() != dims or not t.is_contiguous() or t.device != self.device:
            raise ValueError(f"{name}: expected a contiguous {dims}-d {dtype} tensor on {self.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t

    def _rows(self, t, heads, name):
        """[tokens, heads, head_dim] with packed heads; any stride between tokens."""
        if t.dtype != self.dtype or t.dim() != 3 or t.shape[1] != heads or t.shape[2] != self.head_dim or t.device != self.device:
            raise ValueError(f"{name}: expected {self.dtype} [tokens, {heads}, {self.head_dim}] on {self.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
        if t.stride(2) != 1 or t.stride(1) != self.head_dim:
            raise ValueError(f"{name}: the heads of a token must be packed, got strides {t.stride()}")
        return t.stride(0) if t.shape[0] > 1 else heads * self.head_dim

    # ---- records ----------------------------------------------------------------------------
    def new_cache(self):
        """A page pool of the configuration (uninitialised), bound."""
        shape = (self.n_pages, self.n_kv_heads, self.page_tokens)
        aside = self._aside()
        k, v = (self._empty(shape + (self.head_dim,), self._elem, aside) for _ in range(2))
        ks, vs = (None, None) if self.cache == "16" else (self._empty(shape, self._torch.float32, aside) for _ in range(2))
        return self.bind_cache(k, v, ks, vs)

    def bind_cache(self, k, v, k_scale=None, v_scale=None):
        """Name caller-owned pages: k, v [n_pages, n_kv_heads, page_tokens, head_dim], scales [n_pages, n_kv_heads, page_tokens]."""
        shape = (self.n_pages, self.n_kv_heads, self.page_tokens)
        for t, name in ((k, "k"), (v, "v")):
            if tuple(self._array(t, self._elem, name, 4).shape) != shape + (self.head_dim,):
                raise ValueError(f"{name}: expected {shape + (self.head_dim,)}, got {tuple(t.shape)}")
        if self.cache != "16":
            for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
                if t is None or tuple(self._array(t, self._torch.float32, name, 3).shape) != shape:
                    raise ValueError(f"{name}: expected float32 {shape}")
        ptr = [t.data_ptr() if t is not None else None for t in (k, v, k_scale, v_scale)]
        return _Record(KvPages(*ptr), (k, v, k_scale, v_scale), self._caches)

    def batch(self, q_start, kv_len, page_table, n_tokens, max_q_len, max_kv_len):
        """One step's sequences (device int32 tensors) and their host bounds."""
        i32 = self._torch.int32
        n = self._array(kv_len, i32, "kv_len").shape[0]
        if self._array(q_start, i32, "q_start").shape[0] != n + 1:
            raise ValueError(f"q_start: expected {n + 1} entries, got {q_start.shape[0]}")
        if tuple(self._array(page_table, i32, "page_table", 2).shape) != (n, self.max_pages):
            raise ValueError(f"page_table: expected {(n, self.max_pages)}, got {tuple(page_table.shape)}")
        tensors = (q_start, kv_len, page_table)
        return _Record(SeqBatch(*(t.data_ptr() for t in tensors), n, int(n_tokens), int(max_q_len), int(max_kv_len)), tensors, self._batches, int(n_tokens))

    def shaping(self, history=None, history_start=None, prompt_len=None, repetition=None, presence=None, frequency=None,
                bias_id=None, bias_value=None, bias_start=None, mask=None, mask_index=None):
        """What `shape_logits` does to each row; parts left out are not applied.  Device tensors: int32 ids and offsets, float32
        factors, mask words as int32 [masks, words]."""
        torch = self._torch
        given = locals()
        tensors = []
        for name in SHAPING_ARRAYS:
            t = given[name]
            if t is not None:
                self._array(t, torch.float32 if name in ("repetition", "presence", "frequency", "bias_value") else torch.int32, name, 2 if name == "mask" else 1)
            tensors.append(t)
        if bias_id is not None and bias_value is not None and bias_id.shape != bias_value.shape:
            raise ValueError("bias_id and bias_value differ in length")
        rows = {t.shape[0] - (name in ("history_start", "bias_start")) for name, t in given.items()
                if t is not None and name in ("history_start", "prompt_len", "repetition", "presence", "frequency", "bias_start", "mask_index")}
        if len(rows) > 1:
            raise ValueError(f"the per-row arrays name different numbers of rows: {sorted(rows)}")
        # An array that was given but is empty has no memory to point to; the kernels have to know of it all the same, to tell who asks for what it
        # does not hold, and never read it (its length is 0).
        # (A history or bias list without offsets, though, is none.)
        nowhere, alone = self._ws.data_ptr(), {"history": history_start is None, "bias_id": bias_start is None}
        c = ShapingRecord(*(None if t is None else t.data_ptr() if t.numel() else None if alone.get(name) else nowhere for name, t in zip(SHAPING_ARRAYS, tensors)),
                          history.shape[0] if history is not None else 0, bias_id.shape[0] if bias_id is not None else 0,
                          mask.shape[0] if mask is not None else 0, mask.shape[1] if mask is not None else 0)
        return _Record(c, tuple(tensors), self._shapings, rows.pop() if rows else None)

    # ---- the operators ----------------------------------------------------------------------
    def append(self, cache, batch, k, v):
        """Write the new tokens' keys and values ([n_tokens, n_kv_heads, head_dim]) to their pages."""
        self._fits(cache, self._caches)
        self._fits(batch, self._batches)
        ks, vs = self._rows(k, self.n_kv_heads, "k"), self._rows(v, self.n_kv_heads, "v")
        if k.shape[0] != batch.extra or v.shape[0] != batch.extra:
            raise ValueError(f"k and v must hold the batch's {batch.extra} tokens")
        if self._aside():
            self._used(k, v, *cache.tensors, *batch.tensors)
        self._check(self._lib.wwws_cache_append(self._h, batch.at, cache.at, k.data_ptr(), ks, v.data_ptr(), vs))

    def read(self, cache, batch, row_start, n_rows):
        """Whole sequences back: (k, v), each [n_rows, n_kv_heads, head_dim]; sequence i's tokens from row row_start[i] on."""
        self._fits(cache, self._caches)
        self._fits(batch, self._batches)
        self._array(row_start, self._torch.int32, "row_start")
        if row_start.shape[0] != batch.c.n_seqs + 1:
            raise ValueError(f"row_start: expected {batch.c.n_seqs + 1} entries, got {row_start.shape[0]}")
        aside = self._aside()
        kv = self._empty((2, n_rows, self.n_kv_heads, self.head_dim), self.dtype, aside)
        if aside:
            self._used(row_start, *cache.tensors, *batch.tensors)
        k, v = kv.unbind(0)
        self._check(self._lib.wwws_cache_read(self._h, batch.at, cache.at, row_start.data_ptr(), n_rows, k.data_ptr(), v.data_ptr()))
        return k, v

    def attend(self, cache, batch, q, out=None, scale=None, window=0, sinks=0):
        """Attention of the new tokens ([n_tokens, n_heads, head_dim]) over the cache; scale defaults to head_dim ** -0.5."""
        self._fits(cache, self._caches)
        self._fits(batch, self._batches)
        qs = self._rows(q, self.n_heads, "q")
        aside = self._aside()
        if out is None:
            out, os = self._empty(q.shape, self.dtype, aside), self.n_heads * self.head_dim
        else:
            os = self._rows(out, self.n_heads, "out")
        if window < 0 or sinks < 0:
            raise ValueError(f"window and sinks must be 0 or more, got {window} and {sinks}")
        if q.shape[0] != batch.extra or out.shape[0] != batch.extra:
            raise ValueError(f"q and out must hold the batch's {batch.extra} tokens")
        if aside:
            self._used(q, out, *cache.tensors, *batch.tensors)
        self._check(self._lib.wwws_attend(self._h, batch.at, cache.at, q.data_ptr(), qs, out.data_ptr(), os, self._scale if scale is None else scale, window, sinks))
        return out

    def shape_logits(self, logits, shaping, out=None, tokens=True):
        """(shaped logits, token per row): penalties, biases and masks on logits [rows, vocab] (bf16, f16 or f32)."""
        self._fits(shaping, self._shapings)
        dtype = self._codes.get(logits.dtype)
        if logits.dim() != 2 or dtype is None or logits.device != self.device or logits.stride(1) != 1 and logits.shape[1] > 1:
            raise ValueError(f"logits: expected [rows, vocab] of bf16, f16 or f32 with packed rows on {self.device}")
        rows, vocab = logits.shape
        if shaping.extra is not None and shaping.extra != rows:
            raise ValueError(f"the shaping names {shaping.extra} rows, logits has {rows}")
        aside = self._aside()
        if out is None:
            out = self._empty((rows, vocab), logits.dtype, aside)
        elif out.shape != logits.shape or out.dtype != logits.dtype or out.stride(1) != 1 and vocab > 1 or out.device != self.device:
            raise ValueError("out: expected the shape and type of logits")
        token = self._empty((rows,), self._torch.int32, aside) if tokens else None
        if aside:
            self._used(logits, out, token, *shaping.tensors)
        self._check(self._lib.wwws_shape_logits(self._h, shaping.at, rows, vocab, dtype, logits.data_ptr(), logits.stride(0) if rows > 1 else vocab,
                                                out.data_ptr(), out.stride(0) if rows > 1 else vocab, token.data_ptr() if tokens else None))
        return out, token

    def sync(self):
        """Wait for the stream; raises if a kernel met an id, offset or length out of range."""
        self._check(self._lib.wwws_backend_sync(self._h))
