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

With several drafted tokens or several beams per request:

    rotation = b.rotation(128, theta=1e6, q_weight=..., k_weight=...)
    q = b.rotate_append(cache, batch, q, k, v, rotation)     # norms, rotation and the write to the cache in one pass
    o = b.attend(cache, batch, q, tree=masks)                # the new tokens are a tree
    b.compact(caches, batch, path, path_len)                 # accepted tokens to their places, caches = b.caches([cache of each layer])
    score, parent, token = b.select_beams(logits, totals, beams=4, keep=8)
    refs, table, held, moves = b.fork(refs, table, held, source, keep, room)
    b.copy_pages(caches, moves)                              # the pages that two sequences would write

Calls are enqueued on the stream that was current at creation (or the one given).  Tensors that a caller fills on another
stream must be ready before the call; the binding records the backend's stream on them, so that their memory is not
handed out again before the call has run.
"""
from __future__ import annotations

import ctypes as C
from fractions import Fraction

from .binding import WwwsError, load

EXPORTS = ("wwws_backend_workspace_bytes", "wwws_create_backend", "wwws_destroy_backend", "wwws_cache_append", "wwws_cache_read",
           "wwws_attend", "wwws_attend_tree", "wwws_rotate", "wwws_rotate_append", "wwws_pages_fork", "wwws_cache_copy", "wwws_cache_compact",
           "wwws_beams_scratch_bytes", "wwws_select_beams", "wwws_shape_logits", "wwws_backend_sync", "wwws_backend_last_error")
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


class RotationRecord(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("turns", "axis", "q_weight", "k_weight")] + [("eps", C.c_float)] + [(k, C.c_uint32) for k in ("dim", "n_axes", "interleaved")]


class ForkRecord(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("refs", "refs_out", "table", "held", "source", "keep", "room", "table_out", "held_out", "moves")] + \
               [("n_old", C.c_uint32), ("n_new", C.c_uint32)]


# One turn in radians, to more digits than any frequency's 2^-64 of a turn needs.
TAU = Fraction(6283185307179586476925286766559005768394, 10 ** 39)

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
            "wwws_attend_tree": [vp, vp, vp, vp, u64, vp, u64, C.c_float, u32, u32, vp, u32],
            "wwws_rotate": [vp, vp, u32, vp, vp, u64, vp, u64, vp, u64, vp, u64],
            "wwws_rotate_append": [vp, vp, vp, vp, vp, vp, u64, vp, u64, vp, u64, vp, u64],
            "wwws_pages_fork": [vp, vp],
            "wwws_cache_copy": [vp, vp, u32, vp, u32],
            "wwws_cache_compact": [vp, vp, vp, u32, vp, vp, u32],
            "wwws_beams_scratch_bytes": [u32, u32, u32, u32, C.POINTER(u64)],
            "wwws_select_beams": [vp, u32, u32, u32, u32, vp, u64, vp, u32, vp, u64, vp, vp, vp],
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
        self._layers, self._rotations = ("list of caches", *self._caches[1:]), ("rotation", self.device, head_dim)
        self._h = None
        self._like, self._beam_bytes = {}, {}
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

    def _check_plain(self, status):
        """Of a call that has no handle."""
        if status:
            raise WwwsError(status, self._lib.wwws_backend_last_error(None).decode())

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
            # a new tensor like one that is kept costs half of one made from a shape, a type and a device; what is kept is one element, expanded
            like = self._like.get((shape, dtype))
            if like is None:
                if len(self._like) >= 256:
                    self._like.clear()
                like = self._like[shape, dtype] = self._torch.empty(1, dtype=dtype, device=self.device).expand(shape)
            return self._torch.empty_like(like)
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
        shape, stride = t.shape, t.stride()
        if t.dtype != self.dtype or len(shape) != 3 or shape[1] != heads or shape[2] != self.head_dim or t.device != self.device:
            raise ValueError(f"{name}: expected {self.dtype} [tokens, {heads}, {self.head_dim}] on {self.device}, got {t.dtype} {tuple(shape)} on {t.device}")
        if stride[2] != 1 or stride[1] != self.head_dim:
            raise ValueError(f"{name}: the heads of a token must be packed, got strides {stride}")
        return stride[0] if shape[0] > 1 else heads * self.head_dim

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

    def caches(self, caches):
        """The caches of a model's layers as one record, for what moves tokens in all of them."""
        for c in caches:
            self._fits(c, self._caches)
        return _Record((KvPages * len(caches))(*(c.c for c in caches)), tuple(t for c in caches for t in c.tensors), self._layers, len(caches))

    def rotation(self, dim, theta=10000.0, frequencies=None, axes=None, interleaved=False, q_weight=None, k_weight=None, eps=1e-6):
        """How queries and keys are turned: the first `dim` elements of a head, pair i by frequencies[i] radians per position (default
        theta ** (-2 i / dim)) along axis axes[i] of the positions (default the only one).  Pairs are (i, dim / 2 + i), interleaved (2 i, 2 i + 1).
        q_weight, k_weight: float32 [head_dim], the weights of a norm over the head before that."""
        torch = self._torch
        if dim < 16 or dim % 16 or dim > self.head_dim:
            raise ValueError(f"dim must be a multiple of 16, 16 .. {self.head_dim}, got {dim}")
        if frequencies is None:
            frequencies = [float(theta) ** (-2.0 * i / dim) for i in range(dim // 2)]
        axes = list(axes) if axes is not None else None
        if len(frequencies) != dim // 2 or axes is not None and len(axes) != dim // 2:
            raise ValueError(f"frequencies and axes must name {dim // 2} pairs")
        if axes is not None and not all(0 <= a < 8 for a in axes):
            raise ValueError("axes must be 0 .. 7")
        turns = [round(Fraction(float(f)) / TAU * 2 ** 64) % 2 ** 64 for f in frequencies]
        for t, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
            if t is not None and self._array(t, torch.float32, name).shape[0] != self.head_dim:
                raise ValueError(f"{name}: expected {self.head_dim} entries, got {t.shape[0]}")
        with torch.cuda.stream(self._stream):
            turns = torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in turns], dtype=torch.int64, device=self.device)
            axis = torch.tensor(axes, dtype=torch.uint8, device=self.device) if axes is not None else None
        n_axes = max(axes) + 1 if axes is not None else 1
        tensors = (turns, axis, q_weight, k_weight)
        return _Record(RotationRecord(*(None if t is None else t.data_ptr() for t in tensors), eps, dim, n_axes, int(bool(interleaved))), tensors, self._rotations, n_axes)

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

    def attend(self, cache, batch, q, out=None, scale=None, window=0, sinks=0, tree=None):
        """Attention of the new tokens ([n_tokens, n_heads, head_dim]) over the cache; scale defaults to head_dim ** -0.5.  (Single tokens and
        prompts may share a call, but calls of their own take less time.)
        tree: int32 [n_tokens, words], the new tokens are drafts behind the context and see those whose bits are set in their row (their
        ancestors and themselves); 32 places a word, lowest bit first.  With a tree the window hides context alone."""
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
        if tree is not None and self._array(tree, self._torch.int32, "tree", 2).shape[0] != batch.extra:
            raise ValueError(f"tree: expected a row for each of the batch's {batch.extra} tokens, got {tree.shape[0]}")
        if aside:
            self._used(q, out, tree, *cache.tensors, *batch.tensors)
        given = self._h, batch.at, cache.at, q.data_ptr(), qs, out.data_ptr(), os, self._scale if scale is None else scale, window, sinks
        self._check(self._lib.wwws_attend(*given) if tree is None else self._lib.wwws_attend_tree(*given, tree.data_ptr(), tree.shape[1]))
        return out

    def _given_or_new(self, out, like, heads, name, aside):
        if out is None:
            return self._empty(like.shape, self.dtype, aside), heads * self.head_dim
        if out.shape != like.shape:
            raise ValueError(f"{name}: expected {tuple(like.shape)}, got {tuple(out.shape)}")
        return out, self._rows(out, heads, name)

    def _positions(self, positions, n_tokens, rotation):
        if positions.dim() == 1 and rotation.extra == 1:
            positions = positions.unsqueeze(1)
        if tuple(self._array(positions, self._torch.int32, "positions", 2).shape) != (n_tokens, rotation.extra):
            raise ValueError(f"positions: expected {(n_tokens, rotation.extra)}, got {tuple(positions.shape)}")
        return positions

    def rotate(self, q, k, positions, rotation, q_out=None, k_out=None):
        """(q, k) normed and turned: q [n_tokens, n_heads, head_dim], k [n_tokens, n_kv_heads, head_dim], positions int32 [n_tokens] or
        [n_tokens, axes].  An output may be its input."""
        self._fits(rotation, self._rotations)
        qs, ks = self._rows(q, self.n_heads, "q"), self._rows(k, self.n_kv_heads, "k")
        n = q.shape[0]
        if k.shape[0] != n:
            raise ValueError(f"q and k hold different numbers of tokens: {n} and {k.shape[0]}")
        positions = self._positions(positions, n, rotation)
        aside = self._aside()
        q_out, qos = self._given_or_new(q_out, q, self.n_heads, "q_out", aside)
        k_out, kos = self._given_or_new(k_out, k, self.n_kv_heads, "k_out", aside)
        if aside:
            self._used(q, k, q_out, k_out, positions, *rotation.tensors)
        self._check(self._lib.wwws_rotate(self._h, rotation.at, n, positions.data_ptr(), q.data_ptr(), qs, k.data_ptr(), ks, q_out.data_ptr(), qos, k_out.data_ptr(), kos))
        return q_out, k_out

    def rotate_append(self, cache, batch, q, k, v, rotation, positions=None, q_out=None):
        """The new tokens' queries normed and turned; their keys, normed and turned too, and values written to their pages.  positions
        default to the tokens' places in their sequences."""
        self._fits(cache, self._caches)
        self._fits(batch, self._batches)
        self._fits(rotation, self._rotations)
        qs, ks, vs = self._rows(q, self.n_heads, "q"), self._rows(k, self.n_kv_heads, "k"), self._rows(v, self.n_kv_heads, "v")
        if q.shape[0] != batch.extra or k.shape[0] != batch.extra or v.shape[0] != batch.extra:
            raise ValueError(f"q, k and v must hold the batch's {batch.extra} tokens")
        if positions is not None:
            positions = self._positions(positions, batch.extra, rotation)
        aside = self._aside()
        q_out, qos = self._given_or_new(q_out, q, self.n_heads, "q_out", aside)
        if aside:
            self._used(q, k, v, q_out, positions, *cache.tensors, *batch.tensors, *rotation.tensors)
        self._check(self._lib.wwws_rotate_append(self._h, batch.at, cache.at, rotation.at, positions.data_ptr() if positions is not None else None, q.data_ptr(), qs, k.data_ptr(), ks,
                                                 v.data_ptr(), vs, q_out.data_ptr(), qos))
        return q_out

    def compact(self, caches, batch, path, path_len):
        """Move new token path[i, m] (int32 [n_seqs, most], ascending) of sequence i to place m of its new tokens, m < path_len[i], in every layer."""
        self._fits(caches, self._layers)
        self._fits(batch, self._batches)
        n = batch.c.n_seqs
        if self._array(path, self._torch.int32, "path", 2).shape[0] != n or self._array(path_len, self._torch.int32, "path_len").shape[0] != n:
            raise ValueError(f"path and path_len must name the batch's {n} sequences")
        if self._aside():
            self._used(path, path_len, *caches.tensors, *batch.tensors)
        self._check(self._lib.wwws_cache_compact(self._h, batch.at, caches.at, caches.extra, path.data_ptr(), path_len.data_ptr(), path.shape[1]))

    def fork(self, refs, page_table, held, source, keep, room, in_place=False):
        """Sequences continued, dropped and given room: new sequence i takes the first keep[i] tokens of old sequence source[i] (none if
        below 0) and pages for room[i] tokens.  refs int32 [n_pages] counts who holds a page (0: free), page_table int32 [old, max_pages] and
        held int32 [old] are what the old sequences hold; all of them end.  Returns (refs, page_table, held, moves) of the new ones; moves
        int32 [new, 3] is for `copy_pages`.  in_place: the counts are written over refs."""
        i32, device = self._torch.int32, self.device
        n, m = self._array(source, i32, "source").shape[0], self._array(held, i32, "held").shape[0]
        for t, name, shape in ((refs, "refs", (self.n_pages,)), (page_table, "page_table", (m, self.max_pages)), (keep, "keep", (n,)), (room, "room", (n,))):
            if t.shape != shape or t.dtype != i32 or t.device != device or not t.is_contiguous():
                raise ValueError(f"{name}: expected a contiguous int32 tensor {shape} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
        aside = self._aside()
        refs_out = refs if in_place else self._empty((self.n_pages,), i32, aside)
        table_out, held_out, moves = self._empty((n, self.max_pages), i32, aside), self._empty((n,), i32, aside), self._empty((n, 3), i32, aside)
        if aside:
            self._used(refs, page_table, held, source, keep, room)
        record = ForkRecord(*(t.data_ptr() for t in (refs, refs_out, page_table, held, source, keep, room, table_out, held_out, moves)), m, n)
        self._check(self._lib.wwws_pages_fork(self._h, C.addressof(record)))
        return refs_out, table_out, held_out, moves

    def copy_pages(self, caches, moves):
        """Copy the first tokens of pages to other pages in every layer: moves int32 [n, 3] of (from, to, tokens), to < 0: none."""
        self._fits(caches, self._layers)
        if self._array(moves, self._torch.int32, "moves", 2).shape[1] != 3:
            raise ValueError(f"moves: expected [n, 3], got {tuple(moves.shape)}")
        if self._aside():
            self._used(moves, *caches.tensors)
        self._check(self._lib.wwws_cache_copy(self._h, caches.at, caches.extra, moves.data_ptr(), moves.shape[0]))

    def _logits(self, logits):
        dtype = self._codes.get(logits.dtype)
        if logits.dim() != 2 or dtype is None or logits.device != self.device or logits.stride(1) != 1 and logits.shape[1] > 1:
            raise ValueError(f"logits: expected [rows, vocab] of bf16, f16 or f32 with packed rows on {self.device}")
        return dtype

    def select_beams(self, logits, totals, beams, keep):
        """The best continuations of each request: logits [requests * beams, vocab] (bf16, f16 or f32), totals float32 [requests * beams].
        Returns (score float32, parent int32, token int32), each [requests, keep], best first: total + log-softmax of the logits, the row it
        continues, the token; -infinity, -1, -1 where a request has fewer."""
        dtype = self._logits(logits)
        rows, vocab = logits.shape
        if self._array(totals, self._torch.float32, "totals").shape[0] != rows:
            raise ValueError(f"totals: expected {rows} entries, got {totals.shape[0]}")
        if beams < 1 or rows % beams:
            raise ValueError(f"beams must divide the {rows} rows, got {beams}")
        if keep < 1:
            raise ValueError(f"keep must be 1 or more, got {keep}")
        nbytes = self._beam_bytes.get((rows, vocab, dtype, keep))
        if nbytes is None:
            asked = C.c_uint64()
            self._check_plain(self._lib.wwws_beams_scratch_bytes(rows, vocab, dtype, keep, C.byref(asked)))
            if len(self._beam_bytes) >= 256:
                self._beam_bytes.clear()
            nbytes = self._beam_bytes[rows, vocab, dtype, keep] = asked.value
        aside = self._aside()
        scratch = self._empty((nbytes,), self._torch.uint8, aside)
        shape = (rows // beams, keep)
        score, parent, token = self._empty(shape, self._torch.float32, aside), self._empty(shape, self._torch.int32, aside), self._empty(shape, self._torch.int32, aside)
        if aside:
            self._used(logits, totals)
        self._check(self._lib.wwws_select_beams(self._h, rows, beams, vocab, dtype, logits.data_ptr(), logits.stride(0) if rows > 1 else vocab, totals.data_ptr(), keep, scratch.data_ptr(),
                                                nbytes, score.data_ptr(), parent.data_ptr(), token.data_ptr()))
        return score, parent, token

    def shape_logits(self, logits, shaping, out=None, tokens=True):
        """(shaped logits, token per row): penalties, biases and masks on logits [rows, vocab] (bf16, f16 or f32)."""
        self._fits(shaping, self._shapings)
        dtype = self._logits(logits)
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
