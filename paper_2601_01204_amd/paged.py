"""ctypes binding of the paged cache's part of the C ABI (include/kvx.h, argument marshalling only)."""
from __future__ import annotations

import ctypes as C
import threading

from .binding import KV_BF16, KvError, load_library

KV_F16, KV_E4M3 = 2, 3
KV_ROPE_HALF, KV_ROPE_INTERLEAVED = 0, 1
KV_ROPE_PLAIN, KV_ROPE_LINEAR, KV_ROPE_BASE, KV_ROPE_PARTS = 0, 1, 2, 3
KV_PAGED_BAD_PAGE, KV_PAGED_BAD_LENGTH = 1, 2


class KvPagedConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_q_heads", "n_kv_heads", "head_dim", "page_size", "dtype", "cache_dtype", "max_seqs", "max_tokens", "max_len", "max_evicted")] + [
        ("softmax_scale", C.c_float)] + [(n, C.c_int32) for n in ("rotary_dim", "rope_layout", "rope_scaling", "rope_original_len")] + [
        (n, C.c_double) for n in ("rope_base", "rope_factor", "rope_low_turns", "rope_high_turns")] + [
        ("rope_magnitude", C.c_float), ("rope_freqs", C.c_void_p)]


class KvRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("tok_stride", C.c_int64), ("head_stride", C.c_int64)]


class KvPagesStruct(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_stride", C.c_int64), ("slot_stride", C.c_int64), ("head_stride", C.c_int64),
                ("n_pages", C.c_int32), ("pages_per_seq", C.c_int32), ("page_table", C.c_void_p), ("table_stride", C.c_int64),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("weights", C.c_void_p), ("ids", C.c_void_p)]


class KvPagedBatchStruct(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_seqs", "n_tokens", "max_new", "max_len")] + [(n, C.c_void_p) for n in ("q_start", "kv_lens", "seen")]


_declared = False


def _library():
    global _declared
    lib = load_library()
    if not _declared:
        P, I = C.c_void_p, C.c_int32
        lib.kv_paged_init.argtypes = [P, P]
        lib.kv_paged_append.argtypes = [P] * 9
        lib.kv_paged_attend.argtypes = [P, P, P, P, P, P, I, I, P, P]
        lib.kv_paged_evict.argtypes = [P, P, P, I, I, I, P, P, P, P]
        lib.kv_paged_status.argtypes = [P, P]
        lib.kv_paged_destroy.argtypes = [P]
        lib.kv_paged_destroy.restype = None
        lib.kv_paged_last_error.argtypes = [P]
        lib.kv_paged_last_error.restype = C.c_char_p
        for name in ("init", "append", "attend", "evict", "status"):
            getattr(lib, "kv_paged_" + name).restype = C.c_int
        _declared = True
    return lib


def _current_device():
    import torch
    return torch.device("cuda", torch.cuda.current_device())


def _is(t, dtype):
    return str(t.dtype) == "torch." + dtype


def _int_array(t, name, n=None):
    if not _is(t, "int32") or t.dim() != 1 or not t.is_contiguous() or (n is not None and t.numel() != n):
        raise AssertionError(f"{name} must be a contiguous int32 vector" + ("" if n is None else f" of {n}"))
    return t.data_ptr()


class KvPages:
    """A pool of pages and the sequences' tables: kv_pages.  k_pages, v_pages: [pages, slots, heads, d], or with heads_first
    [pages, heads, slots, d], of the same strides; page_table: int32 [sequences, entries].  weights (fp32) and ids (int32):
    [pages, heads, slots], contiguous.  Keeps the tensors alive; describes them as they are now."""

    def __init__(self, k_pages, v_pages, page_table, heads_first=False, k_scale=None, v_scale=None, weights=None, ids=None):
        assert k_pages.dim() == 4 and k_pages.shape == v_pages.shape and k_pages.dtype == v_pages.dtype and k_pages.device == v_pages.device
        assert k_pages.stride() == v_pages.stride() and k_pages.stride(3) == 1, "k_pages and v_pages must have the same strides and contiguous channels"
        assert _is(page_table, "int32") and page_table.dim() == 2 and page_table.stride(1) == 1, "page_table must be int32 [sequences, entries]"
        assert page_table.shape[0] == 1 or page_table.stride(0) >= page_table.shape[1], "rows of page_table must not overlap"
        slot, head = (2, 1) if heads_first else (1, 2)
        n, self.n_heads, self.page_size, self.head_dim = k_pages.shape[0], k_pages.shape[head], k_pages.shape[slot], k_pages.shape[3]
        for t, name, dt in ((weights, "weights", "float32"), (ids, "ids", "int32")):
            assert t is None or (tuple(t.shape) == (n, self.n_heads, self.page_size) and _is(t, dt) and t.is_contiguous()), f"{name} must be a contiguous {dt} [pages, heads, slots]"
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            assert t is None or (tuple(t.shape) == (self.n_heads,) and _is(t, "float32") and t.is_contiguous()), f"{name} must be a float32 vector of the key heads"
        self.device, self.n_seqs = k_pages.device, page_table.shape[0]
        self.form = (self.n_heads, self.head_dim, self.page_size, str(k_pages.dtype))
        self.weights, self.ids = weights, ids
        for t in (page_table, k_scale, v_scale, weights, ids):
            assert t is None or t.device == self.device, "the pool's tensors must be on one device"
        self._keep = (k_pages, v_pages, page_table, k_scale, v_scale, weights, ids)
        d = self.head_dim
        # (a dimension of one element may carry any stride)
        strides = [k_pages.stride(i) if k_pages.shape[i] > 1 else max(d, -(-k_pages.stride(i) // 16) * 16) for i in (0, slot, head)]
        ptr = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
        self.struct = KvPagesStruct(k_pages.data_ptr(), v_pages.data_ptr(), *strides, n, page_table.shape[1], page_table.data_ptr(),
                                    max(page_table.stride(0), page_table.shape[1]), ptr(k_scale), ptr(v_scale), ptr(weights), ptr(ids))
        self.ref = C.byref(self.struct)


class KvPagedBatch:
    """The sequences of a call: kv_paged_batch.  q_start int32 [sequences + 1], kv_lens and seen int32 [sequences]."""

    def __init__(self, q_start, kv_lens, n_tokens, max_new, max_len, seen=None):
        self.n_seqs, self.n_tokens, self.device = kv_lens.numel(), n_tokens, kv_lens.device
        p_lens, p_start = _int_array(kv_lens, "kv_lens"), _int_array(q_start, "q_start", self.n_seqs + 1)
        p_seen = _int_array(seen, "seen", self.n_seqs) if seen is not None else None
        assert q_start.device == self.device and (seen is None or seen.device == self.device)
        self._keep = (q_start, kv_lens, seen)
        self.struct = KvPagedBatchStruct(self.n_seqs, n_tokens, max_new, max_len, p_start, p_lens, p_seen)
        self.ref = C.byref(self.struct)


class KvPaged:
    """Owner of one kv_paged handle.  Tensors only supply data_ptr(), strides, types and devices, which are checked against the handle's: its device is
    the one that was current when it was made.  Threads may share a handle: a call's launches are enqueued before another call's."""

    def __init__(self, rope_freqs=None, **cfg):
        self.lib = _library()
        c = KvPagedConfig()
        defaults = dict(head_dim=128, page_size=16, dtype=KV_BF16, cache_dtype=None, max_seqs=1, max_tokens=1, max_len=1)
        defaults.update(cfg)
        if defaults["cache_dtype"] is None:
            defaults["cache_dtype"] = defaults["dtype"]
        known = {n for n, _ in KvPagedConfig._fields_}
        for k, v in defaults.items():
            if k not in known:
                raise TypeError(f"KvPaged: unknown configuration field {k!r}")
            setattr(c, k, v)
        freqs = None
        if rope_freqs is not None:
            assert len(rope_freqs) == c.rotary_dim // 2, "rope_freqs must have rotary_dim / 2 entries"
            freqs = (C.c_double * max(1, len(rope_freqs)))(*[float(x) for x in rope_freqs])
            c.rope_freqs = C.cast(freqs, C.c_void_p)
        self.cfg = c
        self._h = C.c_void_p()
        rc = self.lib.kv_paged_init(C.byref(c), C.byref(self._h))
        if rc != 0:
            raise KvError(rc, self.lib.kv_paged_last_error(None).decode())
        c.rope_freqs = None
        self.device = _current_device()
        self._hq, self._hkv, self._d = c.n_q_heads, c.n_kv_heads, c.head_dim
        self._append, self._attend, self._evict = self.lib.kv_paged_append, self.lib.kv_paged_attend, self.lib.kv_paged_evict
        self._lock = threading.Lock()                     # of the records and the call: the library runs without the interpreter's lock
        self._records = [KvRows() for _ in range(4)]      # of the running call
        self._refs = [C.byref(r) for r in self._records]
        self._type = None                                 # the tensors' dtype, once one has been seen
        names = {KV_BF16: "torch.bfloat16", KV_F16: "torch.float16", KV_E4M3: "torch.float8_e4m3fn"}
        self._dtype, self._form = names[c.dtype], (c.n_kv_heads, c.head_dim, c.page_size, names[c.cache_dtype])

    def _check(self, rc):
        if rc != 0:
            raise KvError(rc, self.lib.kv_paged_last_error(self._h).decode())

    def _pages(self, pages, batch):
        if pages.form != self._form:
            raise AssertionError(f"the pool's (heads, channels, page size, type) are {pages.form}, the handle's {self._form}")
        if pages.device != self.device:
            raise AssertionError(f"the pool is on {pages.device}, the handle on {self.device}")
        if batch.device != pages.device or batch.n_seqs > pages.n_seqs:
            raise AssertionError("the batch's device or sequences are not the page table's")

    def _rows(self, t, heads, batch, name, place):
        """Address and strides of a call's tensor in the handle's record number `place` (a call takes microseconds, and so does making a record)."""
        n, d = batch.n_tokens, self._d
        if t.shape != (n, heads, d) or t.dtype is not self._type or t.device != batch.device:
            if t.shape != (n, heads, d) or str(t.dtype) != self._dtype or t.device != batch.device:
                raise AssertionError(f"{name} must be [{n}, {heads}, {d}] {self._dtype} on {batch.device}")
            self._type = t.dtype
        if n == 0:
            return None                                   # (an empty tensor has no address)
        ts, hs, one = t.stride()
        if one != 1:
            raise AssertionError(f"{name} must have contiguous channels")
        r = self._records[place]
        r.data = t.data_ptr()
        r.tok_stride = ts if n > 1 else d                 # (a dimension of one element may carry any stride)
        r.head_stride = hs if heads > 1 else d
        return self._refs[place]

    def append(self, pages, batch, k, v, q=None, q_out=None, positions=None, hip_stream: int = 0):
        """kv_paged_append.  k, v: [tokens, key heads, d]; q, q_out: [tokens, query heads, d] (q_out may be q); positions: int32 [tokens]."""
        self._pages(pages, batch)
        p = None
        if positions is not None:
            assert positions.device == batch.device
            p = _int_array(positions, "positions", batch.n_tokens)
        with self._lock:
            rq = self._rows(q, self._hq, batch, "q", 0) if q is not None else None
            ro = self._rows(q_out, self._hq, batch, "q_out", 1) if q_out is not None else None
            rc = self._append(self._h, pages.ref, batch.ref, p, rq, ro, self._rows(k, self._hkv, batch, "k", 2), self._rows(v, self._hkv, batch, "v", 3), hip_stream)
            if rc:
                self._check(rc)

    def attend(self, pages, batch, q, out, lse=None, causal=True, window: int = 0, weights_out=None, hip_stream: int = 0):
        """kv_paged_attend.  q, out: [tokens, query heads, d]; lse: fp32 [tokens, query heads]; weights_out: as pages.weights."""
        self._pages(pages, batch)
        p_lse = None
        if lse is not None:
            assert _is(lse, "float32") and lse.shape == (batch.n_tokens, self._hq) and lse.is_contiguous() and lse.device == batch.device, \
                "lse must be a contiguous float32 [tokens, query heads]"
            p_lse = lse.data_ptr()
        p_weights = None if weights_out is None else self._meta(pages, weights_out, pages.weights, "weights")
        with self._lock:
            rc = self._attend(self._h, pages.ref, batch.ref, self._rows(q, self._hq, batch, "q", 0), self._rows(out, self._hq, batch, "out", 1), p_lse,
                              1 if causal else 0, window, p_weights, hip_stream)
            if rc:
                self._check(rc)

    @staticmethod
    def _meta(pages, t, like, name):
        if t is None:
            return None
        assert like is None or (t.shape == like.shape and t.dtype == like.dtype and t.is_contiguous() and t.device == like.device), \
            f"{name}_out must be laid out as the pool's {name}"
        return t.data_ptr()

    def evict(self, pages, batch, budget: int, sinks: int = 0, recent: int = 0, weights_out=None, ids_out=None, lens_out=None, hip_stream: int = 0):
        """kv_paged_evict.  weights_out, ids_out: as pages.weights and pages.ids; lens_out: int32 [sequences]."""
        self._pages(pages, batch)
        p_lens = None
        if lens_out is not None:
            assert lens_out.device == batch.device
            p_lens = _int_array(lens_out, "lens_out", batch.n_seqs)
        p_weights, p_ids = self._meta(pages, weights_out, pages.weights, "weights"), self._meta(pages, ids_out, pages.ids, "ids")
        with self._lock:
            self._check(self._evict(self._h, pages.ref, batch.ref, budget, sinks, recent, p_weights, p_ids, p_lens, hip_stream))

    def status(self) -> int:
        """kv_paged_status: KV_PAGED_BAD_PAGE | KV_PAGED_BAD_LENGTH met since the last call (synchronises)."""
        f = C.c_int32(0)
        with self._lock:
            self._check(self.lib.kv_paged_status(self._h, C.byref(f)))
        return f.value

    def close(self):
        if self._h:
            self.lib.kv_paged_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
