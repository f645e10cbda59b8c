"""ctypes binding of libsa_prefill.so: argument marshalling only.

Every step of the path runs in the HIP library; PyTorch is used for device
memory and streams.  The library must be present: nothing here falls back to
another implementation.
"""
from __future__ import annotations

import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsa_prefill.so")

SA_PATTERN_AUTO, SA_TRIANGULAR, SA_INTERVAL_SLASH, SA_BLOCK_CLUSTER = -1, 0, 1, 2
SA_ROTARY_HALF, SA_ROTARY_INTERLEAVED = 0, 1
SA_SCALING_NONE, SA_SCALING_LINEAR, SA_SCALING_BASE, SA_SCALING_WAVELENGTH, SA_SCALING_RAMP = 0, 1, 2, 3, 4
SA_CACHE_E4M3, SA_CACHE_E5M2 = 0, 1
_STATUS = {0: "SA_OK", 1: "SA_ERR_INVALID_ARG", 2: "SA_ERR_UNSUPPORTED",
           3: "SA_ERR_BUFFER_TOO_SMALL", 4: "SA_ERR_HIP"}


class SaError(RuntimeError):
    def __init__(self, status, msg=""):
        super().__init__(f"{_STATUS.get(status, status)} {msg}".strip())
        self.status = status


class SaConfig(C.Structure):
    _fields_ = [("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("seq_len", C.c_int32), ("block", C.c_int32), ("last_q", C.c_int32),
                ("softmax_scale", C.c_float),
                ("sink_blocks", C.c_int32), ("local_blocks", C.c_int32),
                ("k_vertical", C.c_int32), ("k_slash", C.c_int32), ("k_blocks", C.c_int32),
                ("probe_v", C.c_int32), ("probe_s", C.c_int32), ("lift_num", C.c_int32),
                ("lift_den", C.c_int32),
                ("q_head_stride", C.c_int64), ("q_row_stride", C.c_int64),
                ("kv_head_stride", C.c_int64), ("kv_row_stride", C.c_int64),
                ("block_select", C.c_int32), ("diagonal_select", C.c_int32),
                ("lazy_block_map", C.c_int32)]


class SaScores(C.Structure):
    _fields_ = [("v", C.c_void_p), ("s", C.c_void_p), ("blk", C.c_void_p)]


class SaIndex(C.Structure):
    _fields_ = [("pattern", C.c_void_p), ("n_cols", C.c_void_p), ("cols", C.c_void_p),
                ("n_offs", C.c_void_p), ("offs", C.c_void_p), ("rowptr", C.c_void_p),
                ("blkcols", C.c_void_p)]


class SaRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("head_stride", C.c_int64), ("row_stride", C.c_int64)]


class SaRotaryConfig(C.Structure):
    _fields_ = [("rotary_dim", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32), ("transposed", C.c_int32),
                ("theta", C.c_double), ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double),
                ("original_len", C.c_double), ("amplitude", C.c_double)]


class SaCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("k_open", C.c_void_p), ("v_open", C.c_void_p), ("capacity", C.c_int64), ("type", C.c_int32)]


_lib = None


def library():
    """Load libsa_prefill.so (built by paper_2412_06198_amd.build); fail loudly if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise SaError(4, f"{LIB_PATH} is missing: run `python -m paper_2412_06198_amd.build`")
        lib = C.CDLL(LIB_PATH)
        vp, st = C.c_void_p, C.c_int
        lib.sa_version.restype = C.c_char_p
        lib.sa_last_error.restype = C.c_char_p
        lib.sa_last_error.argtypes = [vp]
        lib.sa_default_budgets.argtypes = [C.POINTER(SaConfig), C.c_double]
        lib.sa_create.argtypes = [C.POINTER(SaConfig), C.POINTER(vp)]
        lib.sa_destroy.argtypes = [vp]
        lib.sa_destroy.restype = None
        lib.sa_scores_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
        lib.sa_index_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
        lib.sa_workspace_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
        lib.sa_set_workspace.argtypes = [vp, vp, C.c_size_t]
        lib.sa_estimate_patterns.argtypes = [vp, vp, vp, SaScores, vp]
        lib.sa_build_index.argtypes = [vp, SaScores, C.POINTER(C.c_int32), SaIndex, vp]
        lib.sa_estimate_and_index.argtypes = [vp, vp, vp, SaScores, C.POINTER(C.c_int32), SaIndex, vp]
        lib.sa_sparse_prefill.argtypes = [vp, vp, vp, vp, SaIndex, vp, vp]
        lib.sa_sparse_prefill_counted.argtypes = [vp, vp, vp, vp, SaIndex, vp, vp, vp]
        lib.sa_sparse_decode.argtypes = [vp, vp, vp, vp, SaIndex, C.c_int64, vp, vp]
        lib.sa_sparse_decode_static.argtypes = [vp, vp, vp, vp, SaIndex, C.c_int64, vp, vp]
        lib.sa_search_scratch_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
        lib.sa_search_patterns.argtypes = [vp, vp, vp, vp, SaScores, C.c_int64, C.c_int64, vp, C.c_size_t,
                                           C.POINTER(SaSearchHead), vp]
        lib.sa_rotary_create.argtypes = [C.POINTER(SaRotaryConfig), C.POINTER(vp)]
        lib.sa_rotary_destroy.argtypes = [vp]
        lib.sa_rotary_destroy.restype = None
        lib.sa_rotary_embed.argtypes = [vp, vp, SaRows, SaRows, C.c_int64, C.c_int64, vp, SaRows, SaRows, vp]
        lib.sa_cache_bytes.argtypes = [vp, C.c_int64, C.POINTER(C.c_size_t)]
        lib.sa_cache_append.argtypes = [vp, C.POINTER(SaCache), SaRows, SaRows, C.c_int64, C.c_int64, vp]
        lib.sa_cache_decode.argtypes = [vp, C.POINTER(SaCache), vp, SaIndex, C.c_int64, vp, vp]
        lib.sa_cache_attend_scratch_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
        lib.sa_cache_attend_plan.argtypes = [vp, C.c_int64, C.c_int64, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        lib.sa_cache_attend.argtypes = [vp, C.POINTER(SaCache), SaRows, C.c_int64, C.c_int64, SaRows, vp, C.c_size_t, vp]
        for f in ("sa_rotary_create", "sa_rotary_embed", "sa_cache_bytes", "sa_cache_append", "sa_cache_decode",
                  "sa_cache_attend_scratch_bytes", "sa_cache_attend_plan", "sa_cache_attend"):
            getattr(lib, f).restype = st
        for f in ("sa_default_budgets", "sa_create", "sa_scores_bytes", "sa_index_bytes",
                  "sa_workspace_bytes", "sa_set_workspace", "sa_estimate_patterns",
                  "sa_build_index", "sa_sparse_prefill", "sa_sparse_prefill_counted",
                  "sa_search_scratch_bytes", "sa_search_patterns", "sa_sparse_decode",
                  "sa_sparse_decode_static", "sa_estimate_and_index"):
            getattr(lib, f).restype = st
        _lib = lib
    return _lib


def _ptr(x):
    """Device address of a torch tensor, or an int passed through."""
    if x is None:
        return None
    return x if isinstance(x, int) else x.data_ptr()


def _check(status, ctx=None):
    if status != 0:
        msg = library().sa_last_error(ctx).decode() if ctx else ""
        raise SaError(status, msg)


def sa_version() -> str:
    return library().sa_version().decode()


def sa_last_error(ctx) -> str:
    return library().sa_last_error(ctx).decode()


def sa_default_budgets(cfg: SaConfig, keep_fraction: float) -> SaConfig:
    _check(library().sa_default_budgets(C.byref(cfg), keep_fraction))
    return cfg


def sa_create(cfg: SaConfig):
    ctx = C.c_void_p()
    _check(library().sa_create(C.byref(cfg), C.byref(ctx)))
    return ctx


def sa_destroy(ctx):
    library().sa_destroy(ctx)


def sa_scores_bytes(ctx):
    out = (C.c_size_t * 3)()
    _check(library().sa_scores_bytes(ctx, out), ctx)
    return list(out)


def sa_index_bytes(ctx):
    out = (C.c_size_t * 7)()
    _check(library().sa_index_bytes(ctx, out), ctx)
    return list(out)


def sa_workspace_bytes(ctx) -> int:
    out = C.c_size_t()
    _check(library().sa_workspace_bytes(ctx, C.byref(out)), ctx)
    return out.value


def sa_set_workspace(ctx, dev, nbytes):
    _check(library().sa_set_workspace(ctx, _ptr(dev), nbytes), ctx)


def sa_estimate_patterns(ctx, Q, K, scores: SaScores, stream=None):
    _check(library().sa_estimate_patterns(ctx, _ptr(Q), _ptr(K), scores, stream), ctx)


def _override_array(pattern_override, n_q_heads):
    """Host int32 array of exactly n_q_heads entries (the library reads that many), or None."""
    if pattern_override is None:
        return None
    if n_q_heads is None or len(pattern_override) != n_q_heads:
        raise SaError(1, f"pattern_override needs one entry per query head ({n_q_heads}), got {len(pattern_override)}")
    return (C.c_int32 * n_q_heads)(*[int(p) for p in pattern_override])


def sa_build_index(ctx, scores: SaScores, pattern_override, index: SaIndex, stream=None, n_q_heads=None):
    ov = _override_array(pattern_override, n_q_heads)
    _check(library().sa_build_index(ctx, scores, ov, index, stream), ctx)


def sa_estimate_and_index(ctx, Q, K, scores: SaScores, pattern_override, index: SaIndex, stream=None,
                          n_q_heads=None):
    ov = _override_array(pattern_override, n_q_heads)
    _check(library().sa_estimate_and_index(ctx, _ptr(Q), _ptr(K), scores, ov, index, stream), ctx)


def sa_sparse_prefill(ctx, Q, K, V, index: SaIndex, O, stream=None):
    _check(library().sa_sparse_prefill(ctx, _ptr(Q), _ptr(K), _ptr(V), index, _ptr(O), stream), ctx)


def sa_sparse_prefill_counted(ctx, Q, K, V, index: SaIndex, O, counters, stream=None):
    _check(library().sa_sparse_prefill_counted(ctx, _ptr(Q), _ptr(K), _ptr(V), index, _ptr(O),
                                               _ptr(counters), stream), ctx)


def sa_sparse_decode(ctx, q, K, V, index: SaIndex, pos, o, stream=None):
    _check(library().sa_sparse_decode(ctx, _ptr(q), _ptr(K), _ptr(V), index, int(pos), _ptr(o), stream), ctx)


def sa_sparse_decode_static(ctx, q, K, V, index: SaIndex, pos, o, stream=None):
    _check(library().sa_sparse_decode_static(ctx, _ptr(q), _ptr(K), _ptr(V), index, int(pos), _ptr(o), stream),
           ctx)


class SaSearchHead(C.Structure):
    _fields_ = [("pattern", C.c_int32), ("param", C.c_int32 * 3), ("pairs", C.c_int64 * 3),
                ("err", C.c_double * 3)]


def sa_search_scratch_bytes(ctx) -> int:
    out = C.c_size_t()
    _check(library().sa_search_scratch_bytes(ctx, C.byref(out)), ctx)
    return out.value


def sa_search_patterns(ctx, Q, K, V, scores: SaScores, target_pairs, eps_pairs, scratch, scratch_bytes,
                       n_heads, stream=None):
    out = (SaSearchHead * n_heads)()
    _check(library().sa_search_patterns(ctx, _ptr(Q), _ptr(K), _ptr(V), scores, C.c_int64(int(target_pairs)),
                                        C.c_int64(int(eps_pairs)), _ptr(scratch), C.c_size_t(scratch_bytes),
                                        out, stream), ctx)
    return [{"pattern": int(r.pattern), "param": list(r.param), "pairs": list(r.pairs), "err": list(r.err)}
            for r in out]


def sa_rotary_create(cfg: SaRotaryConfig):
    rotary = C.c_void_p()
    _check(library().sa_rotary_create(C.byref(cfg), C.byref(rotary)))
    return rotary


def sa_rotary_destroy(rotary):
    library().sa_rotary_destroy(rotary)


def sa_rotary_embed(ctx, rotary, Q: SaRows, K: SaRows, n, pos, positions, Q_out: SaRows, K_out: SaRows, stream=None):
    """Q, K, Q_out, K_out as _rows makes them; an empty SaRows() leaves a side out."""
    handle = rotary.handle if isinstance(rotary, Rotary) else rotary
    _check(library().sa_rotary_embed(ctx, handle, Q, K, n, pos, _ptr(positions), Q_out, K_out, stream), ctx)


def sa_cache_bytes(ctx, capacity):
    out = (C.c_size_t * 6)()
    _check(library().sa_cache_bytes(ctx, capacity, out))
    return list(out)


def _cache(cache):
    return cache.struct() if isinstance(cache, Cache) else cache


def sa_cache_append(ctx, cache, K: SaRows, V: SaRows, n, pos, stream=None):
    _check(library().sa_cache_append(ctx, _cache(cache), K, V, n, pos, stream), ctx)


def sa_cache_decode(ctx, cache, q, index: SaIndex, pos, o, stream=None):
    _check(library().sa_cache_decode(ctx, _cache(cache), _ptr(q), index, pos, _ptr(o), stream), ctx)


def sa_cache_attend_scratch_bytes(ctx) -> int:
    out = C.c_size_t()
    _check(library().sa_cache_attend_scratch_bytes(ctx, C.byref(out)), ctx)
    return out.value


def sa_cache_attend_plan(ctx, n, pos):
    """(query rows of a workgroup, splits of the keys) of sa_cache_attend at these sizes."""
    rows, splits = C.c_int32(), C.c_int32()
    _check(library().sa_cache_attend_plan(ctx, n, pos, C.byref(rows), C.byref(splits)))
    return rows.value, splits.value


def sa_cache_attend(ctx, cache, Q: SaRows, n, pos, O: SaRows, scratch, scratch_bytes, stream=None):
    _check(library().sa_cache_attend(ctx, _cache(cache), Q, n, pos, O, _ptr(scratch), scratch_bytes, stream), ctx)


class Rotary:
    """Frequencies of a rotation; the keywords are the fields of sa_rotary_config."""

    def __init__(self, **config):
        self.handle = None
        cfg = SaRotaryConfig()
        for k, v in config.items():
            if k not in _ROTARY_FIELDS:
                raise SaError(1, f"sa_rotary_config has no field {k}")
            setattr(cfg, k, v)
        self.cfg = cfg
        self.handle = sa_rotary_create(cfg)

    def __del__(self):
        try:
            if self.handle is not None:
                sa_rotary_destroy(self.handle)
                self.handle = None
        except Exception:
            pass


_NO_ROWS = SaRows()
_ROTARY_FIELDS = {name for name, _ in SaRotaryConfig._fields_}


class Cache:
    """The six buffers of an 8-bit key/value cache (see sa_cache in include/sa.h): k, v uint8 [n_kv_heads, capacity, 128],
    k_scale, v_scale fp32 [n_kv_heads, capacity / block], k_open, v_open bf16 [n_kv_heads, block, 128], contiguous."""

    def __init__(self, k, v, k_scale, v_scale, k_open, v_open, cache_type=SA_CACHE_E4M3):
        if k.ndim != 3 or k_open.ndim != 3 or k_open.shape[1] == 0:
            raise SaError(1, "k and k_open of a cache are [n_kv_heads, capacity, 128] and [n_kv_heads, block, 128]")
        heads, capacity, d = k.shape
        block = k_open.shape[1]
        want = [(heads, capacity, d)] * 2 + [(heads, capacity // block)] * 2 + [(heads, block, d)] * 2
        self.tensors = (k, v, k_scale, v_scale, k_open, v_open)
        for t, shape, size in zip(self.tensors, want, (1, 1, 4, 4, 2, 2)):
            if tuple(t.shape) != shape or t.element_size() != size or not t.is_contiguous() or t.device != k.device:
                raise SaError(1, f"a cache buffer is not a contiguous tensor of {shape} with {size} bytes an element on {k.device}")
        if d != 128 or capacity % block:
            raise SaError(1, "a cache holds rows of 128 elements and whole blocks")
        self.k, self.v, self.k_scale, self.v_scale, self.k_open, self.v_open = self.tensors
        self.heads, self.capacity, self.block, self.type, self.device = heads, capacity, block, cache_type, k.get_device()
        self._struct = SaCache(*[t.data_ptr() for t in self.tensors], capacity, cache_type)

    def struct(self):
        return self._struct


def _rows(t, shape, bf16, device, what):
    """A bf16 tensor of `shape` [heads, n, 128] on GPU `device` as sa_rows; its last dimension adjacent, any order of the others."""
    if t.shape != shape or t.dtype is not bf16 or t.get_device() != device:
        raise SaError(1, f"{what} must be a bf16 tensor {list(shape)} on the session's device {device}, not {t.dtype} {list(t.shape)} on {t.device}")
    heads, row, one = t.stride()
    if one != 1 or (heads <= 0 and row <= 0 and shape[0] * shape[1] > 1):  # two zeros would stand for contiguous rows
        raise SaError(1, f"{what} must have adjacent elements, and not one row for all")
    return SaRows(t.data_ptr(), heads, row)


class Session:
    """Owns a context plus the torch-allocated score / index / workspace buffers of one shape."""

    def __init__(self, n_q_heads, n_kv_heads, seq_len, block, last_q, keep=None, device="cuda:0",
                 **budgets):
        import torch

        self.torch = torch
        self.device = torch.device(device)
        self._known_index = None
        self._attend_scratch = None
        self._get_device = torch._C._cuda_getDevice
        self._bf16, self._hq, self._hkv, self._block = torch.bfloat16, n_q_heads, n_kv_heads, block
        self._lib = library()
        self._raw_stream = torch._C._cuda_getCurrentRawStream  # current_stream() without the object around it
        cfg = SaConfig()
        cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim = n_q_heads, n_kv_heads, 128
        cfg.seq_len, cfg.block, cfg.last_q = seq_len, block, last_q
        if keep is not None:
            sa_default_budgets(cfg, keep)
        for k, v in budgets.items():
            setattr(cfg, k, v)
        self.cfg = cfg
        self.ctx = sa_create(cfg)
        i32, f32 = torch.int32, torch.float32
        sb = sa_scores_bytes(self.ctx)
        ib = sa_index_bytes(self.ctx)
        H, N, nb = n_q_heads, seq_len, seq_len // block
        dev = self.device
        self.v = torch.empty((H, N), dtype=f32, device=dev)
        self.s = torch.empty((H, N), dtype=f32, device=dev)
        self.blk = torch.empty((H, nb, nb), dtype=f32, device=dev)
        assert [self.v.nbytes, self.s.nbytes, self.blk.nbytes] == sb
        self.cap_b = ib[6] // (4 * H)
        self.pattern = torch.empty(H, dtype=i32, device=dev)
        self.n_cols = torch.empty(H, dtype=i32, device=dev)
        self.cols = torch.empty((H, cfg.k_vertical), dtype=i32, device=dev)
        self.n_offs = torch.empty(H, dtype=i32, device=dev)
        self.offs = torch.empty((H, cfg.k_slash), dtype=i32, device=dev)
        self.rowptr = torch.empty((H, nb + 1), dtype=i32, device=dev)
        self.blkcols = torch.empty((H, self.cap_b), dtype=i32, device=dev)
        assert [t.nbytes for t in self.index_tensors()] == ib
        self.ws = torch.empty(sa_workspace_bytes(self.ctx) + 256, dtype=torch.uint8, device=dev)
        self._gpu = self.ws.get_device()
        off = (-self.ws.data_ptr()) % 256
        sa_set_workspace(self.ctx, self.ws.data_ptr() + off, self.ws.nbytes - off)

    def index_tensors(self):
        return [self.pattern, self.n_cols, self.cols, self.n_offs, self.offs, self.rowptr,
                self.blkcols]

    def scores(self) -> SaScores:
        return SaScores(self.v.data_ptr(), self.s.data_ptr(), self.blk.data_ptr())

    def index(self) -> SaIndex:
        return SaIndex(*[t.data_ptr() for t in self.index_tensors()])

    def _index(self):
        """index() for the calls below: the struct of the last call while no buffer has been replaced.  A
        small call is bound by this side: 0.7 us here and 1.4 us through index()."""
        p = (self.pattern.data_ptr(), self.n_cols.data_ptr(), self.cols.data_ptr(), self.n_offs.data_ptr(),
             self.offs.data_ptr(), self.rowptr.data_ptr(), self.blkcols.data_ptr())
        known = self._known_index
        if known is None or known[0] != p:
            known = self._known_index = (p, SaIndex(*p))
        return known[1]

    def stream(self):
        return self._raw_stream(self._device_index())

    def _device_index(self):
        i = self.device.index
        return self.torch.cuda.current_device() if i is None else i

    def estimate(self, Q, K):
        sa_estimate_patterns(self.ctx, Q, K, self.scores(), self.stream())

    def build_index(self, pattern_override=None):
        sa_build_index(self.ctx, self.scores(), pattern_override, self._index(), self.stream(),
                       n_q_heads=self.cfg.n_q_heads)

    def estimate_and_index(self, Q, K, pattern_override=None):
        sa_estimate_and_index(self.ctx, Q, K, self.scores(), pattern_override, self._index(), self.stream(),
                              n_q_heads=self.cfg.n_q_heads)

    def prefill(self, Q, K, V, O):
        sa_sparse_prefill(self.ctx, Q, K, V, self._index(), O, self.stream())

    def prefill_counted(self, Q, K, V, O):
        """Returns (32x32 sub-tiles computed, diagonals among them; kept query-key pairs) of one prefill call."""
        cnt = self.torch.zeros(2, dtype=self.torch.int64, device=self.device)
        sa_sparse_prefill_counted(self.ctx, Q, K, V, self._index(), O, cnt, self.stream())
        self.torch.cuda.synchronize(self.device)
        return [int(x) for x in cnt.cpu()]

    def decode(self, q, K, V, pos, o):
        """One decode step at position pos >= seq_len over the current index."""
        sa_sparse_decode(self.ctx, q, K, V, self._index(), pos, o, self.stream())

    def decode_static(self, q, K, V, pos, o):
        """The same step through the entry point that keeps its partial results in the library's
        static device array (no workspace needed, nothing allocated)."""
        sa_sparse_decode_static(self.ctx, q, K, V, self._index(), pos, o, self.stream())

    def rotate(self, rotary, Q, K, Q_out, K_out, pos=0, positions=None):
        """Rotary positions of Q [n_q_heads, n, 128] and K [n_kv_heads, n, 128] (either may be None), positions pos,
        pos + 1, ... or an int32 tensor of n; the outputs may be the inputs."""
        device, bf16 = self._gpu, self._bf16
        if self._get_device() != device:  # the library launches on the current device
            with self.torch.cuda.device(device):
                return self.rotate(rotary, Q, K, Q_out, K_out, pos, positions)
        if Q is None and K is None or (Q is None) != (Q_out is None) or (K is None) != (K_out is None):
            raise SaError(1, "Q and Q_out, K and K_out go together, and one pair is needed")
        n = (K if Q is None else Q).shape[1]
        q = qo = k = ko = _NO_ROWS
        if Q is not None:
            shape = (self._hq, n, 128)
            q = _rows(Q, shape, bf16, device, "Q")
            qo = q if Q_out is Q else _rows(Q_out, shape, bf16, device, "Q_out")
        if K is not None:
            shape = (self._hkv, n, 128)
            k = _rows(K, shape, bf16, device, "K")
            ko = k if K_out is K else _rows(K_out, shape, bf16, device, "K_out")
        at = None
        if positions is not None:
            if (positions.dtype is not self.torch.int32 or positions.shape != (n,) or not positions.is_contiguous() or
                    positions.get_device() != device):
                raise SaError(1, "positions must be a contiguous int32 tensor on the session's device, one per row")
            at = positions.data_ptr()
        st = self._lib.sa_rotary_embed(self.ctx, rotary.handle, q, k, n, pos, at, qo, ko, self._raw_stream(device))
        if st:
            _check(st, self.ctx)

    def cache(self, capacity, cache_type=SA_CACHE_E4M3):
        """An empty 8-bit cache for `capacity` tokens (a multiple of block)."""
        sizes = sa_cache_bytes(self.ctx, capacity)
        h, b, t = self.cfg.n_kv_heads, self.cfg.block, self.torch
        kinds = [((h, capacity, 128), t.uint8)] * 2 + [((h, capacity // b), t.float32)] * 2 + [((h, b, 128), t.bfloat16)] * 2
        bufs = [t.empty(shape, dtype=kind, device=self.ws.device) for shape, kind in kinds]  # self.device may have no index
        assert [x.nbytes for x in bufs] == sizes
        return Cache(*bufs, cache_type)

    def _own(self, cache):
        """The cache's struct, if the cache fits the session."""
        if cache.heads != self._hkv or cache.block != self._block or cache.device != self._gpu:
            raise SaError(1, f"the cache has {cache.heads} heads and blocks of {cache.block} on device {cache.device}, "
                             f"the session {self._hkv} and {self._block} on {self._gpu}")
        return cache.struct()

    def append(self, cache, K, V, pos):
        """K, V [n_kv_heads, n, 128] behind the pos tokens that the cache holds.  To take tokens back across a block that a call
        has filled: copies of cache.k_open and cache.v_open from before it, put back, and append() again from its pos on."""
        device, struct = self._gpu, self._own(cache)
        if self._get_device() != device:
            with self.torch.cuda.device(device):
                return self.append(cache, K, V, pos)
        n = K.shape[1]
        shape = (self._hkv, n, 128)
        st = self._lib.sa_cache_append(self.ctx, struct, _rows(K, shape, self._bf16, device, "K"), _rows(V, shape, self._bf16, device, "V"),
                                       n, pos, self._raw_stream(device))
        if st:
            _check(st, self.ctx)

    def decode_cached(self, cache, q, pos, o):
        """decode() with K and V out of a cache that holds tokens 0..pos."""
        device, struct = self._gpu, self._own(cache)
        if self._get_device() != device:
            with self.torch.cuda.device(device):
                return self.decode_cached(cache, q, pos, o)
        shape, bf16 = (self._hq, 128), self._bf16
        for t in (q, o):
            if t.shape != shape or t.dtype is not bf16 or not t.is_contiguous() or t.get_device() != device:
                raise SaError(1, f"q and o must be contiguous bf16 tensors {list(shape)} on the session's device")
        sa_cache_decode(self.ctx, struct, q, self._index(), pos, o, self._raw_stream(device))

    def attend_scratch(self):
        """The session's scratch of attend(), allocated at the first use and kept: attend() calls that may overlap in time,
        replays of graphs on several streams among them, need sessions of their own."""
        if self._attend_scratch is None:
            size = sa_cache_attend_scratch_bytes(self.ctx)
            raw = self.torch.empty(size + 256, dtype=self.torch.uint8, device=self.ws.device)
            off = (-raw.data_ptr()) % 256
            self._attend_scratch = (raw, raw.data_ptr() + off, size)
        return self._attend_scratch

    def attend(self, cache, Q, pos, O):
        """Causal attention of the newest tokens, Q and O [n_q_heads, n, 128], over a cache that holds pos + n.  Partial results
        go through the session's one scratch, see attend_scratch(): calls that may overlap in time need sessions of their own."""
        device, struct = self._gpu, self._own(cache)
        if self._get_device() != device:
            with self.torch.cuda.device(device):
                return self.attend(cache, Q, pos, O)
        _, scratch, size = self._attend_scratch or self.attend_scratch()
        n = Q.shape[1]
        shape = (self._hq, n, 128)
        q = _rows(Q, shape, self._bf16, device, "Q")
        st = self._lib.sa_cache_attend(self.ctx, struct, q, n, pos, q if O is Q else _rows(O, shape, self._bf16, device, "O"), scratch, size,
                                       self._raw_stream(device))
        if st:
            _check(st, self.ctx)

    def search_patterns(self, Q, K, V, target_pairs, eps_pairs):
        """Alg. 1 on the scores of the last estimate(): one dict per head."""
        nbytes = sa_search_scratch_bytes(self.ctx)
        scratch = self.torch.empty(nbytes + 256, dtype=self.torch.uint8, device=self.device)
        off = (-scratch.data_ptr()) % 256
        return sa_search_patterns(self.ctx, Q, K, V, self.scores(), target_pairs, eps_pairs,
                                  scratch.data_ptr() + off, nbytes, self.cfg.n_q_heads, self.stream())

    def close(self):
        if self.ctx is not None:
            sa_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
