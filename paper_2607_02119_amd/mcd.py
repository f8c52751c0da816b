"""Thin ctypes binding of libmcd (include/mcd.h).

Every function named ``mcd_*`` here marshals its arguments to the C function of
the same name; all computation happens in the library's HIP kernels.  PyTorch
supplies device memory and the stream.  ``Head`` is a small convenience wrapper
that keeps the borrowed weight tensors alive next to the handle.

Importing this module loads ``libmcd.so`` and raises if it has not been built
(``python -m paper_2607_02119_amd.build``); there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch  # loads the HIP runtime libmcd binds to (same soname, one runtime per process)

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmcd.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2607_02119_amd.build`")
_lib = ctypes.CDLL(_LIB_PATH)

MCD_OK, MCD_E_INVALID, MCD_E_UNSUPPORTED, MCD_E_WORKSPACE, MCD_E_HIP = range(5)
MCD_F32, MCD_BF16 = 0, 1
MCD_ROW_COND, MCD_ROW_UNCOND, MCD_ROW_SOLO, MCD_ROW_TEXT = 0, 1, 2, 3
MCD_DEV_BAD_PARAM, MCD_DEV_GRID_RANGE, MCD_DEV_BAD_PLAN, MCD_DEV_BAD_TOKEN = 1, 2, 4, 8
MCD_DEV_BAD_PAGE = 16
MCD_CACHE_PAGE = 64
MCD_MAX_K, MCD_MAX_V = 32, 4096

_vp = ctypes.c_void_p
_i32 = ctypes.c_int32


class mcd_head_desc(ctypes.Structure):
    _fields_ = [("H", _i32), ("K", _i32), ("V", _i32), ("pad_id", _i32),
                ("delays", _vp), ("dtype", ctypes.c_int), ("W", _vp), ("bias", _vp),
                ("V_text", _i32), ("W_text", _vp), ("V_stream", _vp), ("T_text", _i32)]


class mcd_batch_counts(ctypes.Structure):
    _fields_ = [("n_pairs", _i32), ("n_solo", _i32), ("n_text", _i32)]


class mcd_step_args(ctypes.Structure):
    _fields_ = [("R", _i32), ("counts", mcd_batch_counts), ("plan", _vp), ("hidden", _vp),
                ("cfg_w", _vp), ("temperature", _vp), ("top_k", _vp), ("top_p", _vp),
                ("rng_key", _vp), ("step", _vp), ("n_frames", _vp), ("grid_slot", _vp),
                ("seed", ctypes.c_uint64), ("tokens_out", _vp), ("frame_grid", _vp),
                ("modality_out", _vp), ("n_slots", _i32), ("F_max", _i32), ("scores", _vp), ("workspace", _vp),
                ("workspace_bytes", ctypes.c_size_t)]


class mcd_next_input_args(ctypes.Structure):
    _fields_ = [("R", _i32), ("H", _i32), ("K", _i32), ("V", _i32), ("pad_id", _i32),
                ("dtype", ctypes.c_int), ("E", _vp), ("V_text", _i32), ("E_text", _vp),
                ("row_kind", _vp), ("tokens", _vp), ("out", _vp), ("workspace", _vp)]


class mcd_phase_desc(ctypes.Structure):
    _fields_ = [("n_bridge", _i32), ("bridge", _vp), ("audio_end", _i32), ("drain_steps", _i32)]


class mcd_sched_desc(ctypes.Structure):
    _fields_ = [("max_rows", _i32), ("token_budget", _i32), ("null_prompt_len", _i32),
                ("drain_steps", _i32), ("max_requests", _i32)]


class mcd_sched_request(ctypes.Structure):
    _fields_ = [("cfg_w", ctypes.c_float), ("prompt_len", _i32), ("text_len", _i32),
                ("n_frames", _i32)]


class mcd_sched_batch(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("row_req", _vp), ("row_member", _vp), ("row_slot", _vp),
                ("row_tokens", _vp), ("row_context", _vp), ("R", _i32), ("head_row", _vp),
                ("pair_map", _vp), ("row_kind", _vp), ("cfg_w", _vp), ("step", _vp),
                ("n_frames", _vp), ("grid_slot", _vp)]


class mcd_cache(ctypes.Structure):
    _fields_ = [("Hkv", _i32), ("D", _i32), ("n_slots", _i32), ("max_pages", _i32),
                ("n_pages", _i32), ("pages", _vp), ("table", _vp), ("weight", _vp)]


class mcd_cache_rows(ctypes.Structure):
    _fields_ = [("R", _i32), ("n_tokens", _i32), ("max_tokens", _i32), ("max_context", _i32),
                ("slot", _vp), ("context", _vp), ("start", _vp)]


class mcd_cache_attend_args(ctypes.Structure):
    _fields_ = [("Hq", _i32), ("dtype", ctypes.c_int), ("scale", ctypes.c_float), ("q", _vp),
                ("q_stride", ctypes.c_int64), ("out", _vp), ("out_stride", ctypes.c_int64),
                ("lse", _vp), ("weight_out", _vp), ("workspace", _vp),
                ("workspace_bytes", ctypes.c_size_t)]


class mcd_cache_evict_args(ctypes.Structure):
    _fields_ = [("R", _i32), ("max_length", _i32), ("keep", _i32), ("recent", _i32),
                ("slot", _vp), ("length", _vp), ("kept", _vp), ("length_out", _vp),
                ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t)]


def _sig(name, res, *args):
    f = getattr(_lib, name)
    f.restype = res
    f.argtypes = list(args)
    return f


_mcd_head_create = _sig("mcd_head_create", ctypes.c_int, ctypes.POINTER(mcd_head_desc),
                        ctypes.POINTER(_vp))
_mcd_head_destroy = _sig("mcd_head_destroy", None, _vp)
_mcd_sched_create = _sig("mcd_sched_create", ctypes.c_int, ctypes.POINTER(mcd_sched_desc),
                         ctypes.POINTER(_vp))
_mcd_sched_destroy = _sig("mcd_sched_destroy", None, _vp)
_mcd_sched_submit = _sig("mcd_sched_submit", ctypes.c_int, _vp,
                         ctypes.POINTER(mcd_sched_request), ctypes.POINTER(_i32))
_mcd_sched_plan = _sig("mcd_sched_plan", ctypes.c_int, _vp, ctypes.POINTER(mcd_sched_batch))
_mcd_sched_commit = _sig("mcd_sched_commit", ctypes.c_int, _vp, _vp, _i32, ctypes.POINTER(_i32))
_mcd_sched_counts = _sig("mcd_sched_counts", ctypes.c_int, _vp, ctypes.POINTER(_i32),
                         ctypes.POINTER(_i32))
_mcd_plan_words = _sig("mcd_plan_words", ctypes.c_size_t, _i32)
_mcd_batch_plan = _sig("mcd_batch_plan", ctypes.c_int, _vp, _i32, _vp, _vp, _vp, ctypes.c_size_t,
                       ctypes.POINTER(mcd_batch_counts))
_mcd_plan_sampled_row = _sig("mcd_plan_sampled_row", ctypes.c_int, _vp, _i32,
                             ctypes.POINTER(_i32), ctypes.POINTER(_i32))
_mcd_workspace_bytes = _sig("mcd_workspace_bytes", ctypes.c_size_t, _vp, _i32)
_mcd_head_step = _sig("mcd_head_step", ctypes.c_int, _vp, ctypes.POINTER(mcd_step_args), _vp)
_mcd_sample_step = _sig("mcd_sample_step", ctypes.c_int, _vp, ctypes.POINTER(mcd_step_args), _vp)
_mcd_head_logits = _sig("mcd_head_logits", ctypes.c_int, _vp, ctypes.POINTER(mcd_step_args), _vp)
_mcd_head_step_noalloc = _sig("mcd_head_step_noalloc", ctypes.c_int, _vp,
                              ctypes.POINTER(mcd_step_args), _vp)
_mcd_deinterleave = _sig("mcd_deinterleave", ctypes.c_int, _vp, _i32, _i32, _i32, _vp, _vp, _vp)
_mcd_interleave = _sig("mcd_interleave", ctypes.c_int, _vp, _i32, _i32, _i32, _vp, _i32, _vp, _vp)
_mcd_next_input = _sig("mcd_next_input", ctypes.c_int, ctypes.POINTER(mcd_next_input_args), _vp)
_mcd_phase_advance = _sig("mcd_phase_advance", ctypes.c_int, ctypes.POINTER(mcd_phase_desc), _i32,
                          _vp, _vp, _vp, _vp, _vp)
_mcd_read_device_status = _sig("mcd_read_device_status", ctypes.c_int, _vp,
                               ctypes.POINTER(ctypes.c_uint32), _vp)
_i64, _size = ctypes.c_int64, ctypes.c_size_t
_cache_p, _rows_p = ctypes.POINTER(mcd_cache), ctypes.POINTER(mcd_cache_rows)
_mcd_cache_page_bytes = _sig("mcd_cache_page_bytes", _size, _i32)
_mcd_cache_workspace_bytes = _sig("mcd_cache_workspace_bytes", _size, _cache_p, _rows_p, _i32)
_mcd_cache_append = _sig("mcd_cache_append", ctypes.c_int, _cache_p, _rows_p, ctypes.c_int, _vp,
                         _i64, _vp, _i64, _vp, _size, _vp)
_mcd_cache_read = _sig("mcd_cache_read", ctypes.c_int, _cache_p, _rows_p, ctypes.c_int, _vp,
                       _i64, _vp, _i64, _vp, _size, _vp)
_mcd_cache_attend = _sig("mcd_cache_attend", ctypes.c_int, _cache_p, _rows_p,
                         ctypes.POINTER(mcd_cache_attend_args), _vp)
_mcd_cache_evict = _sig("mcd_cache_evict", ctypes.c_int, _cache_p, _cache_p,
                        ctypes.POINTER(mcd_cache_evict_args), _vp)
_mcd_status_string = _sig("mcd_status_string", ctypes.c_char_p, ctypes.c_int)
_mcd_last_error = _sig("mcd_last_error", ctypes.c_char_p)

EXPORTED = ["mcd_head_create", "mcd_head_destroy", "mcd_plan_words", "mcd_batch_plan",
            "mcd_plan_sampled_row", "mcd_workspace_bytes", "mcd_head_step", "mcd_head_logits",
            "mcd_head_step_noalloc",
            "mcd_sample_step",
            "mcd_deinterleave", "mcd_interleave", "mcd_phase_advance", "mcd_next_input",
            "mcd_read_device_status",
            "mcd_sched_create", "mcd_sched_destroy", "mcd_sched_submit", "mcd_sched_plan",
            "mcd_sched_commit", "mcd_sched_counts",
            "mcd_cache_page_bytes", "mcd_cache_workspace_bytes", "mcd_cache_append",
            "mcd_cache_read", "mcd_cache_attend", "mcd_cache_evict",
            "mcd_status_string", "mcd_last_error"]


class McdError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        msg = _mcd_last_error().decode(errors="replace")
        super().__init__(f"{where}: {mcd_status_string(code)} ({msg})")


def _check(code, where):
    if code != MCD_OK:
        raise McdError(code, where)


def _ptr(t):
    """Device (or host numpy) pointer of an optional tensor / array."""
    if isinstance(t, torch.Tensor):
        return t.data_ptr()
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return int(t)


# torch.cuda.current_stream() builds a Stream object on every call (2.9 us); the raw handle of the
# same stream takes 0.2 us.  A torch built without a GPU has no such function, and the host-only
# calls need none (there _device() raises first).
_raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device


def _stream(stream):
    if stream is None:
        return _raw_stream(_device())
    return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else int(stream)


# ---------------------------------------------------------------------------
# C functions, one to one

def mcd_status_string(code):
    return _mcd_status_string(code).decode()


def mcd_last_error():
    return _mcd_last_error().decode(errors="replace")


def mcd_head_create(H, K, V, pad_id, delays, dtype, W, bias=None, V_text=0, W_text=None,
                    V_stream=None, T_text=0):
    d = np.ascontiguousarray(delays, dtype=np.int32)
    vs = None if V_stream is None else np.ascontiguousarray(V_stream, dtype=np.int32)
    desc = mcd_head_desc(H, K, V, pad_id, d.ctypes.data, dtype, _ptr(W), _ptr(bias), V_text,
                         _ptr(W_text), _ptr(vs), int(T_text))
    h = _vp()
    _check(_mcd_head_create(ctypes.byref(desc), ctypes.byref(h)), "mcd_head_create")
    return h


def mcd_head_destroy(h):
    _mcd_head_destroy(h)


def mcd_plan_words(R):
    return int(_mcd_plan_words(R))


def mcd_batch_plan(h, pair_map, row_kind):
    """Host plan of a batch -> (plan int32 numpy array, mcd_batch_counts)."""
    pm = np.ascontiguousarray(pair_map, dtype=np.int32)
    rk = np.ascontiguousarray(row_kind, dtype=np.uint8)
    R = pm.shape[0]
    plan = np.zeros(mcd_plan_words(R), dtype=np.int32)
    counts = mcd_batch_counts()
    _check(_mcd_batch_plan(h, R, pm.ctypes.data, rk.ctypes.data, plan.ctypes.data, plan.shape[0],
                           ctypes.byref(counts)), "mcd_batch_plan")
    return plan, counts


def mcd_plan_sampled_row(plan, s):
    row, comp = _i32(), _i32()
    _check(_mcd_plan_sampled_row(plan.ctypes.data, s, ctypes.byref(row), ctypes.byref(comp)),
           "mcd_plan_sampled_row")
    return row.value, comp.value


def mcd_workspace_bytes(h, R):
    return int(_mcd_workspace_bytes(h, R))


def _step_args(R, counts, plan, hidden, cfg_w, temperature, top_k, top_p, rng_key, step,
               n_frames, grid_slot, seed, tokens_out, frame_grid, n_slots, F_max, scores,
               workspace, modality_out=None):
    return mcd_step_args(R, counts, _ptr(plan), _ptr(hidden), _ptr(cfg_w), _ptr(temperature),
                         _ptr(top_k), _ptr(top_p), _ptr(rng_key), _ptr(step), _ptr(n_frames),
                         _ptr(grid_slot), seed, _ptr(tokens_out), _ptr(frame_grid),
                         _ptr(modality_out), n_slots, F_max, _ptr(scores), _ptr(workspace),
                         0 if workspace is None else workspace.numel() * workspace.element_size())


def mcd_head_step(h, stream=None, **kw):
    a = _step_args(**kw)
    _check(_mcd_head_step(h, ctypes.byref(a), _stream(stream)), "mcd_head_step")


def mcd_head_step_noalloc(h, stream=None, **kw):
    """mcd_head_step with the text-head partials in the library's per-GPU
    array; `workspace` only needs the 256-byte status word region."""
    a = _step_args(**kw)
    _check(_mcd_head_step_noalloc(h, ctypes.byref(a), _stream(stream)), "mcd_head_step_noalloc")


MCD_NOALLOC_SCRATCH_BYTES = 8 << 20


def mcd_head_logits(h, stream=None, **kw):
    a = _step_args(**kw)
    _check(_mcd_head_logits(h, ctypes.byref(a), _stream(stream)), "mcd_head_logits")


def mcd_sample_step(h, stream=None, **kw):
    a = _step_args(**kw)
    _check(_mcd_sample_step(h, ctypes.byref(a), _stream(stream)), "mcd_sample_step")


def mcd_deinterleave(streams, delays, grid, stream=None):
    """streams: int32 [n_req][T][K] -> grid int32 [n_req][K][T - max d] (device tensors)."""
    n_req, T, K = streams.shape
    d = np.ascontiguousarray(delays, dtype=np.int32)
    _check(_mcd_deinterleave(_ptr(streams), n_req, T, K, d.ctypes.data, _ptr(grid),
                             _stream(stream)), "mcd_deinterleave")


def mcd_interleave(grid, delays, pad_id, streams, stream=None):
    """grid: int32 [n_req][K][F] -> streams int32 [n_req][F + max d][K] (device tensors)."""
    n_req, K, F = grid.shape
    d = np.ascontiguousarray(delays, dtype=np.int32)
    _check(_mcd_interleave(_ptr(grid), n_req, F, K, d.ctypes.data, pad_id, _ptr(streams),
                           _stream(stream)), "mcd_interleave")


def mcd_next_input(E, tokens, row_kind, pad_id, out, E_text=None, workspace=None, stream=None):
    """Next-step input of every row: E [K][V + 1][H] (bf16 or fp32, device),
    tokens int32 [R][K], row_kind uint8 [R], out [R][H] of E's type (device)."""
    K, V1, H = E.shape
    R = tokens.shape[0]
    dtype = {torch.bfloat16: MCD_BF16, torch.float32: MCD_F32}[E.dtype]
    a = mcd_next_input_args(R, H, K, V1 - 1, int(pad_id), dtype, _ptr(E),
                            0 if E_text is None else E_text.shape[0], _ptr(E_text),
                            _ptr(row_kind), _ptr(tokens), _ptr(out), _ptr(workspace))
    _check(_mcd_next_input(ctypes.byref(a), _stream(stream)), "mcd_next_input")


MCD_PHASE_TEXT, MCD_PHASE_BRIDGE, MCD_PHASE_AUDIO, MCD_PHASE_DRAIN = 0, 1, 2, 3


def mcd_phase_advance(bridge, audio_end, drain_steps, phase, count, token0, modality):
    """One step of the requests' phases (host arrays, updated in place):
    phase uint8 [n], count int32 [n], token0 int32 [n], modality uint8 [n].
    Returns emit int32 [n]."""
    br = np.ascontiguousarray(bridge, dtype=np.int32)
    d = mcd_phase_desc(br.shape[0], br.ctypes.data if br.shape[0] else None, int(audio_end),
                       int(drain_steps))
    for a, dt in ((phase, np.uint8), (count, np.int32)):
        assert a.dtype == dt and a.flags.c_contiguous
    token0 = np.ascontiguousarray(token0, dtype=np.int32)
    modality = np.ascontiguousarray(modality, dtype=np.uint8)
    emit = np.empty(phase.shape[0], dtype=np.int32)
    _check(_mcd_phase_advance(ctypes.byref(d), phase.shape[0], phase.ctypes.data,
                              count.ctypes.data, token0.ctypes.data, modality.ctypes.data,
                              emit.ctypes.data), "mcd_phase_advance")
    return emit


class Scheduler:
    """Paired co-scheduling of CFG requests (host only): the C scheduler of
    libmcd behind plan() / commit()."""

    _I32 = ("row_req", "row_slot", "row_tokens", "row_context", "head_row", "pair_map", "step",
            "n_frames", "grid_slot")

    def __init__(self, max_rows, token_budget, null_prompt_len, drain_steps, max_requests=4096):
        d = mcd_sched_desc(int(max_rows), int(token_budget), int(null_prompt_len),
                           int(drain_steps), int(max_requests))
        h = _vp()
        _check(_mcd_sched_create(ctypes.byref(d), ctypes.byref(h)), "mcd_sched_create")
        self.handle = h.value
        self.max_requests = int(max_requests)
        self._destroy = _mcd_sched_destroy

    def __del__(self):
        h = getattr(self, "handle", None)
        destroy = getattr(self, "_destroy", None)
        if h is not None and destroy is not None:
            destroy(h)
            self.handle = None

    def submit(self, cfg_w, prompt_len, text_len, n_frames):
        q = mcd_sched_request(float(cfg_w), int(prompt_len), int(text_len), int(n_frames))
        rid = _i32()
        _check(_mcd_sched_submit(self.handle, ctypes.byref(q), ctypes.byref(rid)),
               "mcd_sched_submit")
        return rid.value

    def plan(self):
        """The next step as a dict of numpy copies (backbone rows and head rows)."""
        b = mcd_sched_batch()
        _check(_mcd_sched_plan(self.handle, ctypes.byref(b)), "mcd_sched_plan")

        def arr(name, n, ct, dt):
            p = getattr(b, name)
            if n == 0 or not p:
                return np.zeros(0, dtype=dt)
            return np.ctypeslib.as_array(ctypes.cast(p, ctypes.POINTER(ct)), (n,)).astype(dt)

        out = {"n_rows": b.n_rows, "R": b.R}
        for name in self._I32:
            n = b.R if name in ("head_row", "pair_map", "step", "n_frames", "grid_slot") else b.n_rows
            out[name] = arr(name, n, ctypes.c_int32, np.int32)
        out["row_member"] = arr("row_member", b.n_rows, ctypes.c_uint8, np.uint8)
        out["row_kind"] = arr("row_kind", b.R, ctypes.c_uint8, np.uint8)
        out["cfg_w"] = arr("cfg_w", b.R, ctypes.c_float, np.float32)
        return out

    def commit(self):
        """Apply the planned step; returns the ids of the requests it finished."""
        fin = np.empty(self.max_requests, dtype=np.int32)
        n = _i32()
        _check(_mcd_sched_commit(self.handle, fin.ctypes.data, fin.shape[0], ctypes.byref(n)),
               "mcd_sched_commit")
        return fin[:n.value].copy()

    def counts(self):
        w, r = _i32(), _i32()
        _check(_mcd_sched_counts(self.handle, ctypes.byref(w), ctypes.byref(r)),
               "mcd_sched_counts")
        return w.value, r.value


def mcd_read_device_status(workspace, stream=None):
    code = ctypes.c_uint32()
    _check(_mcd_read_device_status(_ptr(workspace), ctypes.byref(code), _stream(stream)),
           "mcd_read_device_status")
    return code.value


# ---------------------------------------------------------------------------
# 4-bit key/value cache

def mcd_cache_page_bytes(D):
    return int(_mcd_cache_page_bytes(D))


def mcd_cache_workspace_bytes(cache, rows, Hq):
    n = int(_mcd_cache_workspace_bytes(cache.ref, rows.ref, Hq))
    if n == 0:
        raise McdError(MCD_E_INVALID, "mcd_cache_workspace_bytes")
    return n


_DTYPES = {torch.bfloat16: MCD_BF16, torch.float32: MCD_F32}


def _tokens(name, t, rows, heads, D, like=None):
    """dtype and row stride of a packed token tensor [n_tokens][heads][D], each head's channels
    and a token's heads without gaps."""
    shape, stride = t.shape, t.stride()
    if shape[0] < rows.n_tokens or shape[1:] != (heads, D):
        raise ValueError(f"{name}: shape {tuple(shape)}, expected [{rows.n_tokens}][{heads}][{D}]")
    if stride[2] != 1 or (stride[1] != D and heads > 1):
        raise ValueError(f"{name}: a token's heads must be contiguous (strides {stride})")
    if t.dtype not in _DTYPES or (like is not None and t.dtype != like.dtype):
        raise ValueError(f"{name}: dtype {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} is not on the GPU")
    return _DTYPES[t.dtype], stride[0] if shape[0] > 1 else heads * D


class Cache:
    """A layer's 4-bit key/value cache and the device tensors it borrows.

    pages: uint8 [n_pages][Hkv][mcd_cache_page_bytes(D)]; table: int32 [n_slots][max_pages];
    weight: float32 [n_slots][Hkv][max_pages * 64] or None.  Cache.alloc makes the pages."""

    def __init__(self, pages, table, D, weight=None):
        self.pages, self.table, self.weight, self.D = pages, table, weight, int(D)
        n_pages, self.Hkv, page_bytes = pages.shape
        self.n_slots, self.max_pages = table.shape
        if page_bytes != mcd_cache_page_bytes(D):
            raise ValueError(f"pages of {page_bytes} bytes, heads of {D} take "
                             f"{mcd_cache_page_bytes(D)}")
        shape = (self.n_slots, self.Hkv, self.max_pages * MCD_CACHE_PAGE)
        for name, t, dt in (("pages", pages, torch.uint8), ("table", table, torch.int32),
                            ("weight", weight, torch.float32)):
            if t is not None and (t.dtype != dt or not t.is_contiguous()):
                raise ValueError(f"{name} must be contiguous {dt}")
        if weight is not None and tuple(weight.shape) != shape:
            raise ValueError(f"weight: shape {tuple(weight.shape)}, expected {shape}")
        self.struct = mcd_cache(self.Hkv, self.D, self.n_slots, self.max_pages, n_pages,
                                _ptr(pages), _ptr(table), _ptr(weight))
        self.ref = ctypes.byref(self.struct)
        self.on_gpu = all(t is None or t.is_cuda for t in (pages, table, weight))

    @classmethod
    def alloc(cls, n_pages, Hkv, D, n_slots, max_pages, weights=False, device="cuda"):
        """Zeroed pages and weights and a table of -1 (no page)."""
        pages = torch.zeros((n_pages, Hkv, mcd_cache_page_bytes(D)), dtype=torch.uint8,
                            device=device)
        table = torch.full((n_slots, max_pages), -1, dtype=torch.int32, device=device)
        weight = torch.zeros((n_slots, Hkv, max_pages * MCD_CACHE_PAGE), device=device) \
            if weights else None
        return cls(pages, table, D, weight)

    def workspace(self, rows, Hq):
        """A zeroed workspace for these rows' bounds and every smaller step."""
        return torch.zeros(mcd_cache_workspace_bytes(self, rows, Hq), dtype=torch.uint8,
                           device=self.pages.device)


class CacheRows:
    """The rows of a step (int32 device tensors, borrowed): context [R], slot [R] or None, start
    [R + 1] or None for one token in every row.  max_tokens and max_context bound every row's
    tokens and its positions after them."""

    def __init__(self, context, start=None, slot=None, n_tokens=None, max_tokens=1,
                 max_context=0):
        self.context, self.start, self.slot = context, start, slot
        self.R = context.shape[0]
        self.n_tokens = self.R if n_tokens is None else int(n_tokens)
        if start is not None and n_tokens is None:
            raise ValueError("start needs n_tokens")
        for name, t, n in (("context", context, self.R), ("start", start, self.R + 1),
                           ("slot", slot, self.R)):
            if t is not None and (t.dtype != torch.int32 or tuple(t.shape) != (n,)
                                  or not t.is_contiguous()):
                raise ValueError(f"{name} must be contiguous int32 [{n}]")
        self.struct = mcd_cache_rows(self.R, self.n_tokens, int(max_tokens), int(max_context),
                                     _ptr(slot), _ptr(context), _ptr(start))
        self.ref = ctypes.byref(self.struct)
        self.on_gpu = all(t is None or t.is_cuda for t in (context, start, slot))


def _on_gpu(*parts):
    if not all(p.on_gpu if hasattr(p, "on_gpu") else p is None or p.is_cuda for p in parts):
        raise ValueError("a tensor of the call is not on the GPU")


def mcd_cache_append(cache, rows, k, v, workspace, stream=None):
    """k, v [n_tokens][Hkv][D] (bf16 or fp32) into the rows' pages."""
    dt, ks = _tokens("k", k, rows, cache.Hkv, cache.D)
    _, vs = _tokens("v", v, rows, cache.Hkv, cache.D, k)
    _on_gpu(cache, rows, workspace)
    _check(_mcd_cache_append(cache.ref, rows.ref, dt, k.data_ptr(), ks, v.data_ptr(), vs,
                             workspace.data_ptr(), workspace.nbytes, _stream(stream)),
           "mcd_cache_append")


def mcd_cache_read(cache, rows, k, v, workspace, stream=None):
    """The values at the rows' positions into k, v [n_tokens][Hkv][D] (bf16 or fp32)."""
    dt, ks = _tokens("k", k, rows, cache.Hkv, cache.D)
    _, vs = _tokens("v", v, rows, cache.Hkv, cache.D, k)
    _on_gpu(cache, rows, workspace)
    _check(_mcd_cache_read(cache.ref, rows.ref, dt, k.data_ptr(), ks, v.data_ptr(), vs,
                           workspace.data_ptr(), workspace.nbytes, _stream(stream)),
           "mcd_cache_read")


def mcd_cache_attend(cache, rows, q, out, workspace, scale=None, lse=None, weight_out=None,
                     stream=None):
    """out = softmax(scale q k^T) v for q, out [n_tokens][Hq][D] (bf16 or fp32); scale: default
    1 / sqrt(D).  weight_out: laid out as cache.weight (which it may be)."""
    Hq = q.shape[1]
    dt, qs = _tokens("q", q, rows, Hq, cache.D)
    _, os_ = _tokens("out", out, rows, Hq, cache.D, q)
    if lse is not None and (lse.dtype != torch.float32 or not lse.is_contiguous()
                            or lse.numel() < rows.n_tokens * Hq):
        raise ValueError("lse must be contiguous float32 [n_tokens][Hq]")
    if weight_out is not None and (
            weight_out.dtype != torch.float32 or not weight_out.is_contiguous()
            or weight_out.numel() != cache.n_slots * cache.Hkv * cache.max_pages * MCD_CACHE_PAGE):
        raise ValueError("weight_out must be laid out as the cache's weight")
    _on_gpu(cache, rows, lse, weight_out, workspace)
    a = mcd_cache_attend_args(Hq, dt, cache.D ** -0.5 if scale is None else scale, q.data_ptr(),
                              qs, out.data_ptr(), os_, _ptr(lse), _ptr(weight_out),
                              workspace.data_ptr(), workspace.nbytes)
    _check(_mcd_cache_attend(cache.ref, rows.ref, ctypes.byref(a), _stream(stream)),
           "mcd_cache_attend")


def mcd_cache_evict(src, dst, length, keep, recent, kept, length_out, workspace, max_length,
                    slot=None, stream=None):
    """Row r: the positions kept of slot[r] (or r) of src, length[r] long, into slot r of dst.
    kept: int32 [R][Hkv][keep]; length, length_out, slot: int32 [R]."""
    R = length.shape[0]
    for name, t, n in (("length", length, R), ("length_out", length_out, R), ("slot", slot, R),
                       ("kept", kept, R * src.Hkv * keep)):
        if t is not None and (t.dtype != torch.int32 or t.numel() != n or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous int32 with {n} elements")
    _on_gpu(src, dst, length, slot, kept, length_out, workspace)
    a = mcd_cache_evict_args(R, int(max_length), int(keep), int(recent), _ptr(slot), _ptr(length),
                             _ptr(kept), _ptr(length_out), workspace.data_ptr(), workspace.nbytes)
    _check(_mcd_cache_evict(src.ref, dst.ref, ctypes.byref(a), _stream(stream)),
           "mcd_cache_evict")


# ---------------------------------------------------------------------------
# Convenience wrapper

class Head:
    """Handle plus the device tensors it borrows."""

    def __init__(self, W, delays, pad_id, bias=None, W_text=None, V_stream=None, T_text=0):
        """W: [K][V][H], or [N][H] with V_stream (the ids of each stream)."""
        assert W.is_cuda and W.is_contiguous()
        if V_stream is None:
            assert W.dim() == 3
            K, V, H = W.shape
        else:
            V_stream = np.ascontiguousarray(V_stream, dtype=np.int32)
            assert W.dim() == 2 and W.shape[0] == int(V_stream.sum())
            K, V, H = V_stream.shape[0], int(V_stream.max()), W.shape[1]
        dtype = {torch.bfloat16: MCD_BF16, torch.float32: MCD_F32}[W.dtype]
        self.W, self.bias, self.W_text, self.V_stream = W, bias, W_text, V_stream
        self.H, self.K, self.V, self.pad_id = H, K, V, int(pad_id)
        self.delays = np.ascontiguousarray(delays, dtype=np.int32)
        self.V_text = 0 if W_text is None else W_text.shape[0]
        self.handle = mcd_head_create(H, K, V, self.pad_id, self.delays, dtype, W, bias,
                                      self.V_text, W_text, V_stream, T_text)
        # the library's own entry, held here: at interpreter exit the module's
        # globals may already be gone when this object is collected
        self._destroy = _mcd_head_destroy

    def __del__(self):
        h = getattr(self, "handle", None)
        destroy = getattr(self, "_destroy", None)
        if h is not None and destroy is not None:
            destroy(h)
            self.handle = None

    def plan(self, pair_map, row_kind, device="cuda"):
        plan, counts = mcd_batch_plan(self.handle, pair_map, row_kind)
        return Plan(plan, counts, torch.from_numpy(plan).to(device))

    def workspace(self, R, device="cuda"):
        return torch.zeros(max(mcd_workspace_bytes(self.handle, R), 256), dtype=torch.uint8,
                           device=device)


class Plan:
    def __init__(self, host, counts, dev):
        self.host, self.counts, self.dev = host, counts, dev
        self.R = int(host[1])
        self.n_pairs, self.n_solo, self.n_text = counts.n_pairs, counts.n_solo, counts.n_text
        self.Rs = self.n_pairs + self.n_solo

    def sampled_rows(self):
        """(row, companion) of each sampled index."""
        return [mcd_plan_sampled_row(self.host, s) for s in range(self.Rs)]
