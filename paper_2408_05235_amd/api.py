"""Python entry points with the names of the C ABI; argument marshalling only.

Every computation runs in the HIP kernels of libtl.so.  Tensors must live on
the current CUDA(HIP) device; work is enqueued on torch's current stream.
Unsigned 64-bit quantities (deadlines, SLOs) travel as ``torch.int64``
tensors holding the same bits; 32-bit flag words as ``torch.int32``.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from . import _lib
from ._lib import check, lib


def _p(t):
    return None if t is None else t.data_ptr()


# The raw handle of torch.cuda.current_stream() without a Stream object, by
# functions that torch keeps for its own use: None where it has them no more.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    if _raw_stream is None or _raw_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


def _stream_on(device):
    """The stream for work on tensors of ``device`` (an index), which has to be
    the current one."""
    now = torch.cuda.current_device() if _raw_device is None else _raw_device()
    if now != device:
        raise ValueError(f"the tensors are on cuda:{device}, the current device is cuda:{now}")
    return _stream() if _raw_stream is None else _raw_stream(now)


def _need(t, dtype, name, shape=None, device=None):
    if (t is not None and (t.is_cuda if device is None else t.get_device() == device) and t.dtype == dtype
            and t.is_contiguous() and (shape is None or t.shape == shape)):
        return t
    if t is None:
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if device is not None and t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, other tensors are on cuda:{device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t


def _opt(t, dtype, name, shape=None):
    return None if t is None else _need(t, dtype, name, shape)


def _project_args(req_offset, prompt_len, generated, remaining, arrival_iter, kv_capacity,
                  horizon, block_tokens, deadline_ns, lost, batch_cap, out):
    """Checked tl_project_args for the scoreboards, with the curve outputs
    (taken from ``out`` or allocated).  Returns (args, outputs)."""
    _need(req_offset, torch.int64, "req_offset")
    S = req_offset.numel() - 1
    R = prompt_len.numel()
    for name, t in (("prompt_len", prompt_len), ("generated", generated),
                    ("remaining", remaining), ("arrival_iter", arrival_iter)):
        _need(t, torch.int32, name, (R,))
    _need(kv_capacity, torch.int32, "kv_capacity", (S,))
    _opt(deadline_ns, torch.int64, "deadline_ns", (R,))
    _opt(lost, torch.uint8, "lost", (R,))
    _opt(batch_cap, torch.int32, "batch_cap", (S,))
    H = int(horizon)
    dev = req_offset.device
    o = out or {}

    def buf(name, shape, dtype):
        t = o.get(name) if o.get(name) is not None else torch.empty(shape, dtype=dtype, device=dev)
        return _need(t, dtype, name, shape)

    res = dict(batch=buf("batch", (S, H), torch.int32), kv=buf("kv", (S, H), torch.int32),
               deadline_at=buf("deadline_at", (S, H), torch.int64), n_iters=buf("n_iters", (S,), torch.int32),
               flags=buf("flags", (S,), torch.int32))
    a = _lib.ProjectArgs()
    a.struct_size = ctypes.sizeof(_lib.ProjectArgs)
    a.horizon = H
    a.n_scenarios = S
    a.n_requests = R
    a.block_tokens = int(block_tokens)
    a.req_offset = _p(req_offset)
    a.prompt_len = _p(prompt_len)
    a.generated = _p(generated)
    a.remaining = _p(remaining)
    a.arrival_iter = _p(arrival_iter)
    a.deadline_ns = _p(deadline_ns)
    a.lost = _p(lost)
    a.kv_capacity = _p(kv_capacity)
    a.batch_cap = _p(batch_cap)
    a.batch, a.kv, a.deadline_at = _p(res["batch"]), _p(res["kv"]), _p(res["deadline_at"])
    a.n_iters, a.flags = _p(res["n_iters"]), _p(res["flags"])
    return a, res


def tl_project(req_offset, prompt_len, generated, remaining, arrival_iter, kv_capacity,
               horizon, block_tokens, deadline_ns=None, lost=None, batch_cap=None,
               freqs_mhz=None, engine_size=None, n_features=3, want_rows=True, out=None):
    """Stage 1 (tl_project).  Returns a dict of device tensors:
    batch, kv [S,H] int32; deadline_at [S,H] int64 (uint64 bits); n_iters [S]
    int32; flags [S] int32 (uint32 bits); rows [S,F,H,n_features] fp32 when
    ``want_rows`` and ``freqs_mhz`` is given."""
    a, res = _project_args(req_offset, prompt_len, generated, remaining, arrival_iter, kv_capacity,
                           horizon, block_tokens, deadline_ns, lost, batch_cap, out)
    S, H = int(a.n_scenarios), int(a.horizon)
    rows_on = bool(want_rows and freqs_mhz is not None)
    if rows_on:
        F = int(freqs_mhz.numel())
        _need(freqs_mhz, torch.float32, "freqs_mhz", (F,))
        if n_features == 4:
            _need(engine_size, torch.float32, "engine_size", (S,))
        o = out or {}
        rows = o.get("rows")
        if rows is None:
            rows = torch.empty((S, F, H, n_features), dtype=torch.float32, device=req_offset.device)
        _need(rows, torch.float32, "rows", (S, F, H, n_features))
        a.n_freqs, a.n_features = F, int(n_features)
        a.freqs_mhz, a.engine_size, a.rows = _p(freqs_mhz), _p(engine_size), _p(rows)
        res["rows"] = rows
    check(lib().tl_project(ctypes.byref(a), _stream()))
    return res


def tl_admit(forest, max_freq_mhz, tbt_slo_ns, cand_prompt, cand_len, req_offset, prompt_len, generated,
             remaining, arrival_iter, kv_capacity, horizon, block_tokens, deadline_ns=None, lost=None,
             batch_cap=None, engine_size=None, cand_deadline_ns=None, out=None, lattice=None):
    """Admission control (tl_admit) for one new query per scenario.  Returns
    the projection with the query (batch, kv, deadline_at, n_iters, flags as
    in tl_project), ips [S,H] fp32 at max_freq_mhz and decision [S] int32
    (TL_ADMIT_* codes)."""
    a, res = _project_args(req_offset, prompt_len, generated, remaining, arrival_iter, kv_capacity,
                           horizon, block_tokens, deadline_ns, lost, batch_cap, out)
    S, H = int(a.n_scenarios), int(a.horizon)
    dev = req_offset.device
    _need(tbt_slo_ns, torch.int64, "tbt_slo_ns", (S,))
    _need(cand_prompt, torch.int32, "cand_prompt", (S,))
    _need(cand_len, torch.int32, "cand_len", (S,))
    _opt(cand_deadline_ns, torch.int64, "cand_deadline_ns", (S,))
    if forest.n_features == 4:
        _need(engine_size, torch.float32, "engine_size", (S,))
    o = out or {}
    ips = o.get("ips") if o.get("ips") is not None else torch.empty((S, H), dtype=torch.float32, device=dev)
    dec = o.get("decision") if o.get("decision") is not None else torch.empty(S, dtype=torch.int32, device=dev)
    _need(ips, torch.float32, "ips", (S, H))
    _need(dec, torch.int32, "decision", (S,))
    b = _lib.AdmitArgs()
    b.struct_size = ctypes.sizeof(_lib.AdmitArgs)
    b.proj = a
    b.forest = forest._h
    b.max_freq_mhz = float(max_freq_mhz)
    b.engine_size = _p(engine_size) if forest.n_features == 4 else None
    b.tbt_slo_ns = _p(tbt_slo_ns)
    b.cand_prompt, b.cand_len, b.cand_deadline_ns = _p(cand_prompt), _p(cand_len), _p(cand_deadline_ns)
    b.ips, b.decision = _p(ips), _p(dec)
    b.lattice = None if lattice is None else lattice._h
    check(lib().tl_admit(ctypes.byref(b), _stream()))
    res.update(ips=ips, decision=dec)
    return res


class Forest:
    """Device copy of a tree ensemble (tl_forest_create / tl_forest_destroy)."""

    def __init__(self, n_trees, depth, n_features, base_score, feature, threshold, leaf):
        feature = np.ascontiguousarray(feature, dtype=np.uint8)
        threshold = np.ascontiguousarray(threshold, dtype=np.float32)
        leaf = np.ascontiguousarray(leaf, dtype=np.float32)
        n_int = (1 << int(depth)) - 1
        if feature.size != n_trees * n_int or threshold.size != n_trees * n_int or leaf.size != n_trees * (n_int + 1):
            raise ValueError("tree array sizes do not match n_trees and depth")
        self.n_trees, self.depth, self.n_features = int(n_trees), int(depth), int(n_features)
        self.base_score = float(np.float32(base_score))
        h = ctypes.c_void_p()
        check(lib().tl_forest_create(self.n_trees, self.depth, self.n_features, self.base_score,
                                     feature.ctypes.data_as(ctypes.c_void_p),
                                     threshold.ctypes.data_as(ctypes.c_void_p),
                                     leaf.ctypes.data_as(ctypes.c_void_p), ctypes.byref(h)))
        self._h = h

    @classmethod
    def from_dict(cls, d):
        return cls(d["n_trees"], d["depth"], d["n_features"], d["base_score"],
                   d["feature"], d["threshold"], d["leaf"])

    def tl_forest_predict(self, rows, out=None):
        """IPS for every row of ``rows`` ([..., n_features] fp32 device tensor)."""
        _need(rows, torch.float32, "rows")
        if rows.shape[-1] != self.n_features:
            raise ValueError(f"rows have {rows.shape[-1]} features, forest has {self.n_features}")
        n = rows.numel() // self.n_features
        if out is None:
            out = torch.empty(rows.shape[:-1], dtype=torch.float32, device=rows.device)
        _need(out, torch.float32, "out")
        if out.numel() != n:
            raise ValueError("out has the wrong number of elements")
        check(lib().tl_forest_predict(self._h, _p(rows), n, _p(out), _stream()))
        return out

    predict = tl_forest_predict

    def tl_forest_predict_grid(self, freqs_mhz, kv, batch, engine_size=None, out=None, noalloc=False):
        """IPS on the projection grid: out[s, f, j] = M(freqs[f], kv[s, j],
        batch[s, j] [, engine[s]]) without materializing the rows.  With
        ``noalloc`` (and ``out`` given) the call goes to
        tl_forest_predict_grid_noalloc, which allocates nothing."""
        _need(kv, torch.int32, "kv")
        if kv.dim() != 2:
            raise ValueError("kv must be [S, H]")
        S, H = kv.shape
        F = freqs_mhz.numel()
        _need(freqs_mhz, torch.float32, "freqs_mhz", (F,))
        _need(batch, torch.int32, "batch", (S, H))
        if self.n_features == 4:
            _need(engine_size, torch.float32, "engine_size", (S,))
        else:
            engine_size = None
        if out is None:
            out = torch.empty((S, F, H), dtype=torch.float32, device=kv.device)
        _need(out, torch.float32, "out", (S, F, H))
        fn = lib().tl_forest_predict_grid_noalloc if noalloc else lib().tl_forest_predict_grid
        check(fn(self._h, S, F, H, _p(freqs_mhz), _p(kv), _p(batch), _p(engine_size), _p(out), _stream()))
        return out

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            lib().tl_forest_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Lattice:
    """The model compiled to its input lattice (tl_lattice_create): every
    (engine size, batch 0..batch_max, frequency, KV 0..kv_max) evaluated once;
    prediction on the projection grid is then a table lookup with the same
    values (tl_lattice_predict_grid).  Keeps the forest alive."""

    def __init__(self, forest, freqs_mhz, kv_max, batch_max, engine_values=None):
        _need(freqs_mhz, torch.float32, "freqs_mhz")
        self.forest = forest
        self.n_freqs = int(freqs_mhz.numel())
        ev = np.ascontiguousarray(engine_values if engine_values is not None else [], dtype=np.float32)
        h = ctypes.c_void_p()
        check(lib().tl_lattice_create(forest._h, self.n_freqs, _p(freqs_mhz), int(ev.size),
                                      ev.ctypes.data_as(ctypes.c_void_p) if ev.size else None, int(kv_max),
                                      int(batch_max), _stream(), ctypes.byref(h)))
        self._h = h
        self.nbytes = int(lib().tl_lattice_bytes(h))

    def tl_lattice_predict_grid(self, kv, batch, engine_size=None, out=None):
        """IPS [S, F, H] for the projection curves kv, batch [S, H] int32."""
        _need(kv, torch.int32, "kv")
        if kv.dim() != 2:
            raise ValueError("kv must be [S, H]")
        S, H = kv.shape
        _need(batch, torch.int32, "batch", (S, H))
        if self.forest.n_features == 4:
            _need(engine_size, torch.float32, "engine_size", (S,))
        if out is None:
            out = torch.empty((S, self.n_freqs, H), dtype=torch.float32, device=kv.device)
        _need(out, torch.float32, "out", (S, self.n_freqs, H))
        check(lib().tl_lattice_predict_grid(self._h, S, H, _p(kv), _p(batch),
                                            _p(engine_size) if self.forest.n_features == 4 else None, _p(out),
                                            _stream()))
        return out

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            lib().tl_lattice_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def tl_select_freq(ips, deadline_at, n_iters, tbt_slo_ns, proj_flags=None, out=None):
    """Stage 3 (tl_select_freq).  ips [S,F,H] fp32.  Returns (freq_idx int32
    [S], status int32 [S])."""
    _need(ips, torch.float32, "ips")
    if ips.dim() != 3:
        raise ValueError("ips must be [S, F, H]")
    S, F, H = ips.shape
    _need(deadline_at, torch.int64, "deadline_at", (S, H))
    _need(n_iters, torch.int32, "n_iters", (S,))
    _need(tbt_slo_ns, torch.int64, "tbt_slo_ns", (S,))
    _opt(proj_flags, torch.int32, "proj_flags", (S,))
    o = out or {}
    idx = o.get("freq_idx") if o.get("freq_idx") is not None else torch.empty(S, dtype=torch.int32, device=ips.device)
    st = o.get("status") if o.get("status") is not None else torch.empty(S, dtype=torch.int32, device=ips.device)
    _need(idx, torch.int32, "freq_idx", (S,))
    _need(st, torch.int32, "status", (S,))
    check(lib().tl_select_freq(_p(ips), S, F, H, _p(deadline_at), _p(n_iters), _p(tbt_slo_ns),
                               _p(proj_flags), _p(idx), _p(st), _stream()))
    return idx, st


def tl_select_freq_binary(forest, freqs_mhz, kv, batch, deadline_at, n_iters, tbt_slo_ns, proj_flags=None,
                          engine_size=None, out=None, lattice=None):
    """The controller's binary search over frequencies (tl_select_freq_binary),
    querying the model only at probed frequencies (read from ``lattice``, a
    Lattice of the same forest built for freqs_mhz, when given).  kv, batch
    [S,H] int32 as written by tl_project.  Returns (freq_idx int32 [S],
    status int32 [S])."""
    _need(kv, torch.int32, "kv")
    if kv.dim() != 2:
        raise ValueError("kv must be [S, H]")
    S, H = kv.shape
    F = int(freqs_mhz.numel())
    _need(freqs_mhz, torch.float32, "freqs_mhz", (F,))
    _need(batch, torch.int32, "batch", (S, H))
    _need(deadline_at, torch.int64, "deadline_at", (S, H))
    _need(n_iters, torch.int32, "n_iters", (S,))
    _need(tbt_slo_ns, torch.int64, "tbt_slo_ns", (S,))
    _opt(proj_flags, torch.int32, "proj_flags", (S,))
    if forest.n_features == 4:
        _need(engine_size, torch.float32, "engine_size", (S,))
    o = out or {}
    dev = kv.device

    def buf(name, shape, dtype):
        t = o.get(name) if o.get(name) is not None else torch.empty(shape, dtype=dtype, device=dev)
        return _need(t, dtype, name, shape)

    ips = buf("ips_work", (S, H), torch.float32)
    work = buf("search_work", (3, S), torch.int32)
    idx = buf("freq_idx", (S,), torch.int32)
    st = buf("status", (S,), torch.int32)
    check(lib().tl_select_freq_binary(forest._h, S, F, H, _p(freqs_mhz), _p(kv), _p(batch),
                                      _p(engine_size) if forest.n_features == 4 else None, _p(deadline_at),
                                      _p(n_iters), _p(tbt_slo_ns), _p(proj_flags), _p(ips), _p(work), _p(idx),
                                      _p(st), None if lattice is None else lattice._h, _stream()))
    return idx, st


def tl_adjust_lengths(req_offset, generated, pred_len, scale_num, scale_den, max_tokens, out=None):
    """Scoreboard remaining-token counts from predicted total lengths under
    generation-length errors (tl_adjust_lengths).  Per-scenario scale_num,
    scale_den (int32 tensors holding uint32 bits) and max_tokens.  Returns
    remaining [R] int32."""
    _need(req_offset, torch.int64, "req_offset")
    S = req_offset.numel() - 1
    R = generated.numel()
    _need(generated, torch.int32, "generated", (R,))
    _need(pred_len, torch.int32, "pred_len", (R,))
    for name, t in (("scale_num", scale_num), ("scale_den", scale_den), ("max_tokens", max_tokens)):
        _need(t, torch.int32, name, (S,))
    rem = out if out is not None else torch.empty(R, dtype=torch.int32, device=req_offset.device)
    _need(rem, torch.int32, "out", (R,))
    check(lib().tl_adjust_lengths(S, R, _p(req_offset), _p(generated), _p(pred_len), _p(scale_num),
                                  _p(scale_den), _p(max_tokens), _p(rem), _stream()))
    return rem


_KV_DTYPES = {torch.bfloat16: _lib.BF16, torch.float16: _lib.F16}
_VIEW_SIZE, _APPEND_SIZE = ctypes.sizeof(_lib.KvView), ctypes.sizeof(_lib.KvAppendArgs)
_ATTEND_SIZE, _PAGES_SIZE = ctypes.sizeof(_lib.AttendArgs), ctypes.sizeof(_lib.Pages)
_BOUNDS_SIZE, _SELECT_SIZE = ctypes.sizeof(_lib.PageBoundsArgs), ctypes.sizeof(_lib.SelectPagesArgs)
_ATTEND_PAGES_SIZE, _NORM_SIZE = ctypes.sizeof(_lib.AttendPagesArgs), ctypes.sizeof(_lib.NormArgs)
_SAMPLE_SIZE = ctypes.sizeof(_lib.SampleArgs)
_DTYPES = {torch.bfloat16: _lib.BF16, torch.float16: _lib.F16, torch.float32: _lib.F32}


def _strides(t):
    """Strides, 0 where there is nothing to step over."""
    return tuple([0 if n <= 1 else s for n, s in zip(t.shape, t.stride())])


def _rows3(t, dtype, name, device, heads=None, dim=None, tokens=None):
    """The strides of packed rows [tokens, heads, dim], whatever they are for
    tokens and heads (a view into a layer's fused product, say)."""
    shape, strides = t.shape, t.stride()
    if (t.get_device() == device and t.dtype == dtype and len(shape) == 3 and strides[2] == 1
            and (heads is None or shape[1] == heads) and shape[2] == dim and (tokens is None or shape[0] == tokens)):
        return strides if shape[0] > 1 and shape[1] > 1 else _strides(t)
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, the pages are on cuda:{device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if len(shape) != 3 or (shape[2] > 1 and strides[2] != 1):
        raise ValueError(f"{name} must be [tokens, heads, head_dim] with contiguous heads")
    want = (tokens, heads, dim)
    if any(w is not None and w != g for w, g in zip(want, shape)):
        raise ValueError(f"{name} must have shape {want}, got {tuple(shape)}")
    return _strides(t)


def _kv_view(key_pages, value_pages, page_table, length, device):
    shape, strides, dtype = key_pages.shape, key_pages.stride(), key_pages.dtype
    kind = _KV_DTYPES.get(dtype)
    if kind is None:
        raise ValueError(f"key_pages must be bfloat16 or float16, got {dtype}")
    if device < 0 or not value_pages.is_cuda:
        raise ValueError("pages must be device tensors")
    if value_pages.get_device() != device:
        raise ValueError(f"key_pages are on cuda:{device}, value_pages on {value_pages.device}")
    if len(shape) != 4 or shape != value_pages.shape or dtype != value_pages.dtype:
        raise ValueError("key_pages and value_pages must be [n_pages, n_kv_heads, page_tokens, head_dim] alike")
    n_pages, heads, tokens, dim = shape
    if value_pages.stride() != strides or strides[3] != 1 or n_pages == 1 or heads == 1 or tokens == 1:
        strides = _strides(key_pages)
        if strides != _strides(value_pages) or strides[3] > 1:
            raise ValueError("key_pages and value_pages must have the same strides and contiguous heads")
    if page_table.dim() != 2:
        raise ValueError("page_table must be [n_seqs, table_width]")
    n_seqs, width = page_table.shape
    if page_table.get_device() != device or page_table.dtype != torch.int32 or not page_table.is_contiguous():
        _need(page_table, torch.int32, "page_table", None, device)
    if (length is None or length.get_device() != device or length.dtype != torch.int32 or not length.is_contiguous()
            or length.shape != (n_seqs,)):
        _need(length, torch.int32, "length", (n_seqs,), device)
    return _lib.KvView(_VIEW_SIZE, kind, heads, dim, tokens, width, n_pages, n_seqs, strides[0], strides[1],
                       strides[2], key_pages.data_ptr(), value_pages.data_ptr(), page_table.data_ptr(),
                       length.data_ptr())


def _int32(x, name):
    """``x`` as a 32-bit argument, which ctypes would cut to its low bits."""
    x = int(x)
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError(f"{name} {x} does not fit 32 bits")
    return x


def _no_gradients(who):
    """Where gradients would be asked for: the paged cache is for serving."""
    if torch.is_grad_enabled():
        raise ValueError(f"{who} has no gradients: call it under torch.no_grad(), or with detached tensors")


def _granted(t, n, device):
    return _need(t, torch.int32, "granted", (n + 1,), device).data_ptr()


def tl_kv_append(key, value, key_pages, value_pages, page_table, length, q_offset=None, granted=None):
    """New keys and values [T, n_kv_heads, head_dim] to their pages
    (tl_kv_append).  Pages are [n_pages, n_kv_heads, page_tokens, head_dim]
    with any strides (``x.transpose(1, 2)`` of token-major pages); page_table
    [B, width] and length [B] int32, length with the new tokens; q_offset
    [B + 1] int64, or None for one token per sequence.  ``granted`` [B + 1] int32
    is what tl_pages_extend gave the sequences: with it the rows of one that
    got less than it has rows (none, where it was refused) are not written; without,
    they are taken for the last of its ``length`` tokens.  No gradients."""
    if key.requires_grad or value.requires_grad or key_pages.requires_grad or value_pages.requires_grad:
        _no_gradients("tl_kv_append")
    device = key_pages.get_device()
    v = _kv_view(key_pages, value_pages, page_table, length, device)
    dtype, (_, heads, _, dim), T = key_pages.dtype, key_pages.shape, key.shape[0]
    ks, vs = _rows3(key, dtype, "key", device, heads, dim), _rows3(value, dtype, "value", device, heads, dim, T)
    if q_offset is not None:
        _need(q_offset, torch.int64, "q_offset", (page_table.shape[0] + 1,), device)
    a = _lib.KvAppendArgs(_APPEND_SIZE, 0, v, T, _p(q_offset), key.data_ptr(), value.data_ptr(), ks[0], ks[1], vs[0],
                          vs[1], None if granted is None else _granted(granted, page_table.shape[0], device))
    check(lib().tl_kv_append(ctypes.byref(a), _stream_on(device)))


def tl_attend(query, key_pages, value_pages, page_table, length, q_offset=None, window=0, sinks=0, scale=None,
              max_length=0, out=None, want_lse=False, workspace=None, granted=None):
    """Attention of the new tokens' queries [T, n_heads, head_dim] over the
    paged cache (tl_attend); the cache as in tl_kv_append, with the new tokens
    already in it.  ``window`` 0 sees every earlier token, else the last
    ``window`` and the first ``sinks``; ``scale`` is head_dim ** -0.5 unless
    given; ``max_length`` is an upper bound of ``length`` where the caller
    knows one.  ``workspace`` is an uint8 tensor (as many bytes as the call can
    use are allocated when None).  Rows of a sequence that ``granted`` ([B + 1]
    int32, tl_pages_extend's) says was refused see nothing.  Returns out [T, n_heads,
    head_dim], and the log-sums [T, n_heads] fp32 too with ``want_lse``.  For serving:
    no gradients (refused where a tensor asks for one)."""
    if (query.requires_grad or key_pages.requires_grad or value_pages.requires_grad
            or out is not None and out.requires_grad):
        _no_gradients("tl_attend")
    window, sinks, max_length = int(window), int(sinks), int(max_length)
    if (window | sinks | max_length) >> 31:
        for name, x in (("window", window), ("sinks", sinks), ("max_length", max_length)):
            _int32(x, name)
    index = key_pages.get_device()
    v = _kv_view(key_pages, value_pages, page_table, length, index)
    dtype, shape, device = key_pages.dtype, query.shape, query.device
    qs = _rows3(query, dtype, "query", index, None, key_pages.shape[3])
    T, heads, dim = shape
    if q_offset is not None:
        _need(q_offset, torch.int64, "q_offset", (page_table.shape[0] + 1,), index)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=device)
    else:
        _need(out, dtype, "out", shape, index)
    lse = torch.empty((T, heads), dtype=torch.float32, device=device) if want_lse else None
    a = _lib.AttendArgs(_ATTEND_SIZE, heads, v, T, _p(q_offset), query.data_ptr(), qs[0], qs[1],
                        dim ** -0.5 if scale is None else float(scale), window, sinks, max_length,
                        out.data_ptr(), _p(lse), None, 0,
                        None if granted is None else _granted(granted, page_table.shape[0], index))
    L, ref = lib(), ctypes.byref(a)
    if workspace is None:
        n = L.tl_attend_workspace_bytes(ref)
        if n:
            workspace = torch.empty(n, dtype=torch.uint8, device=device)
    else:
        _need(workspace, torch.uint8, "workspace", None, index)
    if workspace is not None:
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    check(L.tl_attend(ref, _stream_on(index)))
    return (out, lse) if want_lse else out


def _summaries(bounds, scale, n_pages, heads, dim, device):
    """The checked summaries' stride between the scales of pages."""
    if (bounds is None or bounds.get_device() != device or bounds.dtype != torch.int8
            or bounds.shape != (n_pages, heads, 2, dim) or not bounds.is_contiguous()):
        _need(bounds, torch.int8, "bounds", (n_pages, heads, 2, dim), device)
    if (scale is None or scale.get_device() != device or scale.dtype != torch.float32
            or scale.shape != (n_pages, heads) or heads > 1 and scale.stride(1) != 1):
        if scale is None or scale.shape != (n_pages, heads) or scale.stride(1) != 1:
            _need(scale, torch.float32, "scale", (n_pages, heads), device)
        _need(scale[:1], torch.float32, "scale", None, device)      # its device and type
    return scale.stride(0) if n_pages > 1 else heads


def tl_page_bounds(key_pages, bounds, scale, page_table, length, n_tokens, q_offset=None, granted=None):
    """The summaries of the pages that the ``n_tokens`` new tokens lie in, in
    place (tl_page_bounds), after tl_kv_append has written their keys: ``bounds``
    [n_pages, n_kv_heads, 2, head_dim] int8 and ``scale`` [n_pages, n_kv_heads]
    fp32 (its rows any distance apart).  The cache, ``q_offset`` and ``granted`` as in
    tl_kv_append.  No gradients."""
    if key_pages.requires_grad or scale.requires_grad:
        _no_gradients("tl_page_bounds")
    n_tokens, device = int(n_tokens), key_pages.get_device()
    v = _kv_view(key_pages, key_pages, page_table, length, device)
    n_pages, heads, _, dim = key_pages.shape
    stride = _summaries(bounds, scale, n_pages, heads, dim, device)
    if q_offset is not None:
        _need(q_offset, torch.int64, "q_offset", (page_table.shape[0] + 1,), device)
    if n_tokens >> 31 or page_table.shape[1] >> 31:
        _int32(n_tokens, "n_tokens")
        _int32(page_table.shape[1], "table_width")
    a = _lib.PageBoundsArgs(_BOUNDS_SIZE, 0, v, n_tokens, _p(q_offset), bounds.data_ptr(), scale.data_ptr(), stride,
                            None if granted is None else _granted(granted, page_table.shape[0], device))
    check(lib().tl_page_bounds(ctypes.byref(a), _stream_on(device)))


def tl_select_pages(query, bounds, scale, page_table, length, page_tokens, n_select, q_offset=None, first=1, last=1,
                    out=None, workspace=None, granted=None):
    """The ``n_select`` pages that score best for each new token and KV head by
    their summaries (tl_page_bounds'), of them the ``first`` and the ``last`` ones always
    (tl_select_pages).  ``query`` [T, n_heads, head_dim]; table, length, ``q_offset``
    and ``granted`` as in tl_attend.  ``workspace`` is an uint8 tensor (allocated when
    None).  Returns [T, n_kv_heads, n_select] int32, places in the table's rows,
    ascending, -1 behind them where a token has fewer.  No gradients: the choice has
    none (refused where a tensor asks for one)."""
    if query.requires_grad or scale.requires_grad:
        _no_gradients("tl_select_pages")
    page_tokens, n_select, first, last = int(page_tokens), int(n_select), int(first), int(last)
    if (page_tokens | n_select | first | last) >> 31:
        for name, x in (("page_tokens", page_tokens), ("n_select", n_select), ("first", first), ("last", last)):
            _int32(x, name)
    index = query.get_device()
    kind = _KV_DTYPES.get(query.dtype)
    if kind is None:
        raise ValueError(f"query must be bfloat16 or float16, got {query.dtype}")
    if index < 0:
        raise ValueError("query must be a device tensor")
    if bounds is None or bounds.dim() != 4:
        raise ValueError("bounds must be [n_pages, n_kv_heads, 2, head_dim]")
    n_pages, kv_heads, _, dim = bounds.shape
    qs = _rows3(query, query.dtype, "query", index, None, dim)
    T, heads, _ = query.shape
    stride = _summaries(bounds, scale, n_pages, kv_heads, dim, index)
    if page_table is None or page_table.dim() != 2:
        raise ValueError("page_table must be [n_seqs, table_width]")
    n_seqs, width = page_table.shape
    if (heads | kv_heads | dim | width) >> 31:
        for name, n in (("heads", heads), ("n_kv_heads", kv_heads), ("head_dim", dim), ("table_width", width)):
            _int32(n, name)
    if page_table.get_device() != index or page_table.dtype != torch.int32 or not page_table.is_contiguous():
        _need(page_table, torch.int32, "page_table", None, index)
    if (length is None or length.get_device() != index or length.dtype != torch.int32 or not length.is_contiguous()
            or length.shape != (n_seqs,)):
        _need(length, torch.int32, "length", (n_seqs,), index)
    if q_offset is not None:
        _need(q_offset, torch.int64, "q_offset", (n_seqs + 1,), index)
    if out is None:
        out = torch.empty((T, kv_heads, n_select), dtype=torch.int32, device=query.device)
    else:
        _need(out, torch.int32, "out", (T, kv_heads, n_select), index)
    v = _lib.KvView(_VIEW_SIZE, kind, kv_heads, dim, page_tokens, width, n_pages, n_seqs, 0, 0, 0, None, None,
                    page_table.data_ptr(), length.data_ptr())
    a = _lib.SelectPagesArgs(_SELECT_SIZE, heads, v, T, _p(q_offset), query.data_ptr(), qs[0], qs[1], bounds.data_ptr(),
                             scale.data_ptr(), stride, n_select, first, last, 0, out.data_ptr(), None, 0,
                             None if granted is None else _granted(granted, n_seqs, index))
    L, ref = lib(), ctypes.byref(a)
    if workspace is None:
        n = L.tl_select_pages_workspace_bytes(ref)
        if n:
            workspace = torch.empty(n, dtype=torch.uint8, device=query.device)
    else:
        _need(workspace, torch.uint8, "workspace", None, index)
    if workspace is not None:
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    check(L.tl_select_pages(ref, _stream_on(index)))
    return out


def tl_attend_pages(query, key_pages, value_pages, page_table, length, selected, q_offset=None, scale=None, out=None,
                    want_lse=False, workspace=None, granted=None):
    """Attention of the new tokens' queries over the pages that ``selected``
    [T, n_kv_heads, n_select] int32 (tl_select_pages') names for each of them and KV
    head (tl_attend_pages).  The rest is as in tl_attend.  For serving: no gradients
    (refused where a tensor asks for one)."""
    if (query.requires_grad or key_pages.requires_grad or value_pages.requires_grad
            or out is not None and out.requires_grad):
        _no_gradients("tl_attend_pages")
    index = key_pages.get_device()
    v = _kv_view(key_pages, value_pages, page_table, length, index)
    dtype, shape, device = key_pages.dtype, query.shape, query.device
    qs = _rows3(query, dtype, "query", index, None, key_pages.shape[3])
    T, heads, dim = shape
    if (selected is None or selected.get_device() != index or selected.dtype != torch.int32 or selected.dim() != 3
            or selected.shape[:2] != (T, key_pages.shape[1]) or not selected.is_contiguous()):
        _need(selected, torch.int32, "selected", None, index)
        raise ValueError(f"selected must be [{T}, {key_pages.shape[1]}, n_select], got {tuple(selected.shape)}")
    if (heads | selected.shape[2] | page_table.shape[1]) >> 31:
        for name, n in (("heads", heads), ("n_select", selected.shape[2]), ("table_width", page_table.shape[1])):
            _int32(n, name)
    if q_offset is not None:
        _need(q_offset, torch.int64, "q_offset", (page_table.shape[0] + 1,), index)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=device)
    else:
        _need(out, dtype, "out", shape, index)
    lse = torch.empty((T, heads), dtype=torch.float32, device=device) if want_lse else None
    a = _lib.AttendArgs(_ATTEND_SIZE, heads, v, T, _p(q_offset), query.data_ptr(), qs[0], qs[1],
                        dim ** -0.5 if scale is None else float(scale), 0, 0, 0, out.data_ptr(), _p(lse), None, 0,
                        None if granted is None else _granted(granted, page_table.shape[0], index))
    a = _lib.AttendPagesArgs(_ATTEND_PAGES_SIZE, selected.shape[2], a, selected.data_ptr())
    L, ref = lib(), ctypes.byref(a)
    if workspace is None:
        n = L.tl_attend_pages_workspace_bytes(ref)
        if n:
            workspace = torch.empty(n, dtype=torch.uint8, device=device)
    else:
        _need(workspace, torch.uint8, "workspace", None, index)
    if workspace is not None:
        a.attend.workspace, a.attend.workspace_bytes = workspace.data_ptr(), workspace.numel()
    check(L.tl_attend_pages(ref, _stream_on(index)))
    return (out, lse) if want_lse else out


def _rows2(t, name, dtype=None, shape=None, device=None):
    """The stride between the rows of ``t`` [rows, columns]."""
    if t is not None and t.is_cuda and (device is None or t.get_device() == device) and t.dim() == 2:
        rows, cols = size = t.shape
        step, one = t.stride()
        if (dtype is None or t.dtype == dtype) and (shape is None or size == shape) and (one == 1 or cols <= 1):
            return step if rows > 1 else cols
    if t is None or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if device is not None and t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, other tensors are on cuda:{device}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 2 or shape is not None and t.shape != shape:
        raise ValueError(f"{name} must be " + ("[rows, columns]" if shape is None else f"{tuple(shape)}")
                         + f", got {tuple(t.shape)}")
    raise ValueError(f"{name} must have contiguous rows")


def tl_norm(x, weight, eps=1e-6, residual=None, group=None, out=None, sum_out=None):
    """The norm before a product: h / sqrt(mean h^2 + eps) * weight per row of
    h = x (+ residual), x [rows, columns] (tl_norm).  Returns y in x's type; with
    ``group`` (q, scale), y in 8 bits (float8_e4m3fn) with a scale a row (0) or for
    ``group`` columns (a power of two from 16 to 512).  With ``residual`` the sum h comes
    last.  ``out`` and ``sum_out`` (contiguous; ``sum_out=residual`` adds in place)
    take y or q, and h.  No gradients (refused where a tensor asks for one)."""
    if (x.requires_grad or weight.requires_grad or residual is not None and residual.requires_grad):
        _no_gradients("tl_norm")
    dtype, shape, device = x.dtype, x.shape, x.get_device()
    kind = _DTYPES.get(dtype)
    if kind is None:
        raise ValueError(f"x must be bfloat16, float16 or float32, got {dtype}")
    xs = _rows2(x, "x")
    rows, cols = shape
    if cols >> 31:
        _int32(cols, "columns")
    if weight.get_device() != device or weight.dtype != dtype or weight.shape != (cols,) or not weight.is_contiguous():
        _need(weight, dtype, "weight", (cols,), device)
    number, kept, scale = _lib.NORM_SAME, dtype, None
    if group is not None:
        number, kept = int(group), torch.float8_e4m3fn
        if number < 0 or number >> 31:
            raise ValueError(f"group {number} is neither 0 nor a power of two from 16 to 512")
        scale = torch.empty((rows, -(-cols // number)) if number else (rows,), dtype=torch.float32, device=x.device)
    if out is None:
        out = torch.empty(shape, dtype=kept, device=x.device)
    else:
        _need(out, kept, "out", shape, device)
    rs = r = total = None
    if residual is not None:
        rs, r = _rows2(residual, "residual", dtype, shape, device), residual.data_ptr()
        if sum_out is None:
            sum_out = torch.empty(shape, dtype=dtype, device=x.device)
        else:
            _need(sum_out, dtype, "sum_out", shape, device)
        total = sum_out.data_ptr()
    elif sum_out is not None:
        raise ValueError("sum_out needs residual")
    a = _lib.NormArgs(_NORM_SIZE, kind, rows, cols, number, eps, 0, x.data_ptr(), r, weight.data_ptr(), xs, rs or 0,
                      out.data_ptr(), None if scale is None else scale.data_ptr(), total)
    check(lib().tl_norm(ctypes.byref(a), _stream_on(device)))
    if group is None:
        return out if residual is None else (out, sum_out)
    return (out, scale) if residual is None else (out, scale, sum_out)


def tl_sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, want_logprob=False, out=None):
    """The next tokens of rows of logits [rows, tokens], drawn with the numbers
    ``u`` [rows] fp32 in [0, 1) (tl_sample).  ``temperature``, ``top_p``, ``min_p`` fp32
    and ``top_k`` int32 are [rows], or None: 1 and no filter.  Returns token [rows]
    int32, and its log-probability among the kept ones [rows] fp32 too with
    ``want_logprob``.  No gradients (refused where the logits ask for them)."""
    if logits.requires_grad:
        _no_gradients("tl_sample")
    device, kind = logits.get_device(), _DTYPES.get(logits.dtype)
    if kind is None:
        raise ValueError(f"logits must be bfloat16, float16 or float32, got {logits.dtype}")
    stride = _rows2(logits, "logits")
    rows, cols = logits.shape
    if cols >> 31:
        _int32(cols, "columns")
    row = (rows,)
    _need(u, torch.float32, "u", row, device)
    for name, t in (("temperature", temperature), ("top_p", top_p), ("min_p", min_p)):
        if t is not None:
            _need(t, torch.float32, name, row, device)
    if top_k is not None:
        _need(top_k, torch.int32, "top_k", row, device)
    if out is None:
        out = torch.empty(row, dtype=torch.int32, device=logits.device)
    else:
        _need(out, torch.int32, "out", row, device)
    logprob = torch.empty(row, dtype=torch.float32, device=logits.device) if want_logprob else None
    a = _lib.SampleArgs(_SAMPLE_SIZE, kind, rows, cols, 0, logits.data_ptr(), stride, u.data_ptr(), _p(temperature),
                        _p(top_k), _p(top_p), _p(min_p), out.data_ptr(), _p(logprob))
    check(lib().tl_sample(ctypes.byref(a), _stream_on(device)))
    return (out, logprob) if want_logprob else out


def _pages(ref, page_table, length, page_tokens, granted=None):
    page_tokens = int(page_tokens)
    if page_tokens >> 31:
        _int32(page_tokens, "page_tokens")
    _need(ref, torch.int32, "ref")
    device = ref.get_device()
    if (page_table is None or page_table.get_device() != device or page_table.dtype != torch.int32
            or not page_table.is_contiguous()):
        _need(page_table, torch.int32, "page_table", None, device)
    if ref.dim() != 1 or page_table.dim() != 2:
        raise ValueError("ref must be [n_pages] and page_table [n_slots, table_width]")
    n_slots, width = page_table.shape
    if (length is None or length.get_device() != device or length.dtype != torch.int32 or length.shape != (n_slots,)
            or not length.is_contiguous()):
        _need(length, torch.int32, "length", (n_slots,), device)
    return _lib.Pages(_PAGES_SIZE, page_tokens, ref.shape[0], n_slots, width, 0, ref.data_ptr(),
                      page_table.data_ptr(), length.data_ptr(),
                      None if granted is None else _granted(granted, n_slots, device))


def _pages_work(g, ref, work):
    """`work` for the pool's calls on ``g``, checked or allocated."""
    words = lib().tl_pages_work_words(ctypes.byref(g))
    if work is None:
        return torch.empty(words, dtype=torch.int32, device=ref.device)
    if _need(work, torch.int32, "work", None, ref.get_device()).numel() < words:
        raise ValueError("work is too small (tl_pages_work_words)")
    return work


def tl_pages_extend(ref, page_table, length, add, page_tokens, status=None, work=None, granted=None):
    """Room for ``add`` [n_slots] int32 more tokens in every slot, in place
    (tl_pages_extend).  Returns status [n_slots] int32 (PAGES_* codes).
    ``granted`` [n_slots + 1] int32 (its last word not 0 at first) keeps what
    each slot got since the last append, for tl_kv_append and tl_attend."""
    g = _pages(ref, page_table, length, page_tokens, granted)
    work = _pages_work(g, ref, work)
    device = ref.get_device()
    _need(add, torch.int32, "add", (g.n_slots,), device)
    if status is None:
        status = torch.empty(g.n_slots, dtype=torch.int32, device=ref.device)
    _need(status, torch.int32, "status", (g.n_slots,), device)
    check(lib().tl_pages_extend(ctypes.byref(g), _p(add), _p(status), _p(work), _stream_on(device)))
    return status


def tl_pages_fork(ref, page_table, length, parent, child, page_tokens, work=None, granted=None):
    """Empty slots ``child`` become copies of slots ``parent`` (int32 [F]), in
    place (tl_pages_fork; ``granted`` as in tl_pages_extend).  Returns (copy_src,
    copy_dst, status) int32 [F]; the pages still have to be copied (tl_pages_copy)."""
    g = _pages(ref, page_table, length, page_tokens, granted)
    work = _pages_work(g, ref, work)
    F, device = parent.numel(), ref.get_device()
    _need(parent, torch.int32, "parent", (F,), device)
    _need(child, torch.int32, "child", (F,), device)
    src, dst, status = torch.empty((3, F), dtype=torch.int32, device=ref.device).unbind(0)
    check(lib().tl_pages_fork(ctypes.byref(g), F, _p(parent), _p(child), _p(src), _p(dst), _p(status), _p(work),
                              _stream_on(device)))
    return src, dst, status


def tl_pages_free(ref, page_table, length, slots, page_tokens):
    """The sequences in ``slots`` (int32) leave, in place (tl_pages_free)."""
    g = _pages(ref, page_table, length, page_tokens)
    device = ref.get_device()
    _need(slots, torch.int32, "slots", None, device)
    check(lib().tl_pages_free(ctypes.byref(g), slots.numel(), _p(slots), _stream_on(device)))


def tl_pages_compact(ref, page_table, length, page_tokens, out=None, work=None):
    """The live pages to the front of the pool (tl_pages_compact).  Returns a
    dict with the state after it (ref, page_table; taken from ``out``, which may
    hold the arguments themselves, or allocated) and the moves (copy_src,
    copy_dst, n_copies [1], all int32), which tl_pages_copy has to make."""
    g = _pages(ref, page_table, length, page_tokens)
    o, half, device = out or {}, ref.shape[0] // 2, ref.get_device()
    # what is not given comes in as few allocations as can be
    sizes = [half, half, 1, lib().tl_pages_work_words(ctypes.byref(g)) if work is None else 0]
    moves = list(torch.empty(sum(sizes), dtype=torch.int32, device=ref.device).split(sizes))
    work = moves.pop() if work is None else _pages_work(g, ref, work)

    def buf(name, shape, default=None):
        t = o.get(name)
        if t is None:
            return torch.empty(shape, dtype=torch.int32, device=ref.device) if default is None else default
        return _need(t, torch.int32, name, shape, device)

    r = dict(ref=buf("ref", ref.shape), page_table=buf("page_table", page_table.shape),
             copy_src=buf("copy_src", (half,), moves[0]), copy_dst=buf("copy_dst", (half,), moves[1]),
             n_copies=buf("n_copies", (1,), moves[2]))
    check(lib().tl_pages_compact(ctypes.byref(g), _p(r["ref"]), _p(r["page_table"]), _p(r["copy_src"]),
                                 _p(r["copy_dst"]), _p(r["n_copies"]), _p(work), _stream_on(device)))
    return r


def tl_pages_copy(pages, copy_src, copy_dst, n_copies=None):
    """Pages ``copy_src`` to ``copy_dst`` (int32) in every plane of ``pages``
    [..., n_pages, n_kv_heads, page_tokens, head_dim] (contiguous; the leading
    dimensions are planes); only the first ``n_copies`` (int32 [1], on the
    device) when given (tl_pages_copy)."""
    if not pages.is_cuda or not pages.is_contiguous() or pages.dim() < 4:
        raise ValueError("pages must be a contiguous device tensor [..., n_pages, n_kv_heads, page_tokens, head_dim]")
    n, device = copy_src.numel(), pages.get_device()
    _need(copy_src, torch.int32, "copy_src", (n,), device)
    _need(copy_dst, torch.int32, "copy_dst", (n,), device)
    if n_copies is not None:
        _need(n_copies, torch.int32, "n_copies", (1,), device)
    n_pages = pages.shape[-4]
    page = pages.shape[-3] * pages.shape[-2] * pages.shape[-1] * pages.element_size()
    planes = pages.numel() * pages.element_size() // (page * n_pages) if page * n_pages else 0
    check(lib().tl_pages_copy(_p(pages), n_pages, page, page, planes, page * n_pages, _p(copy_src), _p(copy_dst), n,
                              _p(n_copies), _stream_on(device)))


class KVCache:
    """A paged cache of ``n_layers`` layers and the sequences in its slots:
    pages of ``page_tokens`` tokens, the page table, the lengths and the pages'
    counts, all on the device.  One iteration of an engine extends the slots
    by their new tokens, then appends and attends in every layer; finished
    sequences are freed.  With ``summaries`` append keeps those of the pages up
    to date too, which select looks for the pages in that attend_pages then reads.  Where the pool has no room for a slot, nothing of what
    the others do depends on it, and its cached tokens stay as they are.  Nothing here
    waits for the device."""

    def __init__(self, n_layers, n_pages, n_kv_heads, page_tokens, head_dim, n_slots, max_tokens,
                 dtype=torch.bfloat16, device="cuda", summaries=False):
        if dtype not in _KV_DTYPES:
            raise ValueError(f"dtype must be bfloat16 or float16, got {dtype}")
        self.page_tokens, self.max_tokens = int(page_tokens), int(max_tokens)
        width = -(-self.max_tokens // self.page_tokens)
        i32 = dict(dtype=torch.int32, device=device)
        self.pages = torch.empty((n_layers, 2, n_pages, n_kv_heads, page_tokens, head_dim), dtype=dtype, device=device)
        self.bounds = self.scales = None
        if summaries:
            self.bounds = torch.zeros((n_layers, n_pages, n_kv_heads, 2, head_dim), dtype=torch.int8, device=device)
            # (whole 16 bytes a page, which tl_pages_copy moves)
            self.scales = torch.zeros((n_layers, n_pages, 1, 1, -(-n_kv_heads // 4) * 4), device=device)
        self.ref = torch.zeros(n_pages, **i32)
        self.page_table = torch.full((n_slots, width), -1, **i32)
        self.length = torch.zeros(n_slots, **i32)
        # what extend gave since the last append (before the first one: no limit)
        self.granted = torch.full((n_slots + 1,), 2 ** 31 - 1, **i32)
        g = _lib.Pages(_PAGES_SIZE, self.page_tokens, n_pages, n_slots, width, 0, _p(self.ref),
                       _p(self.page_table), _p(self.length))
        self.work = torch.empty(lib().tl_pages_work_words(ctypes.byref(g)), **i32)

    def _state(self):
        return self.ref, self.page_table, self.length

    def extend(self, add, status=None):
        """Room for ``add`` [n_slots] new tokens; returns the statuses.  A slot
        that is refused keeps its length and its tokens: rows that it has in append
        all the same are not written, and in attend they give zeros."""
        return tl_pages_extend(*self._state(), add, self.page_tokens, status, self.work, self.granted)

    def append(self, layer, key, value, q_offset=None):
        """The new tokens' keys and values (after extend) into one layer.  Slots
        with more rows than tokens that they got since the last append (refused ones,
        and without ``q_offset`` those that asked for none) are left as they are."""
        k, v = self.pages[layer]
        tl_kv_append(key, value, k, v, self.page_table, self.length, q_offset, self.granted)
        if self.bounds is not None:
            bounds, scale = self._summaries(layer)
            tl_page_bounds(k, bounds, scale, self.page_table, self.length, key.shape[0], q_offset, self.granted)

    def _summaries(self, layer):
        if self.bounds is None:
            raise ValueError("the cache was made without summaries")
        return self.bounds[layer], self.scales[layer, :, 0, 0, :self.bounds.shape[2]]

    def select(self, layer, query, n_select, q_offset=None, **kw):
        """The pages of one layer that score best for the new tokens (after
        append; tl_select_pages)."""
        bounds, scale = self._summaries(layer)
        return tl_select_pages(query, bounds, scale, self.page_table, self.length, self.page_tokens, n_select, q_offset,
                               granted=self.granted, **kw)

    def attend_pages(self, layer, query, selected, q_offset=None, **kw):
        """The new tokens' attention over the selected pages of one layer."""
        k, v = self.pages[layer]
        return tl_attend_pages(query, k, v, self.page_table, self.length, selected, q_offset, granted=self.granted, **kw)

    def attend(self, layer, query, q_offset=None, **kw):
        """The new tokens' attention over one layer (after append); zeros for
        tokens that extend refused."""
        k, v = self.pages[layer]
        return tl_attend(query, k, v, self.page_table, self.length, q_offset, granted=self.granted, **kw)

    def fork(self, parent, child):
        """Empty slots ``child`` become copies of ``parent``; returns the
        statuses.  (The summary of a copied page is made with the child's first new
        token, which lies in it.)"""
        src, dst, status = tl_pages_fork(*self._state(), parent, child, self.page_tokens, self.work, self.granted)
        tl_pages_copy(self.pages, src, dst)
        return status

    def free(self, slots):
        """The sequences in ``slots`` leave."""
        tl_pages_free(*self._state(), slots, self.page_tokens)

    def compact(self):
        """The live pages to the front of the pool; returns the number of
        pages moved (int32 [1], on the device)."""
        r = tl_pages_compact(*self._state(), self.page_tokens, dict(ref=self.ref, page_table=self.page_table),
                             self.work)
        for pages in (self.pages, self.bounds, self.scales):
            if pages is not None:
                tl_pages_copy(pages, r["copy_src"], r["copy_dst"], r["n_copies"])
        return r["n_copies"]

    def pages_used(self):
        """Pages in use (int64 scalar, on the device)."""
        return (self.ref > 0).sum()


# short names
project = tl_project
select_freq = tl_select_freq
select_freq_binary = tl_select_freq_binary
admit = tl_admit
adjust_lengths = tl_adjust_lengths
kv_append = tl_kv_append
attend = tl_attend
page_bounds = tl_page_bounds
select_pages = tl_select_pages
attend_pages = tl_attend_pages
norm = tl_norm
sample = tl_sample


def upload(inp, device="cuda"):
    """Copy a numpy input dict (``synth.make_inputs``) to device tensors."""
    def t(a, dtype=None):
        if a is None:
            return None
        a = np.ascontiguousarray(a)
        if a.dtype == np.uint64:
            a = a.view(np.int64)
        if a.dtype == np.uint32:
            a = a.view(np.int32)
        return torch.from_numpy(a).to(device)

    return dict(
        n_scenarios=int(inp["n_scenarios"]), horizon=int(inp["horizon"]),
        block_tokens=int(inp["block_tokens"]), n_features=int(inp["n_features"]),
        req_offset=t(inp["req_offset"]), prompt=t(inp["prompt"]), generated=t(inp["generated"]),
        remaining=t(inp["remaining"]), arrival=t(inp["arrival"]), deadline_ns=t(inp.get("deadline_ns")),
        lost=t(inp.get("lost")), kv_capacity=t(inp["kv_capacity"]), batch_cap=t(inp.get("batch_cap")),
        tbt_slo_ns=t(inp["tbt_slo_ns"]), freqs_mhz=t(inp["freqs_mhz"]),
        engine_size=t(inp.get("engine_size")),
    )


class Controller:
    """The whole hot path for one batch of scenarios: project -> predict ->
    select, enqueued back to back on the current stream with preallocated
    buffers (no host round trip between stages).

    By default the feature rows are formed inside the forest kernel
    (tl_forest_predict_grid); with ``materialize_rows=True`` tl_project writes
    them and tl_forest_predict reads them back (same results)."""

    def __init__(self, dev_inputs, forest, materialize_rows=False):
        self.d = dev_inputs
        self.forest = forest
        self.materialize_rows = materialize_rows
        d = dev_inputs
        S, H = d["n_scenarios"], d["horizon"]
        F, nf = d["freqs_mhz"].numel(), d["n_features"]
        dev = d["req_offset"].device
        self.buf = dict(
            batch=torch.empty((S, H), dtype=torch.int32, device=dev),
            kv=torch.empty((S, H), dtype=torch.int32, device=dev),
            deadline_at=torch.empty((S, H), dtype=torch.int64, device=dev),
            n_iters=torch.empty(S, dtype=torch.int32, device=dev),
            flags=torch.empty(S, dtype=torch.int32, device=dev),
        )
        if materialize_rows:
            self.buf["rows"] = torch.empty((S, F, H, nf), dtype=torch.float32, device=dev)
        self.ips = torch.empty((S, F, H), dtype=torch.float32, device=dev)
        self.sel = dict(freq_idx=torch.empty(S, dtype=torch.int32, device=dev),
                        status=torch.empty(S, dtype=torch.int32, device=dev))

    def project(self):
        d = self.d
        return tl_project(d["req_offset"], d["prompt"], d["generated"], d["remaining"], d["arrival"],
                          d["kv_capacity"], d["horizon"], d["block_tokens"], d["deadline_ns"],
                          d["lost"], d["batch_cap"], d["freqs_mhz"], d["engine_size"],
                          d["n_features"], self.materialize_rows, self.buf)

    def predict(self):
        if self.materialize_rows:
            return self.forest.tl_forest_predict(self.buf["rows"], self.ips)
        return self.forest.tl_forest_predict_grid(self.d["freqs_mhz"], self.buf["kv"], self.buf["batch"],
                                                  self.d["engine_size"], self.ips)

    def select(self):
        return tl_select_freq(self.ips, self.buf["deadline_at"], self.buf["n_iters"],
                              self.d["tbt_slo_ns"], self.buf["flags"], self.sel)

    def step(self):
        self.project()
        self.predict()
        return self.select()

    def select_binary(self, lattice=None):
        """The paper's binary search over the frequencies on the projection
        (tl_select_freq_binary): the model only at probed frequencies, read
        from ``lattice`` when given."""
        d, b = self.d, self.buf
        if "search" not in self.__dict__:
            S, H = d["n_scenarios"], d["horizon"]
            dev = d["req_offset"].device
            self.search = dict(ips_work=torch.empty((S, H), dtype=torch.float32, device=dev),
                               search_work=torch.empty((3, S), dtype=torch.int32, device=dev),
                               freq_idx=torch.empty(S, dtype=torch.int32, device=dev),
                               status=torch.empty(S, dtype=torch.int32, device=dev))
        return tl_select_freq_binary(self.forest, d["freqs_mhz"], b["kv"], b["batch"], b["deadline_at"],
                                     b["n_iters"], d["tbt_slo_ns"], b["flags"], d["engine_size"], self.search,
                                     lattice)
