"""Python binding of the DriveCache C ABI (include/dc.h).

Functions keep the C names; they marshal torch tensors (device memory, owned by
the caller) and numpy arrays (host) into the C calls.  Every computation runs in
libdrivecache.so; nothing here computes.
"""
from __future__ import annotations

import ctypes as C
import struct

import numpy as np

from . import _lib as L
from .inputs import ModelShape, SchedProblem as PySchedProblem

__all__ = ["model_cfg", "DeviceModel", "Workspace", "SamplerBuffers", "profile", "dc_workspace_bytes", "dc_time_modulation",
           "dc_patch_embed", "dc_block_forward", "dc_cache_store", "dc_cache_apply",
           "dc_drift_l1", "dc_head_euler", "dc_schedule_dp", "dc_select_tau", "dc_motion_statistics",
           "dc_select_anchors", "Sampler", "rope_axes", "dc_rope_table", "dc_qk_norm_rope", "dc_quantize_rows",
           "dc_linear_i8", "dc_quantize_f8", "dc_rms_norm_f8", "dc_linear_f8", "dc_cache_store_q", "dc_cache_apply_q", "BlockExt",
           "dc_block_forward_ext"]


def _torch():
    import torch
    return torch


def _ptr(t):
    return C.c_void_p(0 if t is None else int(t.data_ptr()))


def _stream(stream=None):
    torch = _torch()
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(int(s.cuda_stream))


def _idx(idx):
    arr = np.ascontiguousarray(np.asarray(idx, dtype=np.int32))
    return arr, arr.ctypes.data_as(L.i32p), int(arr.size)


def model_cfg(m: ModelShape) -> L.ModelCfg:
    return L.ModelCfg(m.n_blocks, m.hidden, m.heads, m.head_dim, m.mlp_hidden, m.lat_c, m.lat_t,
                      m.lat_h, m.lat_w, m.patch, m.n_txt, L.DC_BF16 if m.dtype == "bf16" else L.DC_F32,
                      m.ln_eps)


class DeviceModel:
    """Generator weights uploaded to the GPU in the library's layout."""

    MATRICES = ("w_qkv", "w_o", "w_1", "w_2")

    def __init__(self, W, device="cuda:0"):
        torch = _torch()
        self.m = W.m
        self.cfg = model_cfg(W.m)
        self.device = device
        mdt = torch.bfloat16 if W.m.dtype == "bf16" else torch.float32

        def up(a, dt=torch.float32):
            return torch.from_numpy(np.ascontiguousarray(a)).to(device=device, dtype=dt)

        self.g = {}
        for name in ("w_pe", "b_pe", "w_t1", "b_t1", "w_t2", "b_t2", "w_m", "b_m", "head_mod", "b_head"):
            self.g[name] = up(W.get(name))
        self.g["pos"] = up(W.get("pos"), mdt)
        self.g["w_head"] = up(W.get("w_head"), mdt)
        self.blocks = []
        for l in range(W.m.n_blocks):
            b = {}
            for name in ("w_qkv", "b_qkv", "w_o", "b_o", "w_1", "b_1", "w_2", "b_2", "mod_offset"):
                b[name] = up(W.block(l, name), mdt if name in self.MATRICES else torch.float32)
            self.blocks.append(b)
        self._cblocks = (L.BlockWeights * W.m.n_blocks)()
        for l, b in enumerate(self.blocks):
            self._cblocks[l] = L.BlockWeights(*[_ptr(b[n]) for n in (
                "w_qkv", "b_qkv", "w_o", "b_o", "w_1", "b_1", "w_2", "b_2", "mod_offset")])
        gw = self.g
        self.cweights = L.ModelWeights(
            _ptr(gw["w_pe"]), _ptr(gw["b_pe"]), _ptr(gw["pos"]), _ptr(gw["w_t1"]), _ptr(gw["b_t1"]),
            _ptr(gw["w_t2"]), _ptr(gw["b_t2"]), _ptr(gw["w_m"]), _ptr(gw["b_m"]), _ptr(gw["head_mod"]),
            _ptr(gw["w_head"]), _ptr(gw["b_head"]), self._cblocks)

    def block(self, l):
        return C.pointer(self._cblocks[l])


def dc_workspace_bytes(m: ModelShape, batch: int = 1) -> int:
    cfg = model_cfg(m)
    n = L.load().dc_workspace_bytes(C.byref(cfg), batch)
    if n == 0:
        raise L.DriveCacheError("dc_workspace_bytes", L.DC_ERR_SHAPE, "unsupported shape")
    return int(n)


class Workspace:
    """Device scratch of dc_workspace_bytes() bytes (256-byte aligned); ext: of
    dc_block_ext_workspace_bytes(), for extended blocks."""

    def __init__(self, m: ModelShape, batch=1, device="cuda:0", ext=False):
        torch = _torch()
        self.nbytes = dc_workspace_bytes(m, batch)
        if ext:
            self.nbytes = int(L.load().dc_block_ext_workspace_bytes(C.byref(model_cfg(m)), batch))
        self.buf = torch.empty(self.nbytes + 256, dtype=torch.uint8, device=device)
        off = (-int(self.buf.data_ptr())) % 256
        self.ptr = C.c_void_p(int(self.buf.data_ptr()) + off)


def dc_time_modulation(dm: DeviceModel, sigmas, mod, ws: Workspace, stream=None):
    sig = np.ascontiguousarray(np.asarray(sigmas, np.float64))
    L.check("dc_time_modulation", L.load().dc_time_modulation(
        C.byref(dm.cfg), C.byref(dm.cweights), sig.ctypes.data_as(C.POINTER(C.c_double)), int(sig.size),
        _ptr(mod), ws.ptr, ws.nbytes, _stream(stream)))


def dc_patch_embed(dm: DeviceModel, x, txt, h_in, idx, ws: Workspace, stream=None):
    arr, p, n = _idx(idx)
    L.check("dc_patch_embed", L.load().dc_patch_embed(
        C.byref(dm.cfg), C.byref(dm.cweights), _ptr(x), _ptr(txt), _ptr(h_in), p, n, ws.ptr, ws.nbytes,
        _stream(stream)))


def dc_block_forward(dm: DeviceModel, l: int, mod, h, idx, ws: Workspace, stream=None):
    arr, p, n = _idx(idx)
    L.check("dc_block_forward", L.load().dc_block_forward(
        C.byref(dm.cfg), dm.block(l), _ptr(mod), _ptr(h), p, n, ws.ptr, ws.nbytes, _stream(stream)))


def dc_cache_store(cfg, h_out, h_in, resid, idx, stream=None):
    arr, p, n = _idx(idx)
    L.check("dc_cache_store", L.load().dc_cache_store(
        C.byref(cfg), _ptr(h_out), _ptr(h_in), _ptr(resid), p, n, _stream(stream)))


def dc_cache_apply(cfg, h_in, resid, g, idx, stream=None):
    arr, p, n = _idx(idx)
    L.check("dc_cache_apply", L.load().dc_cache_apply(
        C.byref(cfg), _ptr(h_in), _ptr(resid), _ptr(g), p, n, _stream(stream)))


def dc_drift_l1(cfg, h_in, mod0, u_ref, snapshot, sums, idx, ws: Workspace, stream=None):
    arr, p, n = _idx(idx)
    L.check("dc_drift_l1", L.load().dc_drift_l1(
        C.byref(cfg), _ptr(h_in), _ptr(mod0), _ptr(u_ref), int(bool(snapshot)), _ptr(sums), p, n,
        ws.ptr, ws.nbytes, _stream(stream)))


def dc_drift_l1_noalloc(cfg, h_in, mod0, u_ref, snapshot, sums, idx, stream=None):
    """dc_drift_l1 without a workspace (the library's fixed per-GPU scratch)."""
    arr, p, n = _idx(idx)
    L.check("dc_drift_l1_noalloc", L.load().dc_drift_l1_noalloc(
        C.byref(cfg), _ptr(h_in), _ptr(mod0), _ptr(u_ref), int(bool(snapshot)), _ptr(sums), p, n,
        _stream(stream)))


def dc_head_euler(dm: DeviceModel, head_mod, g, x, dsigma, idx, ws: Workspace, stream=None):
    arr, p, n = _idx(idx)
    L.check("dc_head_euler", L.load().dc_head_euler(
        C.byref(dm.cfg), C.byref(dm.cweights), _ptr(head_mod), _ptr(g), _ptr(x), float(dsigma), p, n,
        ws.ptr, ws.nbytes, _stream(stream)))


def dc_calibrate_tables(dm: DeviceModel, x1, txt, sigmas, h_max: int, eps: float, stream=None):
    """Anchor calibration of one clip (Eq. 5-7) on the GPU: returns (q, d), f64
    [(K-1), h_max] each.  x1 [C, T, H, W], txt [N_t, d]: the clip's inputs (torch
    tensors on the device); sigmas: the K+1 noise levels.  The network is dm's with plain
    blocks: a model that runs with a BlockExt has other tables."""
    torch = _torch()
    sig = np.ascontiguousarray(np.asarray(sigmas, np.float64))
    K = sig.size - 1
    nbytes = L.load().dc_calibrate_workspace_bytes(C.byref(dm.cfg), K)
    if nbytes == 0:
        raise L.DriveCacheError("dc_calibrate_workspace_bytes", L.DC_ERR_ARG, "bad model or K")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dm.device)
    q = np.zeros((K - 1, h_max), np.float64)
    d = np.zeros((K - 1, h_max), np.float64)
    x1 = x1.to(device=dm.device, dtype=torch.float32).contiguous()
    txt = txt.to(device=dm.device, dtype=torch.float32).contiguous()
    L.check("dc_calibrate_tables", L.load().dc_calibrate_tables(
        C.byref(dm.cfg), C.byref(dm.cweights), _ptr(x1), _ptr(txt),
        sig.ctypes.data_as(C.POINTER(C.c_double)), K, int(h_max), float(eps),
        q.ctypes.data_as(C.POINTER(C.c_double)), d.ctypes.data_as(C.POINTER(C.c_double)),
        int(ws.data_ptr()), nbytes, _stream(stream)))
    return q, d


# ----------------------------------------------------------------------------
# rotary positions, query/key norms, int8 and e4m3 products, quantised cache
# ----------------------------------------------------------------------------
# These calls take a few microseconds on the GPU: binding.cpp checks their tensors (ValueError) and makes the C call.
_current = None         # torch's (raw stream of a device, current device)


def _call(name, stream, first, *args):
    """The binding's function on args, on the current stream of the device that `first` is on (or on `stream`, which
    has to be one of it), with that device current."""
    global _current
    if _current is None:
        torch = _torch()
        _current = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    i = first.get_device()
    if i < 0:
        raise ValueError("tensors must be on a GPU")
    if stream is None:
        s = _current[0](i)
    elif stream.device.index == i:
        s = stream.cuda_stream
    else:
        raise ValueError("the stream belongs to another device")
    f = getattr(L._binding or L.binding(), name)
    if _current[1]() == i:
        rc = f(*args, i, s)
    else:
        with _torch().cuda.device(i):
            rc = f(*args, i, s)
    if rc:
        L.check(name, rc)


_AXES = struct.Struct("3i4x7d")        # dc_rope_axes; a field at a time takes five times as long


def rope_axes(dim, theta=10000.0, start=(0.0, 0.0, 0.0), step=(1.0, 1.0, 1.0)) -> L.RopeAxes:
    """dc_rope_axes: features of a head that turn with time, height and width, and the grid's
    positions start + step * index."""
    try:
        return L.RopeAxes.from_buffer_copy(_AXES.pack(*dim, theta, *start, *step))
    except struct.error as e:
        raise ValueError(f"dim, start and step: three numbers each, dim whole ones: {e}") from e


def dc_rope_table(cfg, axes: L.RopeAxes, pos, table, stream=None):
    """table (f32 [N_v, head_dim / 2, 2]) := cos and sin; pos: f64 [N_v, 3] or None (the grid)."""
    _call("dc_rope_table", stream, table, cfg, axes, pos, table)


def dc_qk_norm_rope(cfg, x, out, idx, q_weight=None, k_weight=None, eps=1e-6, table=None, interleaved=True,
                    q_scale=1.0, stream=None):
    """Norms and rotation of the queries (columns [0, d)) and keys ([d, 2d)) of x [B, N, >= 2d] into out
    (x itself, or a tensor like it): RMS norm with q_weight / k_weight where given, rotation where table is."""
    _call("dc_qk_norm_rope", stream, x, cfg, x, out, idx, q_weight, k_weight, eps, table, interleaved, q_scale)


def dc_quantize_rows(x, q, scale, stream=None):
    """q (int8 [rows, at least cols rounded up to 128]) and scale (f32 [rows]) := the rows of x [rows, cols]."""
    _call("dc_quantize_rows", stream, x, x, q, scale)


def dc_linear_i8(x, x_scale, w, w_scale, out, bias=None, gelu=False, gate=None, residual=None, stream=None):
    """out [M, N] := the product of int8 rows x [M, K] and w [N, K] (K as padded by dc_quantize_rows) with
    their scales, plus bias, through GELU or as residual + gate * (...)."""
    _call("dc_linear_i8", stream, x, x, x_scale, w, w_scale, out, bias, gelu, gate, residual)


def dc_quantize_f8(x, q, scale, block_rows=1, stream=None):
    """q (float8_e4m3fn [rows, at least cols rounded up to 128]) and scale (f32 [rows, cols / 128 rounded up], by rows or by
    blocks at any strides; torch.empty((blocks, rows)).t() is the fastest) := the rows of x [rows, cols], a scale to 128 features.
    block_rows=128: a weight matrix, scale [rows / 128 rounded up, ...], one to 128 x 128 values."""
    _call("dc_quantize_f8", stream, x, x, q, scale, block_rows)


def dc_rms_norm_f8(x, q, scale, weight=None, eps=1e-6, residual=None, out=None, stream=None):
    """q and scale (as dc_quantize_f8's) := the RMS norm of x + residual, times weight (f32 [cols]); out (float32 or
    bfloat16, may be x or residual) := that sum.  x [rows, cols], cols up to 16,384; residual and out like it or None."""
    _call("dc_rms_norm_f8", stream, x, x, q, scale, weight, eps, residual, out)


def dc_linear_f8(x, x_scale, w, w_scale, out, bias=None, gelu=False, gate=None, residual=None, stream=None):
    """out [M, N] := the product of e4m3 rows x [M, K] and w [N, K] (K as padded by dc_quantize_f8) with their scales
    ([M, K / 128], [N / 128 rounded up, K / 128], any strides, x_scale's rows less than 2^21 apart), plus bias, through
    GELU or as residual + gate * (...) (residual of out's type; gate None: 1).  A scale of x times one of w is an fp32
    number: 0, or from 2^-126 to below 2^128."""
    _call("dc_linear_f8", stream, x, x, x_scale, w, w_scale, out, bias, gelu, gate, residual)


def dc_cache_store_q(cfg, bits, h_out, h_in, codes, scales, idx, stream=None):
    """codes (int8 [B, N_v, d], or uint8 [B, N_v, d / 2] for 4 bits) and scales (f32 [B, N_v, d / 64]) :=
    h_out - h_in on the video rows."""
    _call("dc_cache_store_q", stream, h_out, cfg, bits, h_out, h_in, codes, scales, idx)


def dc_cache_apply_q(cfg, bits, h_in, codes, scales, g, idx, stream=None):
    """g := h_in + the cached residual on the video rows (g may be h_in)."""
    _call("dc_cache_apply_q", stream, h_in, cfg, bits, h_in, g, codes, scales, idx)


def _video_tokens(cfg):
    return cfg.lat_t * (cfg.lat_h // cfg.patch) * (cfg.lat_w // cfg.patch)


def _floats(t, shape, device, what):
    if t is None:
        return None
    if t.dtype != _torch().float32 or tuple(t.shape) != shape or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{what}: a contiguous float32 {list(shape)} tensor on {device} is wanted")
    return t.data_ptr()


class BlockExt:
    """Extensions of every block of a DeviceModel: norms and rotation of queries and keys (q_weight,
    k_weight: one [head_dim] tensor per block, or None; table: dc_rope_table's, or None) and, with
    int8=True, the blocks' matrices quantised per output channel (on the current stream)."""

    MATRICES = (("w_qkv", "s_qkv"), ("w_o", "s_o"), ("w_1", "s_1"), ("w_2", "s_2"))

    def __init__(self, dm: DeviceModel, q_weight=None, k_weight=None, eps=1e-6, table=None, interleaved=True,
                 int8=False):
        torch = _torch()
        n = len(dm.blocks)
        self.cfg, self.device = dm.cfg, dm.blocks[0]["b_qkv"].device
        self.keep = [table]             # the tensors themselves: a caller's list may change
        self.c = (L.BlockExt * n)()
        for l, b in enumerate(dm.blocks):
            if q_weight is not None or k_weight is not None or table is not None:
                dh, dev = (dm.cfg.head_dim,), self.device
                wq, wk = (None if w is None else w[l] for w in (q_weight, k_weight))
                qk = L.QkCfg(_floats(wq, dh, dev, "q_weight"), _floats(wk, dh, dev, "k_weight"), eps,
                             _floats(table, (_video_tokens(dm.cfg), dh[0] // 2, 2), dev, "table"), 1 if interleaved else 0)
                self.keep += [wq, wk, qk]
                self.c[l].qk = C.pointer(qk)
            if int8:
                held = L.BlockWeightsI8()
                for name, s_name in self.MATRICES:
                    w = b[name]
                    q = torch.empty(w.shape, dtype=torch.int8, device=w.device)
                    s = torch.empty(w.shape[0], dtype=torch.float32, device=w.device)
                    dc_quantize_rows(w, q, s)
                    setattr(held, name, int(q.data_ptr()))
                    setattr(held, s_name, int(s.data_ptr()))
                    self.keep += [q, s]
                self.keep.append(held)
                self.c[l].i8 = C.pointer(held)

    def block(self, l):
        return C.pointer(self.c[l])

    def of(self, dm):
        """Itself, if it has the shapes and the device of dm: the library reads dm's sizes from what it points to."""
        if bytes(self.cfg) != bytes(dm.cfg):
            raise ValueError("ext was made for a model of another shape")
        if dm.blocks[0]["b_qkv"].device != self.device:
            raise ValueError("ext was made for a model on another device")
        return self


def dc_block_forward_ext(dm: DeviceModel, l: int, ext: BlockExt, mod, h, idx, ws: Workspace, stream=None):
    """dc_block_forward with block l's extensions (None: none); ws: Workspace(..., ext=True)."""
    e = None if ext is None else ext.of(dm).block(l)
    arr, p, n = _idx(idx)
    L.check("dc_block_forward_ext", L.load().dc_block_forward_ext(
        C.byref(dm.cfg), dm.block(l), e, _ptr(mod), _ptr(h), p, n, ws.ptr, ws.nbytes, _stream(stream)))


class _CProblem:
    """A dc_sched_problem whose arrays stay alive with it."""

    def __init__(self, p: PySchedProblem):
        f64 = lambda a: np.ascontiguousarray(np.asarray(a, np.float64))
        self.keep = dict(legal=np.ascontiguousarray(np.asarray(p.legal, np.uint8)),
                         xy=f64(p.pose_xy).reshape(-1), yaw=f64(p.pose_yaw),
                         q0=f64(p.q0).reshape(-1), q1=f64(p.q1).reshape(-1),
                         d0=f64(p.d0).reshape(-1), d1=f64(p.d1).reshape(-1))
        seg = None
        if p.segment is not None:
            self.keep["seg"] = np.ascontiguousarray(np.asarray(p.segment, np.int32))
            seg = self.keep["seg"].ctypes.data_as(C.POINTER(C.c_int32))
        dp = lambda a: a.ctypes.data_as(C.POINTER(C.c_double))
        k = self.keep
        self.c = L.SchedProblem(
            p.K, p.h_max, p.n_cap, k["legal"].ctypes.data_as(C.POINTER(C.c_uint8)), seg,
            len(k["yaw"]), dp(k["xy"]), dp(k["yaw"]), p.L0, p.Th0, p.L1, p.Th1, p.eps,
            dp(k["q0"]), dp(k["q1"]), dp(k["d0"]), dp(k["d1"]), int(p.tau_q), p.start_step,
            int(p.spent_q), p.spent_n)


class ScheduleResult:
    def __init__(self, reuse, chat_q, dbar, s: L.Schedule):
        self.reuse = [int(v) for v in reuse]
        self.chat_q = chat_q
        self.dbar = dbar
        self.n_reuse = int(s.n_reuse)
        self.cost_q = int(s.cost_q)
        self.L, self.Theta, self.zL, self.zTh, self.D = s.L, s.Theta, s.zL, s.zTh, s.D
        self.in_support = bool(s.in_support)


def dc_schedule_dp(p: PySchedProblem) -> ScheduleResult:
    cp = _CProblem(p)
    reuse = np.zeros(p.K, np.uint8)
    nt = max(p.K - 1, 0) * p.h_max
    chat = np.zeros(max(nt, 1), np.int64)
    dbar = np.zeros(max(nt, 1), np.float64)
    out = L.Schedule(reuse.ctypes.data_as(C.POINTER(C.c_uint8)), chat.ctypes.data_as(C.POINTER(C.c_int64)),
                     dbar.ctypes.data_as(C.POINTER(C.c_double)), 0, 0, 0, 0, 0, 0, 0, 0)
    L.check("dc_schedule_dp", L.load().dc_schedule_dp(C.byref(cp.c), C.byref(out)))
    return ScheduleResult(reuse, chat[:nt].reshape(max(p.K - 1, 0), p.h_max),
                          dbar[:nt].reshape(max(p.K - 1, 0), p.h_max), out)


def dc_select_tau(problems, rho: float) -> int:
    cps = [_CProblem(p) for p in problems]
    arr = (L.SchedProblem * len(cps))(*[c.c for c in cps])
    tau = C.c_int64(0)
    L.check("dc_select_tau", L.load().dc_select_tau(arr, len(cps), float(rho), C.byref(tau)))
    return int(tau.value)


def dc_motion_statistics(xy, yaw):
    """Eq. 2 for one pose sequence: (L, Theta)."""
    xy = np.ascontiguousarray(xy, np.float64).reshape(-1, 2)
    yaw = np.ascontiguousarray(yaw, np.float64)
    n = len(yaw)
    Lv, Tv = C.c_double(0.0), C.c_double(0.0)
    dp = C.POINTER(C.c_double)
    L.check("dc_motion_statistics", L.load().dc_motion_statistics(
        xy.ctypes.data_as(dp), yaw.ctypes.data_as(dp), n, C.byref(Lv), C.byref(Tv)))
    return float(Lv.value), float(Tv.value)


def dc_select_anchors(Ls, Ths, eps: float):
    """Sec. 3.1 anchors from calibration clips: ((L0, Th0, L1, Th1), (i0, i1)); i1 = None
    when no clip qualifies (full-inference fallback)."""
    Ls = np.ascontiguousarray(Ls, np.float64)
    Ths = np.ascontiguousarray(Ths, np.float64)
    out = (C.c_double * 4)()
    idx = (C.c_int32 * 2)()
    dp = C.POINTER(C.c_double)
    L.check("dc_select_anchors", L.load().dc_select_anchors(
        Ls.ctypes.data_as(dp), Ths.ctypes.data_as(dp), len(Ls), float(eps), out, idx))
    return tuple(float(v) for v in out), (int(idx[0]), None if idx[1] < 0 else int(idx[1]))


class SamplerBuffers:
    """Caller-owned device buffers for a batch of B scenes (allocated once, reusable).
    branches = 2 (guidance): h_in, h and resid hold 2B entries and the workspace 2B;
    experts = 2: a second modulation table for the low-noise expert; ext: the workspace of
    extended blocks; cache_bits = 8 or 4: resid holds codes, with their scales beside it."""

    def __init__(self, m: ModelShape, B: int, K: int, device="cuda:0", branches=1, experts=1, ext=False,
                 cache_bits=0):
        torch = _torch()
        mdt = torch.bfloat16 if m.dtype == "bf16" else torch.float32
        self.m, self.B, self.K = m, B, K
        E = branches * B
        self.x = torch.empty((B,) + tuple(m.latent_shape), device=device, dtype=torch.float32)
        self.txt = torch.zeros((B, m.n_txt, m.hidden), device=device, dtype=torch.float32)
        self.txt_null = torch.zeros_like(self.txt) if branches == 2 else None
        self.h_in = torch.empty((E, m.n_tok, m.hidden), device=device, dtype=torch.float32)
        self.h = torch.empty_like(self.h_in)
        self.cache_bits, self.ext = cache_bits, ext
        self.cache_scales = None
        if cache_bits:
            if cache_bits not in (8, 4):
                raise ValueError("cache_bits must be 0, 8 or 4")
            self.resid = torch.empty((E, m.n_v, m.hidden * cache_bits // 8), device=device,
                                     dtype=torch.int8 if cache_bits == 8 else torch.uint8)
            self.cache_scales = torch.empty((E, m.n_v, m.hidden // 64), device=device, dtype=torch.float32)
        else:
            self.resid = torch.empty((E, m.n_v, m.hidden), device=device, dtype=mdt)
        self.u_ref = torch.empty((B, m.n_v, m.hidden), device=device, dtype=mdt)
        self.mod = torch.empty((K, m.n_blocks + 1, 6, m.hidden), device=device, dtype=torch.float32)
        self.mod_low = torch.empty_like(self.mod) if experts == 2 else None
        self.sums = torch.zeros((B, 4), device=device, dtype=torch.float64)
        self.ws = Workspace(m, E, device, ext)
        self.c = L.Buffers(_ptr(self.x), _ptr(self.txt), _ptr(self.h_in), _ptr(self.h), _ptr(self.resid),
                           _ptr(self.u_ref), _ptr(self.mod), _ptr(self.sums), self.ws.ptr, self.ws.nbytes)


class Sampler:
    """dc_sampler: the causal controller over caller-owned device buffers.

    x1, txt: initial latents [B, C, T, H, W] and text [B, N_t, d] (torch tensors,
    host or device); they are copied into `bufs` (allocated here if not given)."""

    def __init__(self, dm: DeviceModel, problems, sigmas, x1, txt, drift_metric=0, stream=None,
                 bufs: SamplerBuffers = None, low_expert=None, guidance=None, ext: BlockExt = None,
                 ext_low: BlockExt = None, cache_bits=0):
        """low_expert: (DeviceModel, k_switch), the low-noise expert from step k_switch on
        (every problem's segment must change there); guidance: (w, txt_null [B, N_t, d]),
        guidance branches with separate caches; ext, ext_low: extensions of dm's and of the low
        expert's blocks; cache_bits: 8 or 4 for a quantised residual cache (as bufs were made for)."""
        B = len(problems)
        self.dm, self.B, self.K = dm, B, problems[0].K
        if bufs is None:
            bufs = SamplerBuffers(dm.m, B, self.K, dm.device, branches=2 if guidance else 1,
                                  experts=2 if low_expert else 1, ext=bool(ext or ext_low),
                                  cache_bits=cache_bits)
        self.bufs = bufs
        assert self.bufs.B == B and self.bufs.K == self.K
        if bufs.cache_bits != cache_bits:
            raise ValueError("bufs were made for another cache_bits")
        self.bufs.x.copy_(x1, non_blocking=True)
        if dm.m.n_txt:
            self.bufs.txt.copy_(txt, non_blocking=True)
        self.x = self.bufs.x
        self._cps = [_CProblem(p) for p in problems]
        arr = (L.SchedProblem * B)(*[c.c for c in self._cps])
        sig = np.ascontiguousarray(np.asarray(sigmas, np.float64))
        self._h = C.c_void_p()
        opts = L.SamplerOpts()
        opts.drift_metric = int(drift_metric)
        self._low = None
        if low_expert is not None:
            self._low, k_switch = low_expert
            assert self.bufs.mod_low is not None
            opts.w_low = C.pointer(self._low.cweights)
            opts.k_switch = int(k_switch)
            opts.mod_low = int(self.bufs.mod_low.data_ptr())
        if guidance is not None:
            w, txt_null = guidance
            assert self.bufs.txt_null is not None
            if dm.m.n_txt:
                self.bufs.txt_null.copy_(txt_null, non_blocking=True)
            opts.cfg = 1
            opts.guidance = float(w)
            opts.txt_null = int(self.bufs.txt_null.data_ptr())
        x = L.SamplerExt()
        self._ext = (ext, ext_low)      # the device memory they point to lives as long as the sampler
        if ext is not None:
            x.blocks = ext.of(dm).c
        if ext_low is not None:
            x.blocks_low = ext_low.of(low_expert[0] if low_expert else dm).c
        x.cache_bits = int(cache_bits)
        if cache_bits:
            x.cache_scales = int(self.bufs.cache_scales.data_ptr())
        L.check("dc_sampler_create_ext", L.load().dc_sampler_create_ext(
            C.byref(dm.cfg), C.byref(dm.cweights), B, arr, sig.ctypes.data_as(C.POINTER(C.c_double)),
            C.byref(self.bufs.c), C.byref(opts), C.byref(x), _stream(stream), C.byref(self._h)))
        self.k = 0

    def step(self, stream=None):
        """Run the next denoising step; returns (realized [B] uint8, drift [B] f64)."""
        self.k += 1
        realized = np.zeros(self.B, np.uint8)
        drift = np.zeros(self.B, np.float64)
        L.check("dc_denoise_step", L.load().dc_denoise_step(
            self._h, self.k, _stream(stream), realized.ctypes.data_as(C.POINTER(C.c_uint8)),
            drift.ctypes.data_as(C.POINTER(C.c_double))))
        return realized, drift

    def run(self, stream=None):
        """All K steps; returns (realized [K, B], drift [K, B])."""
        rs, ds = [], []
        for _ in range(self.K):
            r, d = self.step(stream)
            rs.append(r)
            ds.append(d)
        return np.stack(rs), np.stack(ds)

    def plan(self, b=0):
        reuse = np.zeros(self.K, np.uint8)
        nv = C.c_int32(0)
        cq = C.c_int64(0)
        L.check("dc_sampler_plan", L.load().dc_sampler_plan(
            self._h, b, reuse.ctypes.data_as(C.POINTER(C.c_uint8)), C.byref(nv), C.byref(cq)))
        return reuse, int(nv.value), int(cq.value)

    def close(self):
        if self._h:
            L.load().dc_sampler_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class profile:
    """Context manager timing kernel classes with hipEvents (dc_profile_*).

    with api.profile(["attention"]) as p: ...;  p.read() -> {name: (launches, total_ms)}"""

    def __init__(self, classes):
        self.ids = [L.KERNEL_CLASSES.index(c) for c in classes]

    def __enter__(self):
        lib = L.load()
        L.check("dc_profile_reset", lib.dc_profile_reset())
        mask = 0
        for i in self.ids:
            mask |= 1 << i
        L.check("dc_profile_enable", lib.dc_profile_enable(mask))
        return self

    def __exit__(self, *exc):
        L.load().dc_profile_enable(0)
        return False

    def read(self):
        out = {}
        for i in self.ids:
            n = C.c_int64(0)
            ms = C.c_double(0.0)
            L.check("dc_profile_read", L.load().dc_profile_read(i, C.byref(n), C.byref(ms)))
            out[L.KERNEL_CLASSES[i]] = (int(n.value), float(ms.value))
        return out
