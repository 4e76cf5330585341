"""Rotary positions, query/key norms, int8 and e4m3 rows and the quantised cache, from their definitions.

Test infrastructure only (see oracle/__init__.py).  Angles, norms, rotations and sums in float64.  Codes
go by fp32 divisions (a scale is an fp32 number, and x / scale is rounded to fp32 before it is rounded to
an integer), so they are compared for equality."""
from __future__ import annotations

import numpy as np

from . import dit

F = np.float64


def rope_table(positions, dims, theta, pairs):
    """[n, pairs, 2] (cos, sin): pair i of axis a turns by positions[:, a] theta^(-2 i / dims[a])."""
    angle = np.zeros((len(positions), pairs), F)
    at = 0
    for a, d in enumerate(dims):
        for i in range(d // 2):
            angle[:, at] = positions[:, a] * theta ** (-2.0 * i / d)
            at += 1
    return np.stack([np.cos(angle), np.sin(angle)], -1)


def grid_positions(t, h, w, start=(0.0, 0.0, 0.0), step=(1.0, 1.0, 1.0)):
    g = np.stack(np.meshgrid(np.arange(t), np.arange(h), np.arange(w), indexing="ij"), -1).reshape(-1, 3)
    return np.asarray(start, F) + np.asarray(step, F) * g


def qk_norm_rope(x, weight, eps, table, interleaved, scale=1.0):
    """x [N, heads, head_dim] of Q or of K; the first len(table) rows turn."""
    x = np.asarray(x, F)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, F)
    y = x.copy()
    if table is not None:
        n, half = len(table), x.shape[-1] // 2
        first = slice(0, None, 2) if interleaved else slice(0, half)
        second = slice(1, None, 2) if interleaved else slice(half, None)
        c, s = np.asarray(table, F)[:, None, :, 0], np.asarray(table, F)[:, None, :, 1]
        a, b = x[:n, :, first], x[:n, :, second]
        y[:n, :, first] = a * c - b * s
        y[:n, :, second] = b * c + a * s
    return y * scale


def codes(x, levels):
    """(codes, scale) of x along its last axis."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        scale = np.abs(x).max(-1) / np.float32(levels)
        scale = np.where(np.isfinite(x).all(-1), scale, np.float32(np.nan)).astype(np.float32)
        q = np.clip(np.rint(x / scale[..., None]), -levels, levels)
    return np.where(scale[..., None] > 0, q, 0).astype(np.int8), scale


def cache_codes(r, bits):
    """(codes [..., d], scales [..., d / 64]) of a residual."""
    q, s = codes(np.asarray(r, np.float32).reshape(*r.shape[:-1], -1, 64), 127 if bits == 8 else 7)
    return q.reshape(r.shape), s


def cache_values(q, s):
    return (q.reshape(*q.shape[:-1], -1, 64).astype(F) * s[..., None].astype(F)).reshape(q.shape)


def int8_rows(x):
    """The values that int8 rows stand for."""
    q, s = codes(x, 127)
    return q.astype(F) * s[..., None].astype(F)


E4M3_TOP = 448.0


def e4m3(v):
    """The nearest e4m3 number (three fraction bits, exponents from -6 on, at most 448), ties to even."""
    v = np.asarray(v, F)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6))) - 3)
    return np.clip(np.rint(v / step) * step, -E4M3_TOP, E4M3_TOP)


def e4m3_blocks(x, block_rows=1):
    """(numbers that the codes are [R, C padded], scales [blocks of rows, blocks of 128]) of x [R, C]."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    nr, nb = -(-rows // block_rows), -(-cols // 128)
    v = np.zeros((nr * block_rows, nb * 128), np.float32)
    v[:rows, :cols] = x
    v = v.reshape(nr, block_rows, nb, 128)
    with np.errstate(all="ignore"):
        scale = np.abs(v).max((1, 3)) / np.float32(E4M3_TOP)
        scale = np.where(np.isfinite(v).all((1, 3)), scale, np.float32(np.nan)).astype(np.float32)
        step = scale[:, None, :, None]
        q = np.where(step > 0, np.clip(v / step, -E4M3_TOP, E4M3_TOP), np.float32(0))
    return e4m3(q).reshape(nr * block_rows, nb * 128)[:rows], scale


def e4m3_values(q, scale, block_rows=1):
    """What codes with these scales stand for, padding included."""
    s = np.repeat(np.repeat(np.asarray(scale, F), block_rows, 0)[: len(q)], 128, 1)
    return np.asarray(q, F) * s


def rms_norm(h, weight, eps):
    h = np.asarray(h, F)
    y = h / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return y if weight is None else y * np.asarray(weight, F)


def linear_f8(x, x_scale, w, w_scale, bias=None, gelu=False, gate=None, residual=None):
    """dc_linear_f8 on the numbers that codes are, and the sums of its products' magnitudes."""
    a, b = e4m3_values(x, x_scale), e4m3_values(w, w_scale, 128)
    y, size = a @ b.T, np.abs(a) @ np.abs(b).T
    if bias is not None:
        y = y + np.asarray(bias, F)
    if gelu:
        y = dit.gelu_tanh(y)
    if gate is not None:
        y = y * np.asarray(gate, F)
    return (y if residual is None else np.asarray(residual, F) + y), size


def block(P, l, mod6, h, qk=None, int8=False):
    """dit.block with norms and rotation of queries and keys (qk: dict of q_weight, k_weight, eps, table,
    interleaved) and, with int8, every product's operands replaced by what their int8 rows stand for."""
    held = int8_rows if int8 else (lambda a: a)
    m = P.m
    d = m.hidden
    shift1, scale1, gate1, shift2, scale2, gate2 = mod6
    w = {n: held(P.b(l, n)) for n in ("w_qkv", "w_o", "w_1", "w_2")}
    a = held(dit.modulate(h, shift1, scale1, m.ln_eps))
    qkv = a @ w["w_qkv"].T + P.b(l, "b_qkv")
    q, k, v = (qkv[:, i * d: (i + 1) * d] for i in range(3))
    if qk is not None:
        q, k = (qk_norm_rope(x.reshape(len(h), m.heads, -1), qk[n], qk["eps"], qk["table"],
                             qk["interleaved"]).reshape(len(h), d) for x, n in ((q, "q_weight"), (k, "k_weight")))
    o = held(dit.attention(q, k, v, m.heads))
    h = h + gate1 * (o @ w["w_o"].T + P.b(l, "b_o"))
    a = held(dit.modulate(h, shift2, scale2, m.ln_eps))
    z = held(dit.gelu_tanh(a @ w["w_1"].T + P.b(l, "b_1")))
    return h + gate2 * (z @ w["w_2"].T + P.b(l, "b_2"))
