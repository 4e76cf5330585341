"""Rotary table, query/key norms and rotation, int8 rows and products, quantised cache on the GPU,
against the definitions in 64 bits (oracle/ext.py).

Codes and scales are compared for equality.  Elsewhere a rounding is off by at most half a step: relative
2^-24 for fp32 and 2^-8 for bf16."""
import ctypes

import numpy as np
import pytest

from oracle import dit
from oracle import ext as X
from paper_2608_16354_amd import inputs as I
from tests.gpu_util import TILES, _native, compute_units, say, t

pytestmark = pytest.mark.gpu

F32, BF16 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def api():
    from paper_2608_16354_amd import api as A
    A.L.load()
    return A


def shape(heads=4, head_dim=64, lat=(2, 6, 10), n_txt=7, dtype="bf16"):
    d = heads * head_dim
    return I.ModelShape(1, d, heads, head_dim, 4 * d, 16, *lat, 2, n_txt, dtype)


def host(x):
    return x.detach().float().cpu().numpy() if x.is_floating_point() and x.element_size() == 2 else x.cpu().numpy()


# ----------------------------------------------------------------------------
# rotary table
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("lat,head_dim,dims", [
    ((1, 2, 2), 64, (16, 24, 24)), ((13, 60, 90), 64, (16, 24, 24)), ((3, 34, 58), 72, (18, 26, 28)),
    ((4, 6, 10), 64, (0, 32, 30)), ((5, 14, 18), 72, (72, 0, 0)), ((2, 2, 6), 64, (0, 0, 0))])
def test_rope_table(api, dev, lat, head_dim, dims):
    import torch
    m = shape(16 if head_dim == 72 else 4, head_dim, lat)
    n_v, pairs, cfg = m.n_v, head_dim // 2, api.model_cfg(m)
    grid = (lat[0], lat[1] // 2, lat[2] // 2)
    rng = np.random.default_rng(1)
    start, step = (1234.5, -3.0, 0.25), (0.4, 1.0, 0.5)
    given = np.stack([rng.uniform(-1e5, 1e5, n_v), rng.uniform(0, 1e7, n_v), rng.integers(0, 60, n_v)], -1)
    for pos in (None, given):
        table = torch.full((n_v + 1, pairs, 2), 7.0, device=dev)
        say("rope table", lat, head_dim, dims, "given" if pos is not None else "grid")
        api.dc_rope_table(cfg, api.rope_axes(dims, 10000.0, start, step), None if pos is None else t(pos, dev), table[:n_v])
        torch.cuda.synchronize()
        at = X.grid_positions(*grid, start, step) if pos is None else pos
        want = X.rope_table(at, dims, 10000.0, pairs)
        # half a step of a value up to 1, and the angle's error in double: a frequency off by a few 2^-53
        # (its exponent, up to 9.3, carries 2^-53 of itself) moves the angle by up to 30 2^-53 of itself
        tol = F32 + 30 * 2.0 ** -53 * np.abs(at).max()
        assert np.abs(host(table[:n_v]) - want).max() <= tol
        assert (host(table[n_v]) == 7.0).all()


# ----------------------------------------------------------------------------
# norms and rotation
# ----------------------------------------------------------------------------
QK = {
    "bf16-64": shape(30, 64, (2, 34, 58), 77), "bf16-64-one-token": shape(4, 64, (1, 2, 2), 0), "bf16-72": shape(16, 72, (2, 6, 10), 7),
    "bf16-72-odd-heads": shape(16, 72, (3, 14, 18), 21), "bf16-64-wide": shape(48, 64, (1, 10, 10), 3),
    "f32": shape(4, 64, (4, 16, 16), 16, "f32"), "f32-6": shape(6, 64, (1, 6, 10), 1, "f32"), "bf16-2-heads": shape(2, 64, (5, 2, 2), 1),
    "bf16-72-long": shape(16, 72, (4, 32, 56), 21), "f32-long": shape(16, 64, (2, 32, 56), 9, "f32"),
}


def qk_tolerance(x, weight, eps, table, interleaved, scale, bf16):
    """Per value: fp32's roundings on the two products that are added, and the output's.  With a mean square
    of at most 72 terms added in a tree (7 roundings and one each of the square, the mean, eps, the root and
    the quotient: 12), the weights' products (3), the two terms and their sum (3): under 24 roundings of
    |A x| + |B x'|."""
    y = np.abs(X.qk_norm_rope(np.abs(x), None if weight is None else np.abs(weight), eps, None, interleaved, abs(scale)))
    both = y.copy()
    if table is not None:
        n, half = len(table), x.shape[-1] // 2
        a, b = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, half), slice(half, None))
        both[:n, :, a] = both[:n, :, b] = y[:n, :, a] + y[:n, :, b]
    return 24 * F32 * both, (BF16 if bf16 else F32)


@pytest.mark.parametrize("name", list(QK))
@pytest.mark.parametrize("interleaved", [True, False])
def test_qk_norm_rope(api, dev, name, interleaved):
    import torch
    m = QK[name]
    bf, d, N, cfg = m.dtype == "bf16", m.hidden, m.n_tok, api.model_cfg(m)
    dt = torch.bfloat16 if bf else torch.float32
    rng = np.random.default_rng(2)
    x = rng.standard_normal((3, N, 3 * d)).astype(np.float32)
    x[0, 0, : m.head_dim] = 0                       # a head of zeros
    x[2, N - 1] *= 1e-4                             # values about the size of eps
    x[2, 0] *= 1e15
    x = I.round_bf16(x) if bf else x
    wq, wk = (1 + 0.2 * rng.standard_normal((2, m.head_dim))).astype(np.float32)
    table = X.rope_table(rng.uniform(-50, 50, (m.n_v, 3)), (m.head_dim // 2, m.head_dim // 4 * 2 - m.head_dim // 2, 0), 100.0,
                         m.head_dim // 2).astype(np.float32)
    for norm_q, norm_k, turn, ld in ((1, 1, 1, 3 * d), (1, 1, 1, 2 * d), (0, 0, 1, 2 * d), (1, 1, 0, 3 * d), (0, 1, 1, 3 * d),
                                     (1, 0, 0, 2 * d), (0, 0, 0, 2 * d)):
        dx = t(x, dev, dt)
        buf = torch.full((3, N, ld + 16), 5.0, device=dev, dtype=dt)
        out = buf[:, :, :ld]
        say("qk", name, interleaved, norm_q, norm_k, turn, ld)
        kw = dict(q_weight=t(wq, dev) if norm_q else None, k_weight=t(wk, dev) if norm_k else None, eps=1e-6,
                  table=t(table, dev) if turn else None, interleaved=interleaved, q_scale=0.125)
        api.dc_qk_norm_rope(cfg, dx, out, [2, 0], **kw)
        inplace = dx.clone()
        api.dc_qk_norm_rope(cfg, inplace, inplace, [2, 0], **kw)
        torch.cuda.synchronize()
        got, still = host(buf), host(inplace)
        assert (got[1] == 5).all() and (got[:, :, 2 * d:] == 5).all()       # other samples, other columns
        assert np.array_equal(still[[0, 2], :, : 2 * d], got[[0, 2], :, : 2 * d])
        assert np.array_equal(still[1], x[1]) and np.array_equal(still[:, :, 2 * d:], x[:, :, 2 * d:])
        for b in (0, 2):
            for part, w, sc in ((0, wq if norm_q else None, 0.125), (1, wk if norm_k else None, 1.0)):
                rows = x[b, :, part * d: (part + 1) * d].reshape(N, m.heads, m.head_dim).astype(np.float64)
                want = X.qk_norm_rope(rows, w, 1e-6, table if turn else None, interleaved, sc)
                tol, rel = qk_tolerance(rows, w, 1e-6, table if turn else None, interleaved, sc, bf)
                err = np.abs(got[b, :, part * d: (part + 1) * d].reshape(want.shape) - want)
                assert (err <= tol + rel * (np.abs(want) + tol) + 2.0 ** -133).all(), (b, part, err.max())


def test_qk_text_rows_keep_what_a_pair_would_spread(api, dev):
    """A text row is not turned: an infinity there stays in its own feature (without norms)."""
    import torch
    m = shape(2, 64, (1, 2, 2), 3)
    x = torch.ones((1, m.n_tok, 2 * m.hidden), device=dev, dtype=torch.bfloat16)
    x[0, 2, 5] = float("inf")
    x[0, 3, 6] = float("nan")
    table = torch.zeros((m.n_v, 32, 2), device=dev)
    table[..., 0] = 1
    out = torch.empty_like(x)
    api.dc_qk_norm_rope(api.model_cfg(m), x, out, [0], table=table)
    assert np.array_equal(host(out), host(x), equal_nan=True)


# ----------------------------------------------------------------------------
# int8 rows
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1, 3, 7, 8, 9, 64, 127, 128, 129, 513, 1000, 1920, 2049, 4097, 7680, 8192, 8193, 16391, 70001])
def test_quantize_rows(api, dev, dtype, cols):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(cols)
    rows, pad = 11, -(-cols // 128) * 128
    x = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32)
    x[1] = 0
    x[2, cols // 2] = np.inf
    x[3, cols - 1] = np.nan
    x[4] *= np.float32(1e-38)
    x[5] = np.float32(2e-44) * rng.integers(-1, 2, cols)        # a / 127 leaves fp32's range
    x[6] = 3.38e38 * np.sign(x[6])
    x[7] = -0.0
    x[8, 0] = -np.inf
    x = I.round_bf16(x) if dtype == "bf16" else x
    with np.errstate(invalid="ignore"):
        x[3, cols - 1] = np.nan
    want_q, want_s = X.codes(x, 127)
    for lead, extra in ((0, 0), (1, 5)):                        # rows at every element's address, wider strides
        xb = torch.zeros((rows, cols + lead + extra), device=dev, dtype=dt)
        xb[:, lead: lead + cols] = t(x, dev, dt)
        qb = torch.full((rows + 1, pad + 128), 99, device=dev, dtype=torch.int8)
        s = torch.full((rows + 1,), 99.0, device=dev)
        say("quantize", dtype, cols, lead)
        api.dc_quantize_rows(xb[:, lead: lead + cols], qb[:rows, : pad + (128 if extra else 0)], s[:rows])
        torch.cuda.synchronize()
        q, s = host(qb), host(s)
        assert np.array_equal(s[:rows], want_s, equal_nan=True) and s[rows] == 99
        assert np.array_equal(q[:rows, :cols], want_q)
        assert (q[:rows, cols:pad] == 0).all() and (q[:rows, pad:] == 99).all() and (q[rows] == 99).all()


@pytest.mark.parametrize("dtype,rows,cols", [("f32", 1, 1920), ("bf16", 1, 7680), ("bf16", 4099, 1152), ("f32", 1025, 333),
                                             ("bf16", 4099, 1920), ("f32", 4099, 1000), ("bf16", 1000, 7687), ("f32", 3301, 1501),
                                             ("bf16", 12301, 500), ("f32", 9001, 130), ("bf16", 7, 130943), ("f32", 100003, 3),
                                             ("bf16", 100003, 5)])
def test_quantize_many_rows(api, dev, dtype, rows, cols):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn((rows, cols), device=dev, generator=torch.Generator(dev).manual_seed(5)).to(dt)
    q = torch.empty((rows, -(-cols // 128) * 128), device=dev, dtype=torch.int8)
    s = torch.empty(rows, device=dev)
    api.dc_quantize_rows(x, q, s)
    want_q, want_s = X.codes(host(x), 127)
    assert np.array_equal(host(s), want_s) and np.array_equal(host(q)[:, :cols], want_q)


# ----------------------------------------------------------------------------
# int8 products
# ----------------------------------------------------------------------------
def linear_inputs(m, n, k, seed, full=False):
    rng = np.random.default_rng(seed)
    x, w = (rng.integers(-127, 128, (r, k)).astype(np.int8) for r in (m, n))
    if full:
        x[0], w[0] = -128, -128                     # the largest sum there is
        x[-1] = 127
    return (x, rng.uniform(0.001, 0.02, m).astype(np.float32), w, rng.uniform(1e-5, 3e-4, n).astype(np.float32),
            rng.standard_normal(n).astype(np.float32), rng.standard_normal(n).astype(np.float32),
            rng.standard_normal((m, n)).astype(np.float32))


def check_linear(got, x, xs, w, ws, bias, gate, residual, kind, bf16):
    """v = sum x w (exact), fp32: one rounding to fp32, two scales, the bias: 4 roundings of |v| + |bias|.
    GELU: its slope is at most 1.13; y has 4 roundings and a further one as the exponent's argument, exp(-2y) carries
    2|y| times those and 2 steps of its own (__expf: the argument's product with log2 e too, 2 more), the sum and
    the quotient 3 more, and |z sigmoid(2y)| times (2|y| 7 + 7) roundings covers them; |y| <= 40 matters (beyond it the
    value is z or 0).  Residual: 2 more roundings of |gate v| + |residual|."""
    acc = np.rint(x.astype(np.float64) @ w.astype(np.float64).T)
    v = acc * xs[:, None].astype(np.float64) * ws.astype(np.float64)
    tol = 4 * F32 * (np.abs(v) + (0 if bias is None else np.abs(bias)))
    if bias is not None:
        v = v + bias
    if kind == "gelu":
        y = np.minimum(np.abs(0.7978845608 * (v + 0.044715 * v ** 3)), 40)
        z = dit.gelu_tanh(v)
        tol = 1.13 * tol + (14 * y + 7) * F32 * np.abs(z) + 2.0 ** -120
        v = z
    elif kind == "gated":
        tol = np.abs(gate) * tol + 2 * F32 * (np.abs(gate * v) + np.abs(residual))
        v = residual + gate * v
    tol = tol + (BF16 if bf16 else F32) * (np.abs(v) + tol)
    err = np.abs(got - v)
    assert np.isfinite(got).all() and (err <= tol).all(), (err.max(), (err / tol).max(), np.argwhere(err > tol)[:4])


TILE_SHAPES = {     # (M, N, K): the tile on 256 compute units
    (2562, 5760, 1920): "384x192", (1155, 11520, 1920): "320x256", (1155, 7680, 3840): "256x192",
    (1144, 5760, 1920): "256x128", (1155, 1920, 3840): "128x128", (513, 1920, 256): "64x64", (1537, 3456, 2304): "192x128",
    (801, 1920, 7680): "128x64",
    (67, 1153, 1408): "32x32 x 4", (33, 1153, 7680): "32x32 x 5",
}
I8_TILES = TILES + ("192x128", "128x64", "32x32 x 4", "32x32 x 5")


def i8_tile(m, n, k, cus):
    return I8_TILES[_native("_ZN2dc7i8_tileEiiiib", m, n, k // 128, cus, True)]


@pytest.mark.parametrize("mnk", list(TILE_SHAPES))
@pytest.mark.parametrize("kind", ["plain", "gelu", "gated"])
def test_linear_tiles(api, dev, mnk, kind):
    """Every tile of the product, ragged in rows; fp32 outputs, and bf16 ones where there are any."""
    import torch
    m, n, k = mnk
    assert i8_tile(m, n, k, compute_units(dev)) == TILE_SHAPES[mnk]
    x, xs, w, ws, bias, gate, res = linear_inputs(m, n, k, 7)
    dx, dw, dxs, dws, db = t(x, dev), t(w, dev), t(xs, dev), t(ws, dev), t(bias, dev)
    for dt in (torch.float32, torch.bfloat16):
        if kind == "gated" and dt == torch.bfloat16:
            continue
        out = torch.full((m + 1, n), 3.0, device=dev, dtype=dt)
        say("linear tile", mnk, TILE_SHAPES[mnk], kind, dt)
        api.dc_linear_i8(dx, dxs, dw, dws, out[:m], bias=db, gelu=kind == "gelu", gate=t(gate, dev) if kind == "gated" else None,
                         residual=t(res, dev) if kind == "gated" else None)
        torch.cuda.synchronize()
        got = host(out)
        assert (got[m] == 3).all()
        pick = np.unique(np.r_[0, m - 1, np.random.default_rng(0).integers(0, m, 200)])
        check_linear(got[pick], x[pick], xs[pick], w, ws, bias, gate, res[pick], kind, dt == torch.bfloat16)


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 191, 300])
@pytest.mark.parametrize("n,k", [(1, 128), (31, 256), (33, 384), (64, 128), (65, 1920), (193, 512), (250, 7680), (1152, 640)])
def test_linear_ragged(api, dev, m, n, k):
    """Few rows and odd widths, each epilogue, with and without a bias, strided operands and outputs."""
    import torch
    x, xs, w, ws, bias, gate, res = linear_inputs(m, n, k, m + n, full=k == 1920)
    dxs, dws = t(xs, dev), t(ws, dev)
    pad = [torch.full((r, k + 48), 77, device=dev, dtype=torch.int8) for r in (m, n)]
    dx, dw = pad[0][:, 16: 16 + k], pad[1][:, 32: 32 + k]
    dx.copy_(t(x, dev))
    dw.copy_(t(w, dev))
    say("linear ragged", m, n, k)
    for kind, dt, ld, lead, has_bias in (("plain", "f32", n, 0, True), ("plain", "bf16", n + 3, 1, False), ("gelu", "bf16", n + 8, 8, True),
                                         ("gelu", "f32", n + 1, 0, False), ("gated", "f32", n + 5, 1, True), ("gated", "f32", n, 0, False)):
        buf = torch.full((m + 1, ld + lead), 3.0, device=dev, dtype=torch.float32 if dt == "f32" else torch.bfloat16)
        out = buf[:m, lead: lead + n]
        rs = None
        if kind == "gated":
            out.copy_(t(res, dev))
            rs = out if has_bias else t(res, dev)           # in place, and from another tensor
        api.dc_linear_i8(dx, dxs, dw, dws, out, bias=t(bias, dev) if has_bias else None, gelu=kind == "gelu",
                         gate=t(gate, dev) if kind == "gated" else None, residual=rs)
        torch.cuda.synchronize()
        got = host(buf)
        check_linear(got[:m, lead: lead + n], x, xs, w, ws, bias if has_bias else None, gate, res, kind, dt == "bf16")
        assert (got[m] == 3).all() and (got[:, :lead] == 3).all() and (got[:, lead + n:] == 3).all()


def test_linear_longest_sum(api, dev):
    """K = 130,944 of the largest codes: the sum is just below 2^31."""
    import torch
    k = 130944
    x, w = (torch.full((3, k), -128, dtype=torch.int8, device=dev) for _ in range(2))
    x[1] = 127
    x[2, ::2] = 1
    out = torch.empty((3, 3), device=dev)
    one = torch.ones(3, device=dev)
    api.dc_linear_i8(x, one, w, one, out)
    want = x.cpu().numpy().astype(np.int64) @ w.cpu().numpy().astype(np.int64).T
    assert want[0, 0] == 2 ** 31 - 2 ** 21
    assert np.array_equal(host(out), want.astype(np.float32))


def test_linear_rows_beyond_32_bit_offsets(api, dev):
    """Rows 4 MiB apart: the last ones lie past 2^31 bytes, in x and in w."""
    import torch
    x, xs, w, ws, bias, gate, res = linear_inputs(700, 600, 256, 3)
    big = [torch.empty((r, 1 << 22), dtype=torch.int8, device=dev)[:, :256] for r in (700, 600)]
    big[0].copy_(t(x, dev))
    big[1].copy_(t(w, dev))
    out = torch.empty((700, 600), device=dev)
    api.dc_linear_i8(big[0], t(xs, dev), big[1], t(ws, dev), out)
    check_linear(host(out), x, xs, w, ws, None, gate, res, "plain", False)


def test_linear_of_a_row_without_a_number(api, dev):
    """A row that held a NaN or an infinity is NaN in the product, the others are not."""
    import torch
    x = torch.randn((70, 200), device=dev, generator=torch.Generator(dev).manual_seed(1))
    x[3, 7], x[66, 199] = float("nan"), float("inf")
    q, s = torch.empty((70, 256), dtype=torch.int8, device=dev), torch.empty(70, device=dev)
    w = torch.ones((40, 256), dtype=torch.int8, device=dev)
    out = torch.empty((70, 40), device=dev)
    api.dc_quantize_rows(x, q, s)
    api.dc_linear_i8(q, s, w, torch.ones(40, device=dev), out)
    bad = np.isnan(host(out))
    assert bad[[3, 66]].all() and bad.sum() == 80


def test_one_row_of_any_stride(api, dev):
    """A single row's stride says nothing: rows cut out of wider ones are taken as they are."""
    import torch
    wide = torch.randn((1, 203), device=dev, generator=torch.Generator(dev).manual_seed(2))
    q, s, y = torch.zeros((1, 333), dtype=torch.int8, device=dev), torch.zeros(1, device=dev), torch.zeros((1, 41), device=dev)
    x, row, out = (v.as_strided(v[:, :n].shape, (st, 1)) for v, n, st in ((wide, 200, 7), (q, 256, 3), (y, 40, 1)))
    w = torch.randint(-127, 128, (40, 256), dtype=torch.int8, device=dev)
    api.dc_quantize_rows(x, row, s)
    api.dc_linear_i8(row, s, w, torch.ones(40, device=dev), out)
    codes, scale = X.codes(host(wide)[:, :200], 127)
    assert np.array_equal(host(row)[:, :200], codes) and np.array_equal(host(s), scale) and not host(q)[:, 200:256].any()
    want = (codes.astype(np.int64) @ host(w)[:, :200].astype(np.int64).T) * scale.astype(np.float64)
    assert (np.abs(host(out) - want) <= 4 * F32 * np.abs(want)).all() and host(y)[0, 40] == 0


@pytest.mark.parametrize("batch", [1, 3])
def test_single_tokens_of_any_stride(api, dev, batch):
    """A model of one token, its samples cut out of longer ones: against the same rows put together."""
    import torch
    m = shape(lat=(1, 2, 2), n_txt=0)
    cfg, d2, idx = api.model_cfg(m), 2 * m.hidden, list(range(batch))
    wide = torch.randn((batch, 5, 3 * m.hidden), device=dev, generator=torch.Generator(dev).manual_seed(8)).bfloat16()
    w, table = torch.full((64,), 1.5, device=dev), torch.randn((1, 32, 2), device=dev)
    want = torch.zeros((batch, 1, d2), device=dev, dtype=torch.bfloat16)
    whole = wide[:, 2:3].contiguous()
    api.dc_qk_norm_rope(cfg, whole, want, idx, q_weight=w, k_weight=w, table=table)
    x = wide.as_strided((batch, 1, 3 * m.hidden), (5 * 3 * m.hidden, 3, 1), 2 * 3 * m.hidden)
    held = torch.full((batch, 2, d2 + 8), 4.0, device=dev, dtype=torch.bfloat16)
    api.dc_qk_norm_rope(cfg, x, held.as_strided((batch, 1, d2), (2 * (d2 + 8), 5, 1)), idx, q_weight=w, k_weight=w, table=table)
    assert torch.equal(held[:, :1, :d2], want) and (held[:, 1] == 4).all() and (held[:, 0, d2:] == 4).all()
    assert want.float().abs().max() > 0.5


def test_linear_of_no_rows(api, dev):
    import torch
    api.dc_quantize_rows(torch.empty((0, 100), device=dev), torch.empty((0, 128), dtype=torch.int8, device=dev), torch.empty(0, device=dev))
    api.dc_linear_i8(torch.empty((0, 128), dtype=torch.int8, device=dev), torch.empty(0, device=dev),
                     torch.ones((40, 128), dtype=torch.int8, device=dev), torch.ones(40, device=dev), torch.empty((0, 40), device=dev))


# ----------------------------------------------------------------------------
# quantised cache
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("name", ["f32", "bf16-64-one-token", "bf16-72", "bf16-64"])
def test_cache(api, dev, bits, name):
    import torch
    m = QK[name]
    d, N, n_v, cfg = m.hidden, m.n_tok, m.n_v, api.model_cfg(m)
    rng = np.random.default_rng(9)
    h_in = (0.2 * rng.standard_normal((3, N, d))).astype(np.float32)
    h_out = (h_in + rng.standard_normal((3, N, d)) * np.exp(rng.standard_normal(d))).astype(np.float32)
    h_out[2, 0, :64] = h_in[2, 0, :64]              # a group of zeros
    h_out[2, n_v - 1, 70] = np.inf
    h_out[0, n_v - 1, 3] = np.nan
    h_in[0, 0, 64:128], h_out[0, 0, 64:128] = 0, 2e-44
    g0 = np.full((3, N, d), 6.0, np.float32)
    codes = torch.full((3, n_v, d * bits // 8), 9, device=dev, dtype=torch.int8 if bits == 8 else torch.uint8)
    scales = torch.full((3, n_v, d // 64), 9.0, device=dev)
    g = t(g0, dev)
    say("cache", name, bits)
    api.dc_cache_store_q(cfg, bits, t(h_out, dev), t(h_in, dev), codes, scales, [2, 0])
    api.dc_cache_apply_q(cfg, bits, t(h_in, dev), codes, scales, g, [0, 2])
    again = t(h_in, dev)
    api.dc_cache_apply_q(cfg, bits, again, codes, scales, again, [0, 2])        # in place
    torch.cuda.synchronize()
    got, c, s, again = host(g), host(codes), host(scales), host(again)
    assert (c[1] == 9).all() and (s[1] == 9).all() and (got[1] == 6).all() and (got[:, n_v:] == 6).all()
    assert np.array_equal(again[1], h_in[1]) and np.array_equal(again[:, n_v:], h_in[:, n_v:])
    if bits == 4:
        low, high = (c.astype(np.int8) << 4) >> 4, c.view(np.int8) >> 4
        c = np.stack([low, high], -1).reshape(3, n_v, d)
    for b in (0, 2):
        with np.errstate(invalid="ignore"):
            want_c, want_s = X.cache_codes(h_out[b, :n_v] - h_in[b, :n_v], bits)
        assert np.array_equal(s[b], want_s, equal_nan=True) and np.array_equal(c[b], want_c)
        r = X.cache_values(want_c, want_s)
        want = h_in[b, :n_v] + r
        # the product and the sum round once each at most
        tol = F32 * (np.abs(r) + np.abs(want)) * (1 + F32)
        assert np.array_equal(np.isnan(got[b, :n_v]), np.isnan(want)) and np.isnan(want).any() == (d > 64)
        ok = ~np.isnan(want)
        assert (np.abs(got[b, :n_v] - want)[ok] <= tol[ok]).all()
        assert np.array_equal(again[b, :n_v], got[b, :n_v], equal_nan=True)


# ----------------------------------------------------------------------------
# graphs and streams
# ----------------------------------------------------------------------------
def test_captured_and_replayed(api, dev):
    """All of the calls in one graph on a stream of their own, replayed on changing inputs between eager work,
    against the eager calls."""
    import torch
    m = shape(4, 64, (4, 16, 16), 16)
    d, N, n_v, cfg = m.hidden, m.n_tok, m.n_v, api.model_cfg(m)
    gen = torch.Generator(dev).manual_seed(3)
    x = torch.empty((1, N, 3 * d), device=dev, dtype=torch.bfloat16)
    h_in, h_out = (torch.empty((1, N, d), device=dev) for _ in range(2))
    w = torch.randint(-127, 128, (d, 2 * d), device=dev, generator=gen, dtype=torch.int8)
    ws, wq = torch.rand(d, device=dev, generator=gen), 1 + torch.rand(64, device=dev, generator=gen)
    axes = api.rope_axes((16, 24, 24))

    def buffers():
        return dict(table=torch.zeros((n_v, 32, 2), device=dev), qk=torch.zeros((1, N, 2 * d), device=dev, dtype=torch.bfloat16),
                    q=torch.zeros((N, 2 * d), device=dev, dtype=torch.int8), s=torch.zeros(N, device=dev),
                    y=torch.zeros((N, d), device=dev), codes=torch.zeros((1, n_v, d // 2), device=dev, dtype=torch.uint8),
                    scales=torch.zeros((1, n_v, d // 64), device=dev), g=torch.zeros((1, N, d), device=dev))

    def calls(b):
        api.dc_rope_table(cfg, axes, None, b["table"])
        api.dc_qk_norm_rope(cfg, x, b["qk"], [0], q_weight=wq, k_weight=wq, table=b["table"])
        api.dc_quantize_rows(b["qk"][0], b["q"], b["s"])
        api.dc_linear_i8(b["q"], b["s"], w, ws, b["y"], gate=ws, residual=h_in[0])
        api.dc_cache_store_q(cfg, 4, h_out, h_in, b["codes"], b["scales"], [0])
        api.dc_cache_apply_q(cfg, 4, b["y"][None], b["codes"], b["scales"], b["g"], [0])

    def fill():
        x.copy_(torch.randn(x.shape, device=dev, generator=gen))
        h_in.copy_(torch.randn(h_in.shape, device=dev, generator=gen))
        h_out.copy_(torch.randn(h_in.shape, device=dev, generator=gen))

    graphed, eager = buffers(), buffers()
    fill()
    calls(eager)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        calls(graphed)
    for i in range(4):
        fill()
        graph.replay()
        calls(eager)
        torch.cuda.synchronize()
        for n in graphed:
            assert torch.equal(graphed[n], eager[n]), (i, n)
    # on another stream than the current one
    side = torch.cuda.Stream()
    other = torch.zeros_like(eager["table"])
    side.wait_stream(torch.cuda.current_stream())
    api.dc_rope_table(cfg, axes, None, other, stream=side)
    side.synchronize()
    assert torch.equal(other, eager["table"])


def test_two_streams_at_once(api, dev):
    """The calls keep nothing between them: two streams that work side by side get what each gets alone."""
    import torch
    m = shape(10, 64, (3, 34, 58), 78)
    d, N, n_v, cfg = m.hidden, m.n_tok, m.n_v, api.model_cfg(m)

    def state(seed):
        gen = torch.Generator(dev).manual_seed(seed)
        return dict(x=torch.randn((1, N, 3 * d), device=dev, generator=gen).bfloat16(), table=torch.zeros((n_v, 32, 2), device=dev),
                    q=torch.zeros((N, 3 * d), device=dev, dtype=torch.int8), s=torch.zeros(N, device=dev),
                    w=torch.randint(-127, 128, (d, 3 * d), device=dev, generator=gen, dtype=torch.int8),
                    ws=torch.rand(d, device=dev, generator=gen), y=torch.zeros((1, N, d), device=dev),
                    few=torch.zeros((5, d), device=dev), h=torch.randn((1, N, d), device=dev, generator=gen),
                    codes=torch.zeros((1, n_v, d), device=dev, dtype=torch.int8), scales=torch.zeros((1, n_v, d // 64), device=dev))

    def calls(b, stream, theta):
        api.dc_rope_table(cfg, api.rope_axes((16, 24, 24), theta), None, b["table"], stream=stream)
        api.dc_qk_norm_rope(cfg, b["x"], b["x"], [0], table=b["table"], stream=stream)
        api.dc_quantize_rows(b["x"][0], b["q"], b["s"], stream=stream)
        api.dc_linear_i8(b["q"], b["s"], b["w"], b["ws"], b["y"][0], stream=stream)
        api.dc_linear_i8(b["q"][:5], b["s"][:5], b["w"], b["ws"], b["few"], stream=stream)
        api.dc_cache_store_q(cfg, 8, b["y"], b["h"], b["codes"], b["scales"], [0], stream=stream)
        api.dc_cache_apply_q(cfg, 8, b["h"], b["codes"], b["scales"], b["h"], [0], stream=stream)

    alone, together = [state(i) for i in range(2)], [state(i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(2):
        calls(alone[i], streams[0], 100.0 * (i + 1))
        torch.cuda.synchronize()
    for i in range(2):
        calls(together[i], streams[i], 100.0 * (i + 1))
    torch.cuda.synchronize()
    for a, b in zip(alone, together):
        for n in a:
            assert torch.equal(a[n], b[n]), n
    assert torch.equal(alone[0]["few"], alone[0]["y"][0, :5])


# ----------------------------------------------------------------------------
# offsets beyond 32 bits
# ----------------------------------------------------------------------------
def test_last_sample_of_a_long_batch(api, dev):
    """Samples past 2^32 bytes of a batch get what they get alone."""
    import torch
    m = shape(30, 64, (13, 60, 90), 226)
    d, N, n_v, cfg, B = m.hidden, m.n_tok, m.n_v, api.model_cfg(m), 34
    gen = torch.Generator(dev).manual_seed(6)
    h = [torch.empty((B, N, d), device=dev) for _ in range(2)]
    one = [torch.randn((1, N, d), device=dev, generator=gen) for _ in range(2)]
    assert (B - 1) * N * d * 4 > 2 ** 32
    for a, b in zip(h, one):
        a[B - 1:].copy_(b)
    for bits, dt in ((8, torch.int8), (4, torch.uint8)):
        def cache(n):
            return (torch.zeros((n, n_v, d * bits // 8), device=dev, dtype=dt), torch.zeros((n, n_v, d // 64), device=dev))
        (k, s), (k1, s1) = cache(B), cache(1)
        say("long batch", bits)
        api.dc_cache_store_q(cfg, bits, h[0], h[1], k, s, [B - 1])
        api.dc_cache_store_q(cfg, bits, one[0], one[1], k1, s1, [0])
        assert torch.equal(k[B - 1:], k1) and torch.equal(s[B - 1:], s1) and not k[: B - 1].any()
        g1 = one[1].clone()
        api.dc_cache_apply_q(cfg, bits, h[1], k, s, h[1], [B - 1])
        api.dc_cache_apply_q(cfg, bits, one[1], k1, s1, g1, [0])
        assert torch.equal(h[1][B - 1:], g1)
        h[1][B - 1:].copy_(one[1])
    del h
    x = torch.empty((B, N, 3 * d), device=dev, dtype=torch.bfloat16)
    x1 = torch.randn((1, N, 3 * d), device=dev, generator=gen).bfloat16()
    x[B - 1:].copy_(x1)
    table = torch.randn((n_v, 32, 2), device=dev, generator=gen)
    api.dc_qk_norm_rope(cfg, x, x, [B - 1], table=table)
    api.dc_qk_norm_rope(cfg, x1, x1, [0], table=table)
    assert torch.equal(x[B - 1:], x1)


def test_rows_beyond_32_bit_offsets(api, dev):
    import torch
    rows, cols, apart = 700, 384, (1 << 22) + 8
    x1 = torch.randn((rows, cols), device=dev, generator=torch.Generator(dev).manual_seed(7)).bfloat16()
    x = torch.empty((rows, apart), device=dev, dtype=torch.bfloat16)[:, :cols]
    q = torch.empty((rows, apart), device=dev, dtype=torch.int8)[:, :cols]
    q1, s, s1 = torch.empty((rows, cols), device=dev, dtype=torch.int8), torch.empty(rows, device=dev), torch.empty(rows, device=dev)
    x.copy_(x1)
    api.dc_quantize_rows(x, q, s)
    api.dc_quantize_rows(x1, q1, s1)
    assert torch.equal(q, q1) and torch.equal(s, s1)


def test_long_table(api, dev):
    """31 million tokens: eight billion bytes of table, the last token's angles and the first's."""
    import torch
    m = I.ModelShape(1, 256, 4, 64, 1024, 16, 30, 2048, 2048, 2, 0, "bf16")
    table = torch.empty((m.n_v, 32, 2), device=dev)
    api.dc_rope_table(api.model_cfg(m), api.rope_axes((16, 24, 24), 100.0), None, table)
    at = [0, 1, 1024, 1 << 20, m.n_v // 2 + 517, m.n_v - 1]
    pos = np.array([[n >> 20, (n >> 10) & 1023, n & 1023] for n in at], np.float64)
    want = X.rope_table(pos, (16, 24, 24), 100.0, 32)
    assert np.abs(host(table[at]) - want).max() <= F32 + 1e-10


def test_every_sample_of_the_largest_batch(api, dev):
    """64 samples, 49 of them asked for in no order: those get what they get alone, the others stay."""
    import torch
    m = shape(2, 64, (1, 4, 6), 3)
    d, N, n_v, cfg = m.hidden, m.n_tok, m.n_v, api.model_cfg(m)
    gen = torch.Generator(dev).manual_seed(8)
    idx = [b for b in np.random.default_rng(9).permutation(64).tolist() if b % 4 or b == 0]
    rest = [b for b in range(64) if b not in idx]
    a, b = (torch.randn((64, N, d), device=dev, generator=gen) for _ in range(2))
    k, s = torch.full((64, n_v, d), 99, device=dev, dtype=torch.int8), torch.full((64, n_v, d // 64), 99.0, device=dev)
    g = torch.full((64, N, d), 99.0, device=dev)
    api.dc_cache_store_q(cfg, 8, a, b, k, s, idx)
    api.dc_cache_apply_q(cfg, 8, b, k, s, g, idx)
    x = torch.randn((64, N, 2 * d), device=dev, generator=gen).bfloat16()
    y = torch.full_like(x, 99.0)
    table = torch.randn((n_v, 32, 2), device=dev, generator=gen)
    api.dc_qk_norm_rope(cfg, x, y, idx, table=table)
    assert (k[rest] == 99).all() and (s[rest] == 99).all() and (g[rest] == 99).all() and (y[rest] == 99).all()
    for i in idx:
        k1, s1, g1, y1 = torch.zeros_like(k[:1]), torch.zeros_like(s[:1]), torch.full_like(g[:1], 99.0), torch.zeros_like(y[:1])
        api.dc_cache_store_q(cfg, 8, a[i: i + 1], b[i: i + 1], k1, s1, [0])
        api.dc_cache_apply_q(cfg, 8, b[i: i + 1], k1, s1, g1, [0])
        api.dc_qk_norm_rope(cfg, x[i: i + 1], y1, [0], table=table)
        assert torch.equal(k[i], k1[0]) and torch.equal(s[i], s1[0]) and torch.equal(g[i], g1[0]) and torch.equal(y[i], y1[0])
