"""e4m3 rows and weights, the RMS norm of a sum into such rows, and their products on the GPU, against the
definitions in 64 bits (oracle/ext.py).

Codes and scales of given values are compared for equality.  Elsewhere a rounding is off by at most half a step: relative
2^-24 for fp32, 2^-8 for bf16, 2^-4 for e4m3 (2^-10 below its normal numbers)."""
import numpy as np
import pytest

from oracle import dit
from oracle import ext as X
from paper_2608_16354_amd import inputs as I
from tests.gpu_util import _native, compute_units, say, t

pytestmark = pytest.mark.gpu

F32, BF16, E4M3, E4M3_LOW = 2.0 ** -24, 2.0 ** -8, 2.0 ** -4, 2.0 ** -10
MARK = 99                               # a byte that no call writes there


@pytest.fixture(scope="module")
def api():
    from paper_2608_16354_amd import api as A
    A.L.load()
    return A


def kind_of(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def host(x):
    return x.detach().float().cpu().numpy()


def raw(x):
    import torch
    return x.view(torch.uint8).cpu().numpy()


def marked(rows, cols, dev):
    """A buffer of codes that are all MARK."""
    import torch
    return torch.full((rows, cols), MARK, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)


def scales(rows, blocks, dev, major="block", gap=0):
    """Scales of rows x blocks, all 99, and the buffer they lie in: a block's side by side, or a row's."""
    import torch
    if major == "block":
        buf = torch.full((blocks + 1, rows + gap), 99.0, device=dev)
        return buf[:blocks, :rows].t(), buf
    buf = torch.full((rows + 1, blocks + gap), 99.0, device=dev)
    return buf[:rows, :blocks], buf


def codes(a, dev):
    """Numbers that are e4m3 ones, as a tensor of codes."""
    import torch
    return t(np.asarray(a, np.float32), dev).to(torch.float8_e4m3fn)


def special_rows(x):
    """Rows that codes have to be right on: zeros, infinities, NaN, subnormal and very large magnitudes, ties."""
    cols = x.shape[1]
    x[1] = 0
    x[2, cols // 2] = np.inf
    x[3, cols - 1] = np.nan
    x[4] *= np.float32(1e-38)
    x[5] = np.float32(2e-44) * np.sign(x[5])            # a / 448 leaves fp32's range
    x[6] = 3.38e38 * np.sign(x[6])
    x[7] = -0.0
    x[8, 0] = -np.inf
    x[9] = np.round(x[9] * 32) / 32
    x[9, 0] = 448.0 / 64                                # scale 2^-6: ties between codes
    x[10] = np.float32(1e-42) * np.round(3 * x[10])


# ----------------------------------------------------------------------------
# rows and weights
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [1, 3, 7, 8, 9, 64, 121, 127, 128, 129, 384, 513, 1000, 1096, 1920, 7687])
def test_quantize_rows(api, dev, dtype, cols):
    import torch
    dt, rng = kind_of(dtype), np.random.default_rng(cols)
    rows, blocks = 19, -(-cols // 128)
    x = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32)
    special_rows(x)
    if dtype == "bf16":
        x = host(t(x, dev, dt))
    want_q, want_s = X.e4m3_blocks(x)
    for lead, extra, major, gap in ((0, 0, "block", 0), (1, 5, "row", 0), (3, 0, "block", 3), (0, 1, "row", 2)):
        xb = torch.zeros((rows, cols + lead + extra), device=dev, dtype=dt)
        xb[:, lead: lead + cols] = t(x, dev, dt)
        qb = marked(rows + 1, (blocks + 1) * 128, dev)
        s, sb = scales(rows, blocks, dev, major, gap)
        say("quantize rows", dtype, cols, lead, major)
        api.dc_quantize_f8(xb[:, lead: lead + cols], qb[:rows, : (blocks + (1 if extra else 0)) * 128], s)
        torch.cuda.synchronize()
        assert np.array_equal(host(s), want_s, equal_nan=True)
        assert np.array_equal(host(qb[:rows, : blocks * 128]), want_q)
        b = raw(qb)
        assert (b[rows] == MARK).all() and (b[:, blocks * 128:] == MARK).all()
        assert (host(sb) == 99).sum() == sb.numel() - rows * blocks


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 1920), (3, 7), (127, 130), (128, 128), (129, 257), (200, 8), (300, 1001), (640, 384)])
def test_quantize_weights(api, dev, dtype, rows, cols):
    import torch
    dt, rng = kind_of(dtype), np.random.default_rng(rows + cols)
    nr, blocks = -(-rows // 128), -(-cols // 128)
    x = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32)
    if rows > 256:
        x[130, 5] = np.nan
        x[:128, :128] = 0
        x[256:, 128:256] = 1e-44
        x[140, 300] = np.inf
    if dtype == "bf16":
        x = host(t(x, dev, dt))
    want_q, want_s = X.e4m3_blocks(x, 128)
    for lead, major in ((0, "row"), (1, "block")):
        xb = torch.zeros((rows, cols + lead), device=dev, dtype=dt)
        xb[:, lead:] = t(x, dev, dt)
        qb = marked(rows + 1, (blocks + 1) * 128, dev)
        s, sb = scales(nr, blocks, dev, major, 1)
        say("quantize weights", dtype, rows, cols, lead)
        api.dc_quantize_f8(xb[:, lead:], qb[:rows], s, block_rows=128)
        torch.cuda.synchronize()
        assert np.array_equal(host(s), want_s, equal_nan=True)
        assert np.array_equal(host(qb[:rows, : blocks * 128]), want_q)
        b = raw(qb)
        assert (b[rows] == MARK).all() and (b[:, blocks * 128:] == MARK).all()
        assert (host(sb) == 99).sum() == sb.numel() - nr * blocks


@pytest.mark.parametrize("dtype,rows,cols", [("f32", 1, 1920), ("bf16", 1, 7680), ("bf16", 4099, 1152), ("f32", 1025, 333), ("bf16", 3301, 1921),
                                             ("f32", 9001, 130), ("bf16", 7, 130943), ("f32", 100003, 3), ("bf16", 100003, 5)])
def test_quantize_many_rows(api, dev, dtype, rows, cols):
    import torch
    x = torch.randn((rows, cols), device=dev, generator=torch.Generator(dev).manual_seed(5)).to(kind_of(dtype))
    q = marked(rows, -(-cols // 128) * 128, dev)
    s, _ = scales(rows, -(-cols // 128), dev)
    api.dc_quantize_f8(x, q, s)
    want_q, want_s = X.e4m3_blocks(host(x))
    assert np.array_equal(host(s), want_s) and np.array_equal(host(q), want_q)


STREAMED = 10 << 20                     # bytes of x from which on rows are read past the caches


@pytest.mark.parametrize("dtype,rows,cols,wide", [("bf16", 1301, 4999, True), ("bf16", 1203, 7687, True), ("bf16", 1282, 4096, True), ("bf16", 1300, 4095, False),
                                                  ("f32", 701, 4225, True), ("f32", 643, 4100, True), ("f32", 645, 4095, False), ("f32", 2801, 1001, False)])
def test_quantize_streamed_rows(api, dev, dtype, rows, cols, wide):
    """Rows long enough for the streaming loads, and wide ones (4,096 columns on: a workgroup takes 16 rows x 4 blocks in bf16,
    8 x 2 in fp32), with rows and blocks left over; strided and marked, as the short ones."""
    import torch
    e, rng = 2 if dtype == "bf16" else 4, np.random.default_rng(rows)
    assert rows * cols * e >= STREAMED and (cols >= 4096) == wide
    blocks = -(-cols // 128)
    x = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32)
    x[:, -1] = 3 * np.abs(x).max(1)                     # a last block's scale is its last feature's
    special_rows(x)
    special_rows(x[-11:])                               # of a workgroup of fewer rows
    if dtype == "bf16":
        x = host(t(x, dev, kind_of(dtype)))
    want_q, want_s = X.e4m3_blocks(x)
    for lead, extra, major, gap in ((0, 0, "block", 0), (1, 5, "row", 2)):
        xb = torch.zeros((rows, cols + lead + extra), device=dev, dtype=kind_of(dtype))
        xb[:, lead: lead + cols] = t(x, dev)
        qb = marked(rows + 1, (blocks + 1) * 128, dev)
        s, sb = scales(rows, blocks, dev, major, gap)
        say("quantize streamed rows", dtype, rows, cols, lead)
        api.dc_quantize_f8(xb[:, lead: lead + cols], qb[:rows], s)
        torch.cuda.synchronize()
        assert np.array_equal(host(s), want_s, equal_nan=True)
        assert np.array_equal(host(qb[:rows, : blocks * 128]), want_q)
        b = raw(qb)
        assert (b[rows] == MARK).all() and (b[:, blocks * 128:] == MARK).all()
        assert (host(sb) == 99).sum() == sb.numel() - rows * blocks


# ----------------------------------------------------------------------------
# the norm
# ----------------------------------------------------------------------------
def check_codes(q, s, y, cols):
    """Codes and scales of fp32 numbers that are y but for `off` of themselves: a mean square of cols terms that are added
    eight to a lane, over up to eight pieces of it and six exchanges, then over four waves (7 + 8 + 6 + 3
    roundings, half of them on the root), the square, the mean, eps, root, quotient and the two products: under 24."""
    off = 24 * F32
    pad = -(-cols // 128) * 128
    v = np.zeros((len(y), pad))
    v[:, :cols] = y
    top = np.abs(v).reshape(len(y), -1, 128).max(-1)
    assert (np.abs(s - top / 448) <= (off + 2 * F32) * top / 448).all()
    step = np.repeat(s.astype(np.float64), 128, 1)
    # a quotient carries the scale's error, the division's rounding and then that to the nearest code
    tol = (E4M3 * (1 + 4 * off) + 3 * off) * np.abs(v) + E4M3_LOW * step
    err = np.abs(q * step - v)
    assert (err <= tol).all(), ((err / np.maximum(tol, 1e-300)).max(), np.argwhere(err > tol)[:4])
    assert (q[:, cols:] == 0).all()


@pytest.mark.parametrize("cols", [1, 5, 8, 100, 127, 128, 129, 500, 512, 513, 1000, 1024, 1152, 1921, 2048, 4096, 5003, 8200, 16384])
@pytest.mark.parametrize("x_type,r_type,out_type", [("bf16", "f32", "f32"), ("f32", "bf16", "bf16"), ("f32", None, None), ("bf16", "bf16", "bf16"),
                                                    ("bf16", None, "f32"), ("f32", "f32", None)])
def test_norm(api, dev, cols, x_type, r_type, out_type):
    import torch
    rng = np.random.default_rng(cols)
    rows, blocks, eps = 13, -(-cols // 128), 1e-5
    x = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32)
    r = (3 * rng.standard_normal((rows, cols))).astype(np.float32)
    x[3], r[3] = 0, 0
    x[4], r[4] = 1e-30 * x[4], 1e-30 * r[4]             # eps alone is under the root
    w = (1 + rng.standard_normal(cols)).astype(np.float32)
    for lead, weight, major, in_place in ((0, w, "block", None), (1, None, "row", "residual"), (3, w, "row", "x")):
        xd = torch.zeros((rows + 1, cols + lead), device=dev, dtype=kind_of(x_type))
        xd[:rows, lead:] = t(x, dev)
        xd = xd[:rows, lead:]
        rd = None if r_type is None else t(r, dev, kind_of(r_type))
        h = host(xd) + (0 if rd is None else host(rd))
        out = buf = None
        if out_type is not None:
            buf = torch.full((rows + 1, cols + 2), 7.0, device=dev, dtype=kind_of(out_type))
            out = buf[:rows, 1: 1 + cols]
            if in_place == "residual" and r_type == out_type:
                out, buf = rd, None
            elif in_place == "x" and x_type == out_type:
                out, buf = xd, None
        qb = marked(rows + 1, (blocks + 1) * 128, dev)
        s, sb = scales(rows, blocks, dev, major, 1)
        say("norm", cols, x_type, r_type, out_type, lead)
        api.dc_rms_norm_f8(xd, qb[:rows, : blocks * 128], s, weight=None if weight is None else t(w, dev), eps=eps, residual=rd, out=out)
        torch.cuda.synchronize()
        check_codes(host(qb[:rows, : blocks * 128]), host(s), X.rms_norm(h, weight, eps), cols)
        assert not host(s)[3].any() and not host(qb[3, : blocks * 128]).any()
        if out is not None:
            assert np.array_equal(host(out), h if out_type == "f32" else host(t(h, dev, torch.bfloat16)))
        if buf is not None:
            b = host(buf)
            assert (b[rows] == 7).all() and (b[:, 0] == 7).all() and (b[:, 1 + cols:] == 7).all()
        b = raw(qb)
        assert (b[rows] == MARK).all() and (b[:, blocks * 128:] == MARK).all()
        assert (host(sb) == 99).sum() == sb.numel() - rows * blocks


@pytest.mark.parametrize("rows,cols", [(1, 1920), (3704, 1152), (4097, 1920), (2050, 333), (9000, 129), (1030, 5000)])
def test_norm_of_many_rows(api, dev, rows, cols):
    import torch
    gen = torch.Generator(dev).manual_seed(rows)
    x = torch.randn((rows, cols), device=dev, generator=gen).bfloat16()
    r = torch.randn((rows, cols), device=dev, generator=gen)
    h = host(x) + host(r)
    w = 1 + 0.2 * torch.randn(cols, device=dev, generator=gen)
    q, (s, _) = marked(rows, -(-cols // 128) * 128, dev), scales(rows, -(-cols // 128), dev)
    api.dc_rms_norm_f8(x, q, s, weight=w, residual=r, out=r)
    assert np.array_equal(host(r), h)
    check_codes(host(q), host(s), X.rms_norm(h, host(w), 1e-6), cols)


def check_exactly(q, s, y):
    """Codes and scales that are rounded once from 64 bits, the quotient once more to fp32: all but what lies within 2^-40 of
    a border, of which these draws have none.  A scale below fp32's normal range is rounded in steps of 2^-149."""
    rows, cols = y.shape
    blocks = -(-cols // 128)
    v = np.zeros((rows, blocks * 128))
    v[:, :cols] = y
    want_s = (np.abs(v).reshape(rows, blocks, 128).max(-1) / 448).astype(np.float32)
    assert np.array_equal(s, want_s)
    step = np.repeat(want_s.astype(np.float64), 128, 1)
    z = np.divide(v, step, out=np.zeros_like(v), where=step > 0)
    assert np.array_equal(q, X.e4m3(z.astype(np.float32)))


@pytest.mark.parametrize("rows,cols,r_type", [(3704, 1152, "f32"), (4097, 1920, "bf16"), (300, 5003, None), (999, 200, "f32"), (20000, 128, "bf16")])
def test_norm_writes_the_codes_of_the_definition(api, dev, rows, cols, r_type):
    import torch
    gen = torch.Generator(dev).manual_seed(cols)
    x = torch.randn((rows, cols), device=dev, generator=gen).bfloat16()
    r = None if r_type is None else torch.randn((rows, cols), device=dev, generator=gen).to(kind_of(r_type))
    w = 1 + 0.2 * torch.randn(cols, device=dev, generator=gen)
    blocks = -(-cols // 128)
    q, (s, _) = marked(rows, blocks * 128, dev), scales(rows, blocks, dev)
    api.dc_rms_norm_f8(x, q, s, weight=w, eps=1e-6, residual=r)
    check_exactly(host(q), host(s), X.rms_norm(host(x).astype(np.float64) + (0 if r is None else host(r)), host(w), np.float64(np.float32(1e-6))))


def norm_by_definition(api, dev, rows, cols, x_type, r_type, out_type, lead, weighted, in_place):
    """The norm of rows `lead` values into wider ones: the sum as fp32 and its type hold it, codes and scales exactly, and
    nothing written around them."""
    import torch
    gen, blocks, eps = torch.Generator(dev).manual_seed(cols + lead), -(-cols // 128), 1e-5
    size = torch.exp(torch.randn((rows, 1), device=dev, generator=gen))
    x = torch.zeros((rows, cols + lead), device=dev, dtype=kind_of(x_type))[:, lead:]
    x.copy_(size * torch.randn((rows, cols), device=dev, generator=gen))
    x[min(3, rows - 1)] = 0
    r = None
    if r_type is not None:
        r = torch.zeros((rows, cols + 2 * lead), device=dev, dtype=kind_of(r_type))[:, lead: lead + cols]
        r.copy_(3 * torch.randn((rows, cols), device=dev, generator=gen))
        r[min(3, rows - 1)] = 0
    w = 1 + torch.randn(cols, device=dev, generator=gen) if weighted else None
    h64 = host(x).astype(np.float64) + (0 if r is None else host(r))
    out = buf = None
    if in_place is not None:
        out = x if in_place == "x" else r
        assert in_place == "x" and x_type == out_type or in_place == "residual" and r_type == out_type
    elif out_type is not None:
        buf = torch.full((rows + 1, cols + 2), 7.0, device=dev, dtype=kind_of(out_type))
        out = buf[:rows, 1: 1 + cols]
    qb, (s, sb) = marked(rows + 1, (blocks + 1) * 128, dev), scales(rows, blocks, dev, "row" if lead else "block", 1)
    say("norm by definition", rows, cols, x_type, r_type, out_type, lead, in_place)
    api.dc_rms_norm_f8(x, qb[:rows, : blocks * 128], s, weight=w, eps=eps, residual=r, out=out)
    torch.cuda.synchronize()
    check_exactly(host(qb[:rows, : blocks * 128]), host(s), X.rms_norm(h64, None if w is None else host(w), np.float64(np.float32(eps))))
    if out is not None:
        h = h64.astype(np.float32)
        assert np.array_equal(host(out), h if out_type == "f32" else I.round_bf16(h))
    if buf is not None:
        b = host(buf)
        assert (b[rows] == 7).all() and (b[:, 0] == 7).all() and (b[:, 1 + cols:] == 7).all()
    b = raw(qb)
    assert (b[rows] == MARK).all() and (b[:, blocks * 128:] == MARK).all()
    assert (host(sb) == 99).sum() == sb.numel() - rows * blocks


NORM_TYPES = [("bf16", "f32", "f32", "residual"), ("bf16", "f32", "bf16", "x"), ("f32", "f32", "f32", "x"), ("f32", "f32", None, None), ("f32", "bf16", "bf16", "residual"),
              ("f32", "bf16", "f32", None), ("bf16", "bf16", "bf16", "residual"), ("bf16", "bf16", "f32", None), ("f32", None, "f32", "x"), ("f32", None, "bf16", None),
              ("f32", None, None, None), ("bf16", None, "bf16", "x"), ("bf16", None, None, None)]


@pytest.mark.parametrize("cols", [1, 5, 8, 100, 127, 129, 511, 513, 1000, 1152, 1537, 1921, 2049, 4095, 5003, 8200, 16381])
@pytest.mark.parametrize("x_type,r_type,out_type,in_place", NORM_TYPES)
def test_norm_of_any_rows_by_definition(api, dev, cols, x_type, r_type, out_type, in_place):
    """Ragged widths of every kernel, every pair of types, rows at every element's address, in place and not."""
    norm_by_definition(api, dev, 13, cols, x_type, r_type, out_type, 0, True, in_place)
    norm_by_definition(api, dev, 13, cols, x_type, r_type, out_type, 3, False, None)


@pytest.mark.parametrize("cols", [250, 1001, 1500, 1921, 4090, 5003, 16381])
@pytest.mark.parametrize("x_type,r_type,out_type,in_place", NORM_TYPES)
def test_norm_of_streamed_rows_by_definition(api, dev, cols, x_type, r_type, out_type, in_place):
    """The same where rows are read past the caches, for each number of waves and pieces; a workgroup of four rows is left over."""
    size = {"bf16": 2, "f32": 4, None: 0}
    rows = STREAMED // (cols * (size[x_type] + size[r_type])) // 4 * 4 + 5
    assert rows * cols * (size[x_type] + size[r_type]) >= STREAMED
    norm_by_definition(api, dev, rows, cols, x_type, r_type, out_type, 1, True, in_place)


def test_norm_of_rows_of_any_size(api, dev):
    """Rows from the smallest numbers to the largest: none overflows, and those that eps outweighs are small, not lost."""
    import torch
    x = torch.randn((9, 640), device=dev, generator=torch.Generator(dev).manual_seed(1))
    x *= (10.0 ** torch.tensor([-44, -38, -30, -10, 0, 10, 19, 30, 38], device=dev, dtype=torch.float64)).float()[:, None] / 8
    q, (s, _) = marked(9, 640, dev), scales(9, 5, dev)
    api.dc_rms_norm_f8(x, q, s, eps=1e-6)
    check_exactly(host(q), host(s), X.rms_norm(host(x).astype(np.float64), None, np.float64(np.float32(1e-6))))


def test_norm_of_rows_without_a_number(api, dev):
    """A NaN makes its row NaN, an infinity its block (the others of the row are zeros over an infinite root); the
    padding holds zeros all the same, and other rows keep theirs."""
    import torch
    x = torch.randn((6, 300), device=dev, generator=torch.Generator(dev).manual_seed(3))
    x[1, 299], x[4, 130] = float("nan"), float("inf")
    q, (s, _) = marked(6, 384, dev), scales(6, 3, dev)
    out = torch.empty_like(x)
    api.dc_rms_norm_f8(x, q, s, weight=torch.ones(300, device=dev), out=out)
    bad = np.isnan(host(s))
    assert bad[1].all() and bad[4].tolist() == [False, True, False] and bad.sum() == 4
    q = host(q)
    assert not q[1].any() and not q[4].any() and not q[:, 300:].any() and not host(s)[4, [0, 2]].any()
    assert np.array_equal(host(out), host(x), equal_nan=True)
    keep = [0, 2, 3, 5]
    check_codes(q[keep], host(s)[keep], X.rms_norm(host(x)[keep], None, 1e-6), 300)


# ----------------------------------------------------------------------------
# products
# ----------------------------------------------------------------------------
def whole_inputs(m, n, k, seed):
    """Codes of small whole numbers and scales that are powers of two: |sum| <= 16 k, times 1/4 to 4, in steps of 1/4, is
    held exactly by fp32 up to k = 2^17 - and by eight products' 15 bits."""
    rng = np.random.default_rng(seed)
    x, w = (rng.integers(-4, 5, (r, k)).astype(np.float32) for r in (m, n))
    xs = 2.0 ** rng.integers(-1, 2, (m, k // 128))
    ws = 2.0 ** rng.integers(-1, 2, (-(-n // 128), k // 128))
    return x, xs.astype(np.float32), w, ws.astype(np.float32), *vectors(rng, m, n)


def any_inputs(m, n, k, seed):
    """Codes over e4m3's whole range, subnormal ones among them, and any scales."""
    rng = np.random.default_rng(seed)
    x, w = (X.e4m3(rng.standard_normal((r, k)) * np.exp(1.5 * rng.standard_normal((r, k))) * 8).astype(np.float32) for r in (m, n))
    xs = rng.uniform(1e-4, 2e-2, (m, k // 128)).astype(np.float32)
    ws = rng.uniform(1e-4, 2e-2, (-(-n // 128), k // 128)).astype(np.float32)
    return x, xs, w, ws, *vectors(rng, m, n)


def vectors(rng, m, n):
    return (rng.standard_normal(n).astype(np.float32), rng.standard_normal(n).astype(np.float32),
            rng.standard_normal((m, n)).astype(np.float32))


def check_linear(got, x, xs, w, ws, bias, gate, residual, kind, bf16, whole):
    """The sum: none lost where inputs are whole; else, for fp32 outputs, up to a step (2^-23, as an adder may cut) at
    each of the 128 additions of a block and the K / 128 of the blocks, and two roundings of the scales; for bf16 ones a
    product loses up to 2^-15 of the largest of its eight.  Then the bias, and for the rest as many fp32 roundings as
    in the int8 product: GELU's slope is at most 1.13, its argument carries (14 |y| + 7) roundings, |y| <= 40 matters
    (beyond it the value is z or 0); a residual has two more of |gate v| + |residual|, a product with a gate that has been
    applied to the bias one more."""
    v, size = X.linear_f8(x, xs, w, ws)
    tol = 0.0
    if not whole:
        tol = (2 * (128 + x.shape[1] // 128) + 4) * F32 * size + (8 * 2.0 ** -15 * size if bf16 else 0)
    tol = tol + 4 * F32 * (np.abs(v) + (0 if bias is None else np.abs(bias)))
    if bias is not None:
        v = v + bias
    if kind == "gelu":
        y = np.minimum(np.abs(0.7978845608 * (v + 0.044715 * v ** 3)), 40)
        z = dit.gelu_tanh(v)
        tol = 1.13 * tol + (14 * y + 7) * F32 * np.abs(z) + 2.0 ** -120
        v = z
    elif kind in ("gated", "residual"):
        g = gate if kind == "gated" else np.ones_like(gate)
        tol = np.abs(g) * tol + 3 * F32 * (np.abs(g * v) + np.abs(residual))
        v = residual + g * v
    tol = tol + (BF16 if bf16 else F32) * (np.abs(v) + tol)
    err = np.abs(got - v)
    assert np.isfinite(got).all() and (err <= tol).all(), (err.max(), (err / np.maximum(tol, 1e-300)).max(), np.argwhere(err > tol)[:4])
    return v


def run_linear(api, dev, data, kind, dt, bias=True, major="block", lead=0, gap=0):
    """The product on tensors whose rows start `lead` values into wider ones; what lies around is left as it was."""
    import torch
    x, xs, w, ws, b, gate, res = data
    m, n = len(x), len(w)
    buf = torch.full((m + 1, n + lead + gap), 3.0, device=dev, dtype=kind_of(dt))
    out = buf[:m, lead: lead + n]
    rs = None
    if kind in ("gated", "residual"):
        rs = t(res, dev, kind_of(dt))
        if lead:                                        # in place
            out.copy_(rs)
            rs = out
    sx, _ = scales(m, xs.shape[1], dev, major, lead)
    sx.copy_(t(xs, dev))
    api.dc_linear_f8(codes(x, dev), sx, codes(w, dev), t(ws, dev), out, bias=t(b, dev) if bias else None, gelu=kind == "gelu",
                     gate=t(gate, dev) if kind == "gated" else None, residual=rs)
    torch.cuda.synchronize()
    got = host(buf)
    assert (got[m] == 3).all() and (got[:, :lead] == 3).all() and (got[:, lead + n:] == 3).all()
    return got[:m, lead: lead + n]


def of_type(data, dt, dev):
    """The data with the residual as its type holds it."""
    return (*data[:6], host(t(data[6], dev, kind_of(dt))))


KINDS = [("plain", "f32", True, "block", 0, 0), ("plain", "bf16", False, "row", 1, 2), ("gelu", "bf16", True, "block", 8, 0),
         ("gelu", "f32", False, "block", 0, 1), ("gated", "f32", True, "row", 1, 4), ("gated", "bf16", True, "block", 0, 0),
         ("residual", "f32", False, "block", 0, 0), ("residual", "bf16", True, "block", 3, 0)]


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 191, 300])
@pytest.mark.parametrize("n,k", [(1, 128), (31, 256), (33, 384), (64, 128), (65, 1920), (193, 512), (250, 7680), (1152, 640)])
def test_linear_ragged(api, dev, m, n, k):
    """Few rows and odd widths, each epilogue, with and without a bias, strided operands and outputs."""
    data = whole_inputs(m, n, k, m + n)
    say("linear ragged", m, n, k)
    for kind, dt, bias, major, lead, gap in KINDS:
        got = run_linear(api, dev, data, kind, dt, bias, major, lead, gap)
        d = of_type(data, dt, dev)
        v = check_linear(got, *d[:4], d[4] if bias else None, d[5], d[6], kind, dt == "bf16", True)
        if kind == "plain" and dt == "bf16":            # one rounding, of an exact sum
            assert np.array_equal(got, I.round_bf16(v.astype(np.float32)))


F8_TILES = ("192x256", "192x128", "128x128", "64x128", "64x64", "64x64 x 2", "32x64 x 2", "32x32 x 4", "32x32 x 8", "16x16 x 8",
            "column of 2", "column", "192x256 then 192x128", "192x256 then 64x64 x 2", "128x128 then 64x64")
TILE_SHAPES = {     # (M, N, K), type of the outputs: the tile on 256 compute units
    (1608, 5515, 512, "bf16"): "192x256", (1442, 4158, 1280, "bf16"): "128x128", (983, 4757, 512, "bf16"): "192x128",
    (1301, 5765, 1024, "bf16"): "128x128", (637, 3139, 3840, "bf16"): "64x128", (269, 2860, 1664, "bf16"): "64x64",
    (574, 1089, 2048, "bf16"): "64x64 x 2", (65, 5128, 3840, "bf16"): "32x64 x 2", (61, 4095, 3584, "bf16"): "32x32 x 4",
    (127, 2023, 3840, "bf16"): "32x32 x 8", (15, 4927, 2048, "bf16"): "16x16 x 8", (1, 6403, 3840, "bf16"): "column", (2, 6403, 3840, "bf16"): "column of 2",
    (978, 4778, 512, "f32"): "192x128", (1301, 5765, 1024, "f32"): "128x128", (637, 3139, 3840, "f32"): "64x128", (411, 4867, 640, "f32"): "64x64",
    (574, 1089, 2048, "f32"): "64x64 x 2", (65, 5128, 3840, "f32"): "32x64 x 2", (964, 384, 3456, "f32"): "32x32 x 4", (476, 411, 3840, "f32"): "32x32 x 8",
    (15, 4927, 2048, "f32"): "16x16 x 8", (1, 6403, 3840, "f32"): "column", (2, 6403, 3840, "f32"): "column of 2",
    (3273, 5214, 512, "bf16"): "192x256 then 192x128", (3470, 3450, 768, "bf16"): "192x256 then 64x64 x 2", (1740, 5580, 1536, "f32"): "128x128 then 64x64",
    (3694, 2363, 640, "f32"): "128x128 then 64x64", (2945, 1345, 512, "bf16"): "128x128 then 64x64", (700, 7, 640, "bf16"): "16x16 x 8", (700, 3, 640, "f32"): "16x16 x 8",
}


def f8_tile(m, n, k, dt, cus):
    return F8_TILES[_native("_ZN2dc7f8_tileEiiiib", m, n, k // 128, cus, dt == "f32")]


@pytest.mark.parametrize("mnkt", list(TILE_SHAPES))
@pytest.mark.parametrize("kind", ["plain", "gelu", "gated"])
def test_linear_tiles(api, dev, mnkt, kind):
    """Every tile of the product in both types, ragged in rows and columns, and whole lines of outputs."""
    m, n, k, dt = mnkt
    assert f8_tile(m, n, k, dt, compute_units(dev)) == TILE_SHAPES[mnkt]
    data = whole_inputs(m, n, k, 7)
    pick = np.unique(np.r_[0, m - 1, np.random.default_rng(0).integers(0, m, 150)])
    for width in sorted({n, n // 64 * 64 or n}):
        if f8_tile(m, width, k, dt, compute_units(dev)) != TILE_SHAPES[mnkt]:
            continue
        x, xs, w, ws, b, gate, res = data
        cut = (x, xs, w[:width], ws[: -(-width // 128)], b[:width], gate[:width], np.ascontiguousarray(res[:, :width]))
        say("linear tile", mnkt, width, TILE_SHAPES[mnkt], kind)
        got = run_linear(api, dev, cut, kind, dt, kind != "plain")
        d = of_type(cut, dt, dev)
        check_linear(got[pick], d[0][pick], d[1][pick], d[2], d[3], d[4] if kind != "plain" else None, d[5], d[6][pick], kind, dt == "bf16", True)


FEW_STEPS = {       # one to three k-steps, no more than a tile's stages or one more: shapes and tiles as above
    (1690, 5963, 128, "bf16"): "192x256", (676, 7466, 128, "bf16"): "192x128", (8888, 688, 128, "bf16"): "128x128",
    (1739, 1763, 128, "bf16"): "64x128", (1299, 69, 128, "bf16"): "64x64", (131, 41, 128, "bf16"): "16x16 x 8",
    (895, 4717, 128, "bf16"): "128x128 then 64x64", (4070, 2298, 256, "bf16"): "192x256", (677, 7317, 256, "bf16"): "192x128",
    (2075, 2959, 256, "bf16"): "128x128", (558, 5507, 256, "bf16"): "64x128", (1354, 399, 256, "bf16"): "64x64",
    (136, 598, 256, "bf16"): "32x64 x 2", (131, 43, 256, "bf16"): "16x16 x 8", (6997, 2436, 256, "bf16"): "192x256 then 192x128",
    (5182, 2320, 256, "bf16"): "192x256 then 64x64 x 2", (5116, 809, 256, "bf16"): "128x128 then 64x64", (5204, 1764, 384, "bf16"): "192x256",
    (6030, 806, 384, "bf16"): "192x128", (769, 7964, 384, "bf16"): "128x128", (7663, 400, 384, "bf16"): "64x128",
    (359, 1530, 384, "bf16"): "64x64", (624, 398, 384, "bf16"): "32x64 x 2", (506, 144, 384, "bf16"): "32x32 x 4",
    (143, 40, 384, "bf16"): "16x16 x 8", (2832, 6042, 384, "bf16"): "192x256 then 192x128", (7146, 1704, 384, "bf16"): "192x256 then 64x64 x 2",
    (2820, 1452, 384, "bf16"): "128x128 then 64x64", (1337, 3613, 128, "f32"): "192x128", (1028, 5891, 128, "f32"): "128x128",
    (1683, 1831, 128, "f32"): "64x128", (2046, 63, 128, "f32"): "64x64", (53, 119, 128, "f32"): "16x16 x 8",
    (1655, 2588, 128, "f32"): "128x128 then 64x64", (1317, 3739, 256, "f32"): "192x128", (4039, 1493, 256, "f32"): "128x128",
    (386, 7903, 256, "f32"): "64x128", (158, 3499, 256, "f32"): "64x64", (8338, 43, 256, "f32"): "64x64 x 2",
    (289, 395, 256, "f32"): "32x64 x 2", (70, 92, 256, "f32"): "16x16 x 8", (6568, 651, 256, "f32"): "128x128 then 64x64",
    (2959, 1675, 384, "f32"): "192x128", (1986, 3042, 384, "f32"): "128x128", (393, 7845, 384, "f32"): "64x128",
    (2223, 255, 384, "f32"): "64x64", (81, 8396, 384, "f32"): "32x64 x 2", (52, 2275, 384, "f32"): "32x32 x 4",
    (107, 62, 384, "f32"): "16x16 x 8", (2364, 1793, 384, "f32"): "128x128 then 64x64",
}


@pytest.mark.parametrize("mnkt", list(FEW_STEPS))
@pytest.mark.parametrize("kind", ["plain", "gelu", "gated"])
def test_linear_tiles_of_few_k_steps(api, dev, mnkt, kind):
    """Sums that end while a tile's stages are still being filled, or a k-step later."""
    m, n, k, dt = mnkt
    assert f8_tile(m, n, k, dt, compute_units(dev)) == FEW_STEPS[mnkt]
    data = whole_inputs(m, n, k, 9)
    pick = np.unique(np.r_[0, m - 1, np.random.default_rng(0).integers(0, m, 150)])
    say("linear few k-steps", mnkt, FEW_STEPS[mnkt], kind)
    got = run_linear(api, dev, data, kind, dt, kind != "plain")
    d = of_type(data, dt, dev)
    check_linear(got[pick], d[0][pick], d[1][pick], d[2], d[3], d[4] if kind != "plain" else None, d[5], d[6][pick], kind, dt == "bf16", True)


@pytest.mark.parametrize("m,n,k", [(1, 1920, 7680), (2, 333, 5120), (50, 333, 1920), (257, 513, 1152), (700, 1920, 1920), (1, 40, 65536)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_linear_of_any_codes(api, dev, m, n, k, dt):
    data = any_inputs(m, n, k, m + k)
    say("linear any", m, n, k, dt)
    for kind in ("plain", "gelu", "gated"):
        got = run_linear(api, dev, data, kind, dt)
        d = of_type(data, dt, dev)
        check_linear(got, *d, kind, dt == "bf16", False)


@pytest.mark.parametrize("mnkt", list(TILE_SHAPES))
@pytest.mark.parametrize("kind", ["plain", "gated"])
def test_linear_tiles_of_any_codes(api, dev, mnkt, kind):
    """Every tile on codes over their whole range and any scales."""
    m, n, k, dt = mnkt
    assert f8_tile(m, n, k, dt, compute_units(dev)) == TILE_SHAPES[mnkt]
    data = any_inputs(m, n, k, 8)
    pick = np.unique(np.r_[0, m - 1, np.random.default_rng(1).integers(0, m, 150)])
    say("linear tile, any codes", mnkt, TILE_SHAPES[mnkt], kind)
    got = run_linear(api, dev, data, kind, dt, kind != "plain")
    d = of_type(data, dt, dev)
    check_linear(got[pick], d[0][pick], d[1][pick], d[2], d[3], d[4] if kind != "plain" else None, d[5], d[6][pick], kind, dt == "bf16", False)


def test_linear_in_fp32_keeps_small_products(api, dev):
    """Products of 1 beside one of 65,536 in each block: fp32 outputs hold the sum exactly."""
    import torch
    x, w = (np.ones((40, 1024), np.float32) for _ in range(2))
    x[:, 5::128] = 256
    w[:, 5::128] = 256
    one = torch.ones((1, 1), device=dev)
    out = torch.zeros((40, 40), device=dev)
    api.dc_linear_f8(codes(x, dev), one.expand(40, 8), codes(w, dev), one.expand(1, 8), out)
    assert (host(out) == 8 * (65536 + 127)).all()


def test_linear_scales_of_any_strides(api, dev):
    """One scale for all rows or all blocks, a row's scales side by side or not, and codes with rows apart."""
    import torch
    x, xs, w, ws, bias, gate, res = whole_inputs(150, 260, 512, 2)
    xd, wd = (torch.full((len(a), 512 + 48), 0.5, device=dev).to(torch.float8_e4m3fn) for a in (x, w))
    xd[:, 16: 528].copy_(codes(x, dev))
    wd[:, 32: 544].copy_(codes(w, dev))
    xd, wd = xd[:, 16: 528], wd[:, 32: 544]
    wide = torch.zeros((450, 12), device=dev)
    apart = wide[::3, ::3]
    apart.copy_(t(xs, dev))
    two, per_block, per_row = torch.full((1, 1), 2.0, device=dev), t(xs[:1], dev), t(xs[:, :1], dev)
    for sx, host_s in ((apart, xs), (two.expand(150, 4), 2 + 0 * xs), (per_block.expand(150, 4), xs[:1].repeat(150, 0)),
                       (per_row.expand(150, 4), xs[:, :1].repeat(4, 1))):
        for sw, host_w in ((t(ws, dev), ws), (t(ws.T, dev).t(), ws), (two.expand(3, 4), 2 + 0 * ws)):
            out = torch.zeros((150, 260), device=dev)
            api.dc_linear_f8(xd, sx, wd, sw, out)
            check_linear(host(out), x, host_s, w, host_w, None, gate, res, "plain", False, True)


SCALE_SHAPES = [(1, 40, 256), (1, 41, 4224), (2, 333, 640), (9, 5, 384), (20, 70, 384), (50, 300, 1024), (300, 400, 512), (1301, 5765, 384),
                (1608, 5515, 512), (3273, 5214, 512)]


@pytest.mark.parametrize("m,n,k", SCALE_SHAPES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_linear_scales_at_the_ends_of_their_range(api, dev, m, n, k, dt):
    """Products of two scales from 2^-126 to 2^127, one scale far from 1 or both: the sums are exact, and outputs are
    rounded once."""
    import torch
    x, xs, w, ws, _, _, _ = whole_inputs(m, n, k, 11)
    one, pick = np.zeros_like(x), np.unique(np.r_[0, m - 1, np.random.default_rng(0).integers(0, m, 60)])
    one[np.arange(m), np.arange(m) * 37 % k] = 1        # a row of one 1: outputs are one product
    for codes_x, codes_w, ex, ew in ((x, w, -63, -63), (x, w, 1, -127), (x, w, -126, 0), (x, w, -140, 20), (x, w, 100, -100), (one, np.sign(w), 64, 63),
                                     (one, np.sign(w), 0, 127), (one, np.sign(w), -22, -100)):
        sx, sw = np.float32(2.0) ** np.float32(ex) * np.ones_like(xs), np.float32(2.0) ** np.float32(ew) * np.ones_like(ws)
        out = torch.empty((m, n), device=dev, dtype=kind_of(dt))
        say("linear scales", m, n, k, dt, ex, ew)
        api.dc_linear_f8(codes(codes_x, dev), t(sx, dev), codes(codes_w, dev), t(sw, dev), out)
        want = X.linear_f8(codes_x[pick], sx[pick], codes_w, sw)[0].astype(np.float32)
        assert np.array_equal(host(out)[pick], want if dt == "f32" else I.round_bf16(want))


@pytest.mark.parametrize("m,n,k", SCALE_SHAPES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_linear_scales_outside_their_range(api, dev, m, n, k, dt):
    """Below 2^-126 a product of two scales is off by half a step of 2^-149, and the whole numbers that it is multiplied with
    make of it what they sum to; up to K / 128 + 16 additions (of blocks, of what lanes, waves and groups hold) and the output are
    rounded to 2^-24 or half a step (2^-150; bf16 2^-8 and 2^-134).  From 2^128 on no output is a number."""
    import torch
    x, xs, w, ws, _, _, _ = whole_inputs(m, n, k, 12)
    pick = np.unique(np.r_[0, m - 1, np.random.default_rng(0).integers(0, m, 60)])
    rng = np.random.default_rng(13)
    sx = (rng.uniform(1, 2, xs.shape) * 2.0 ** -70).astype(np.float32)
    sw = (rng.uniform(1, 2, ws.shape) * 2.0 ** -69).astype(np.float32)
    out = torch.empty((m, n), device=dev, dtype=kind_of(dt))
    say("linear small scales", m, n, k, dt)
    api.dc_linear_f8(codes(x, dev), t(sx, dev), codes(w, dev), t(sw, dev), out)
    v, size = X.linear_f8(x[pick], sx[pick], w, sw)
    tol = np.abs(x[pick]).astype(np.float64) @ np.abs(w).T * 2.0 ** -150 + (k // 128 + 16) * (F32 * size + 2.0 ** -150)
    tol = tol + np.maximum((BF16 if dt == "bf16" else F32) * (np.abs(v) + tol), 2.0 ** -134 if dt == "bf16" else 2.0 ** -150)
    err = np.abs(host(out)[pick] - v)
    assert (err <= tol).all(), (err / tol).max()
    sx[:], sw[:] = 2.0 ** 64, 2.0 ** 64
    say("linear large scales", m, n, k, dt)
    api.dc_linear_f8(codes(x, dev), t(sx, dev), codes(w, dev), t(sw, dev), out)
    assert not torch.isfinite(out).any()


def test_linear_rows_beyond_32_bit_offsets(api, dev):
    """Rows 4 MiB apart: the last ones lie past 2^31 bytes, in x and in w."""
    import torch
    x, xs, w, ws, bias, gate, res = whole_inputs(700, 600, 256, 3)
    for dt in ("f32", "bf16"):
        big = [torch.empty((r, 1 << 22), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)[:, :256] for r in (700, 600)]
        big[0].copy_(codes(x, dev))
        big[1].copy_(codes(w, dev))
        out = torch.empty((700, 600), device=dev, dtype=kind_of(dt))
        say("far rows", dt)
        api.dc_linear_f8(big[0], t(xs, dev), big[1], t(ws, dev), out)
        check_linear(host(out), x, xs, w, ws, None, gate, res, "plain", dt == "bf16", True)


def test_linear_of_blocks_without_a_number(api, dev):
    """Rows and weight blocks that held a NaN or an infinity are NaN in the product, the others are not."""
    import torch
    gen = torch.Generator(dev).manual_seed(1)
    x, w = torch.randn((70, 200), device=dev, generator=gen), torch.randn((300, 200), device=dev, generator=gen)
    x[3, 7], x[66, 199], w[290, 150] = float("nan"), float("inf"), float("-inf")
    q, (s, _), wq, (wsc, _) = marked(70, 256, dev), scales(70, 2, dev), marked(300, 256, dev), scales(3, 2, dev, "row")
    api.dc_quantize_f8(x, q, s)
    api.dc_quantize_f8(w, wq, wsc, block_rows=128)
    for dt in ("f32", "bf16"):
        out = torch.empty((70, 300), device=dev, dtype=kind_of(dt))
        api.dc_linear_f8(q, s, wq, wsc, out)
        bad = np.isnan(host(out))
        assert bad[[3, 66]].all() and bad[:, 256:].all() and bad.sum() == 2 * 300 + 68 * 44


@pytest.mark.parametrize("m,n,k", [(1, 40, 256), (1, 41, 4224), (2, 333, 640), (9, 5, 384), (50, 300, 1024), (300, 400, 512), (1740, 5580, 512), (3096, 5202, 640)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_linear_of_codes_that_are_no_numbers(api, dev, m, n, k, dt):
    """The codes 0x7F and 0xFF are NaN: in a product's row and column that meet them, and nowhere else."""
    import torch
    x, xs, w, ws, b, _, _ = whole_inputs(m, n, k, 3)
    xq, wq = codes(x, dev), codes(w, dev)
    i, j = m - 1, n // 2
    xq.view(torch.uint8)[i, k - 1], wq.view(torch.uint8)[j, 0] = 0x7F, 0xFF
    out = torch.empty((m, n), device=dev, dtype=kind_of(dt))
    say("linear no numbers", m, n, k, dt)
    api.dc_linear_f8(xq, t(xs, dev), wq, t(ws, dev), out, bias=t(b, dev))
    bad = torch.isnan(out)
    assert bad[i].all() and bad[:, j].all() and int(bad.sum()) == m + n - 1


@pytest.mark.parametrize("m,n,k,dt", [(2945, 1345, 512, "bf16"), (1740, 5580, 1536, "f32"), (3096, 5202, 640, "bf16"), (1717, 4990, 896, "bf16"), (70, 131, 384, "f32"),
                                        (1608, 5515, 512, "bf16"), (3273, 5214, 512, "bf16")])
def test_linear_onto_its_residual(api, dev, m, n, k, dt):
    """In place, and once more: the same bits as into a tensor of its own."""
    import torch
    x, xs, w, ws, b, gate, res = whole_inputs(m, n, k, 5)
    given = [codes(x, dev), t(xs, dev), codes(w, dev), t(ws, dev)]
    r = t(res, dev, kind_of(dt))
    say("linear in place", m, n, k, dt)
    outs = [torch.empty_like(r), torch.empty_like(r), r.clone()]
    for out in outs:
        api.dc_linear_f8(*given, out, bias=t(b, dev), gate=t(gate, dev), residual=out if out is outs[2] else r)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_no_rows(api, dev):
    import torch
    none = torch.empty((0, 128), device=dev)
    q, s = none.to(torch.float8_e4m3fn), torch.empty((0, 1), device=dev)
    api.dc_quantize_f8(none, q, s)
    api.dc_rms_norm_f8(none, q, s, residual=none, out=none)
    api.dc_linear_f8(q, s, codes(np.ones((8, 128)), dev), torch.ones((1, 1), device=dev), torch.empty((0, 8), device=dev))
    torch.cuda.synchronize()


def test_one_row_of_any_stride(api, dev):
    """A single row's stride says nothing: rows cut out of wider ones are taken as they are."""
    import torch
    wide = torch.randn((1, 203), device=dev, generator=torch.Generator(dev).manual_seed(2))
    q, s, y = marked(1, 333, dev), torch.zeros((1, 2), device=dev), torch.zeros((1, 41), device=dev)
    x, row, out = (v.as_strided((1, n), (st, 1)) for v, n, st in ((wide, 200, 7), (q, 256, 3), (y, 40, 1)))
    api.dc_quantize_f8(x, row, s.as_strided((1, 2), (0, 1)))
    want_q, want_s = X.e4m3_blocks(host(x))
    assert np.array_equal(host(row), want_q) and np.array_equal(host(s), want_s)
    w = np.random.default_rng(1).integers(-4, 5, (40, 256)).astype(np.float32)
    api.dc_linear_f8(row, s, codes(w, dev), torch.ones((1, 2), device=dev), out)
    check_linear(host(out), want_q, want_s, w, np.ones((1, 2)), None, np.ones(40), None, "plain", False, False)
    assert host(y)[0, 40] == 0


# ----------------------------------------------------------------------------
# together, in graphs and on streams
# ----------------------------------------------------------------------------
def mlp_state(dev, m, d, f, seed):
    """A block's MLP: norm of x + h, up with GELU, codes of the hidden rows, down onto the sum."""
    import torch
    gen = torch.Generator(dev).manual_seed(seed)
    s = dict(x=torch.randn((m, d), device=dev, generator=gen).bfloat16(), h=torch.randn((m, d), device=dev, generator=gen),
             weight=1 + 0.2 * torch.randn(d, device=dev, generator=gen), gate=torch.randn(d, device=dev, generator=gen),
             b1=torch.randn(f, device=dev, generator=gen), b2=torch.randn(d, device=dev, generator=gen),
             w1=0.05 * torch.randn((f, d), device=dev, generator=gen), w2=0.05 * torch.randn((d, f), device=dev, generator=gen))
    blocks = [-(-v // 128) for v in (d, f)]
    s.update(q=marked(m, 128 * blocks[0], dev), s=scales(m, blocks[0], dev)[0], z=torch.zeros((m, f), device=dev, dtype=torch.bfloat16),
             zq=marked(m, 128 * blocks[1], dev), zs=scales(m, blocks[1], dev)[0], w1q=marked(f, 128 * blocks[0], dev),
             w2q=marked(d, 128 * blocks[1], dev), w1s=scales(blocks[1], blocks[0], dev, "row")[0],
             w2s=scales(blocks[0], blocks[1], dev, "row")[0], y=torch.zeros((m, d), device=dev))
    return s


def mlp_calls(api, b, stream=None):
    api.dc_quantize_f8(b["w1"], b["w1q"], b["w1s"], block_rows=128, stream=stream)
    api.dc_quantize_f8(b["w2"], b["w2q"], b["w2s"], block_rows=128, stream=stream)
    api.dc_rms_norm_f8(b["x"], b["q"], b["s"], weight=b["weight"], residual=b["h"], out=b["h"], stream=stream)
    api.dc_linear_f8(b["q"], b["s"], b["w1q"], b["w1s"], b["z"], bias=b["b1"], gelu=True, stream=stream)
    api.dc_quantize_f8(b["z"], b["zq"], b["zs"], stream=stream)
    api.dc_linear_f8(b["zq"], b["zs"], b["w2q"], b["w2s"], b["y"], bias=b["b2"], gate=b["gate"], residual=b["h"], stream=stream)


def bits(x):
    import torch
    return x.view(torch.uint8) if x.element_size() == 1 else x


@pytest.mark.parametrize("m,d,f", [(1, 256, 512), (37, 200, 333), (300, 1152, 4608)])
def test_an_mlp(api, dev, m, d, f):
    """Step by step: each call's result from the one before, against the definition of that call."""
    b = mlp_state(dev, m, d, f, 4)
    x, h = host(b["x"]), host(b["h"])
    mlp_calls(api, b)
    assert np.array_equal(host(b["h"]), x + h)
    for w, q, s in (("w1", "w1q", "w1s"), ("w2", "w2q", "w2s")):
        want_q, want_s = X.e4m3_blocks(host(b[w]), 128)
        assert np.array_equal(host(b[q]), want_q) and np.array_equal(host(b[s]), want_s)
    check_codes(host(b["q"]), host(b["s"]), X.rms_norm(x + h, host(b["weight"]), 1e-6), d)
    check_linear(host(b["z"]), host(b["q"]), host(b["s"]), host(b["w1q"]), host(b["w1s"]), host(b["b1"]), None, None, "gelu", True, False)
    want_q, want_s = X.e4m3_blocks(host(b["z"]))
    assert np.array_equal(host(b["zq"]), want_q) and np.array_equal(host(b["zs"]), want_s)
    y = check_linear(host(b["y"]), host(b["zq"]), host(b["zs"]), host(b["w2q"]), host(b["w2s"]), host(b["b2"]), host(b["gate"]),
                     x + h, "gated", False, False)
    # the whole against the unquantised MLP: every operand is within 2^-4 of itself, and errors are of either sign
    z = dit.gelu_tanh(X.rms_norm(x + h, host(b["weight"]), 1e-6) @ host(b["w1"]).astype(np.float64).T + host(b["b1"]))
    full = x + h + host(b["gate"]) * (z @ host(b["w2"]).astype(np.float64).T + host(b["b2"]))
    assert np.linalg.norm(y - full) < 4 * E4M3 * np.linalg.norm(full - x - h)


def test_captured_and_replayed(api, dev):
    """All of the calls in one graph on a stream of their own, replayed on changing inputs between eager work,
    against the eager calls."""
    import torch
    graphed, eager = (mlp_state(dev, 300, 640, 1280, 3) for _ in range(2))
    inputs = ("x", "h", "w1", "w2")
    gen = torch.Generator(dev).manual_seed(9)

    def fill():
        for n in inputs:
            v = torch.randn(eager[n].shape, device=dev, generator=gen)
            for b in (graphed, eager):
                b[n].copy_(v)

    fill()
    mlp_calls(api, eager)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        mlp_calls(api, graphed)
    for i in range(4):
        fill()
        graph.replay()
        mlp_calls(api, eager)
        torch.cuda.synchronize()
        for n in graphed:
            assert torch.equal(bits(graphed[n]), bits(eager[n])), (i, n)
    # on another stream than the current one
    other = mlp_state(dev, 300, 640, 1280, 3)
    want = mlp_state(dev, 300, 640, 1280, 3)
    mlp_calls(api, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mlp_calls(api, other, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(bits(other[n]), bits(want[n])), n


def test_two_streams_at_once(api, dev):
    """The calls keep nothing between them: two streams that work side by side get what each gets alone."""
    import torch
    alone, together = ([mlp_state(dev, m, 640, 1280, m) for m in (700, 9)] for _ in range(2))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for b in alone:
        mlp_calls(api, b, streams[0])
        torch.cuda.synchronize()
    for b, s in zip(together, streams):
        mlp_calls(api, b, s)
    torch.cuda.synchronize()
    for a, b in zip(alone, together):
        for n in a:
            assert torch.equal(bits(a[n]), bits(b[n])), n


def test_rows_beyond_32_bit_offsets(api, dev):
    """Rows 8 MiB apart, the last of them past 2^32 bytes: values, sums and codes."""
    import torch
    rows, cols = 600, 300
    x = torch.randn((rows, cols), device=dev, generator=torch.Generator(dev).manual_seed(8))
    far = [torch.empty((rows, 1 << 21), device=dev)[:, :cols] for _ in range(2)]
    q = torch.empty((rows, 1 << 23), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)[:, :384]
    s, _ = scales(rows, 3, dev)
    far[0].copy_(x)
    api.dc_quantize_f8(far[0], q, s)
    want_q, want_s = X.e4m3_blocks(host(x))
    assert np.array_equal(host(q), want_q) and np.array_equal(host(s), want_s)
    api.dc_rms_norm_f8(far[0], q, s, residual=far[0], out=far[1])
    assert np.array_equal(host(far[1]), 2 * host(x))
    check_codes(host(q), host(s), X.rms_norm(2 * host(x), None, 1e-6), cols)
