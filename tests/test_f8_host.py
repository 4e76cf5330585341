"""The e4m3 entry points refuse bad arguments on the host: every call below ends before any device work (the pointers are
never dereferenced), and the definitions they are tested against hold on small cases worked out by hand."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import ext as X
from paper_2608_16354_amd import _lib as L

FAKE = 0x100000
ARG, SHAPE, DTYPE = L.DC_ERR_ARG, L.DC_ERR_SHAPE, L.DC_ERR_DTYPE


@pytest.fixture(scope="module")
def lib():
    return L.load()


def quantize(**more):
    a = dict(rows=4, cols=200, x=FAKE, x_dtype=1, ld_x=200, block_rows=1, q=2 * FAKE, ld_q=256, scale=3 * FAKE, scale_row=1, scale_block=4)
    a.update(more)
    return L.QuantizeF8Args(**a)


def norm(**more):
    a = dict(rows=4, cols=200, x=FAKE, x_dtype=1, ld_x=200, residual=2 * FAKE, residual_dtype=0, ld_residual=200, sum=3 * FAKE, sum_dtype=0,
             ld_sum=200, weight=FAKE, eps=1e-6, q=4 * FAKE, ld_q=256, scale=5 * FAKE, scale_row=1, scale_block=4)
    a.update(more)
    return L.RmsNormF8Args(**a)


def linear(**more):
    a = dict(rows=4, out_features=200, in_features=256, x=FAKE, ld_x=256, x_scale=FAKE, x_scale_row=1, x_scale_block=4, w=FAKE, ld_w=256,
             w_scale=FAKE, w_scale_row=2, w_scale_block=1, bias=FAKE, gelu=0, gate=None, residual=None, ld_residual=0, out=2 * FAKE,
             out_dtype=0, ld_out=200)
    a.update(more)
    return L.LinearF8Args(**a)


CODES = [(dict(q=None), ARG), (dict(q=FAKE + 4), ARG), (dict(ld_q=255), ARG), (dict(ld_q=260), ARG), (dict(ld_q=248), ARG),
         (dict(scale=None), ARG), (dict(scale=FAKE + 2), ARG), (dict(scale_row=0), ARG), (dict(scale_row=-1), ARG), (dict(scale_block=0), ARG),
         (dict(scale_block=3), ARG), (dict(scale_row=2), ARG), (dict(scale_block=(1 << 31) + 1), ARG), (dict(rows=-1), ARG),
         (dict(rows=1 << 24), ARG), (dict(cols=0), ARG), (dict(x=None), ARG), (dict(x_dtype=2), DTYPE), (dict(ld_x=199), ARG),
         (dict(x=FAKE + 1), ARG), (dict(x=FAKE + 2, x_dtype=0), ARG), (dict(rows=0, x=None, q=None, scale=None), L.DC_OK)]


@pytest.mark.parametrize("more,code", CODES + [
    (dict(block_rows=0), ARG), (dict(block_rows=64), ARG), (dict(cols=1 << 24, ld_x=1 << 24, ld_q=1 << 24), ARG),
    (dict(block_rows=128, rows=300, scale_block=2), ARG),
    (dict(rows=(1 << 24) - 1, cols=(1 << 24) - 1, ld_x=1 << 24, ld_q=1 << 24, scale_block=1 << 24), SHAPE)])
def test_quantize_refuses(lib, more, code):
    a = quantize(**more)
    assert lib.dc_quantize_f8(C.byref(a), None) == code


@pytest.mark.parametrize("more,code", CODES + [
    (dict(cols=16385, ld_x=16385, ld_residual=16385, ld_sum=16385, ld_q=16512), ARG), (dict(eps=0.0), ARG), (dict(eps=-1.0), ARG),
    (dict(eps=math.nan), ARG), (dict(eps=math.inf), ARG), (dict(weight=FAKE + 2), ARG), (dict(residual=FAKE + 2), ARG),
    (dict(residual_dtype=7), DTYPE), (dict(ld_residual=199), ARG), (dict(sum=FAKE + 2), ARG), (dict(sum_dtype=-1), DTYPE), (dict(ld_sum=100), ARG),
    (dict(sum=FAKE), ARG),                                      # x in place: another type
    (dict(sum=FAKE, sum_dtype=1, ld_sum=201), ARG), (dict(sum=2 * FAKE, ld_sum=201), ARG), (dict(sum=2 * FAKE, sum_dtype=1), ARG)])
def test_norm_refuses(lib, more, code):
    a = norm(**more)
    assert lib.dc_rms_norm_f8(C.byref(a), None) == code


RES = dict(residual=FAKE, ld_residual=200)


@pytest.mark.parametrize("more,code", [
    (dict(out_dtype=2), DTYPE), (dict(rows=-1), ARG), (dict(rows=1 << 24), ARG), (dict(out_features=0), ARG),
    (dict(out_features=1 << 24, ld_out=1 << 24), ARG), (dict(gelu=2), ARG), (dict(gate=FAKE), ARG), (dict(RES, gelu=1), ARG),
    (dict(RES, ld_residual=199), ARG), (dict(RES, residual=2 * FAKE, ld_residual=201), ARG), (dict(ld_out=199), ARG),
    (dict(x=None), ARG), (dict(x_scale=None), ARG), (dict(w=None), ARG), (dict(w_scale=None), ARG), (dict(out=None), ARG),
    (dict(x=FAKE + 8), ARG), (dict(w=FAKE + 8), ARG), (dict(out=FAKE + 2), ARG), (dict(out=FAKE + 1, out_dtype=1), ARG), (dict(bias=FAKE + 2), ARG),
    (dict(RES, gate=FAKE + 2), ARG), (dict(RES, residual=FAKE + 2), ARG), (dict(x_scale=FAKE + 2), ARG), (dict(w_scale=FAKE + 1), ARG),
    (dict(ld_out=1 << 32), ARG), (dict(residual=FAKE, ld_residual=1 << 32), ARG),
    (dict(x_scale_row=-1), ARG), (dict(w_scale_block=-1), ARG), (dict(x_scale_row=1 << 21), ARG), (dict(w_scale_row=(1 << 31) + 1), ARG),
    (dict(in_features=0), SHAPE), (dict(in_features=64), SHAPE), (dict(in_features=200), SHAPE),
    (dict(in_features=(1 << 22) + 128, ld_x=(1 << 22) + 128, ld_w=(1 << 22) + 128), SHAPE), (dict(ld_x=240), SHAPE), (dict(ld_w=264), SHAPE),
    (dict(ld_x=(1 << 22) + 16), SHAPE), (dict(rows=(1 << 24) - 1, out_features=1 << 20, ld_out=1 << 20), SHAPE),
    (dict(rows=0, x=None, out=None), L.DC_OK)])
def test_linear_refuses(lib, more, code):
    a = linear(**more)
    assert lib.dc_linear_f8(C.byref(a), None) == code


@pytest.mark.parametrize("f", ["dc_quantize_f8", "dc_rms_norm_f8", "dc_linear_f8"])
def test_null_is_refused(lib, f):
    assert getattr(lib, f)(None, None) == ARG
    assert b"NULL" in lib.dc_last_error()


# ----------------------------------------------------------------------------
# the binding: host tensors, which it refuses last, so that every other check is seen here
# ----------------------------------------------------------------------------
def refused(match, name, *args):
    with pytest.raises(ValueError, match=match):
        getattr(L.binding(), name)(*args, -1, 0)


def f8(*shape):
    import torch
    return torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e4m3fn)


def test_binding_refuses_rows():
    import torch
    x, q, s = torch.zeros(4, 200), f8(4, 256), torch.zeros(2, 4).t()

    def f(match, x=x, q=q, s=s, block_rows=1):
        refused(match, "dc_quantize_f8", x, q, s, block_rows)

    f("on a GPU")
    f("on a GPU", s=torch.zeros(4, 2))
    f("on a GPU", s=torch.zeros(12, 9)[::3, ::5])
    f("on a GPU", x=x.bfloat16()[:, 1:], q=f8(4, 300)[:, 8:])
    f("on a GPU", s=torch.zeros(1, 2), block_rows=128)
    f("on a GPU", x=x[:1], q=q[:1], s=torch.zeros(1, 1).expand(1, 2).contiguous())
    f("on a GPU", x=x[:1], q=q[:1], s=torch.zeros(8).as_strided((1, 2), (0, 1)))
    for bad in (q[:, :128], q[:3], q.view(torch.uint8), q.float(), q.view(torch.uint8).view(torch.float8_e5m2), f8(256, 4).t()):
        f("codes: ", q=bad)
    for bad in (torch.zeros(200, 4).t(), x[:1].expand(4, 200), x[0], x[:, ::2]):
        f("x: ", x=bad)
    for bad in (torch.zeros(4, 2).double(), torch.zeros(4), torch.zeros(2, 4), torch.zeros(4, 1).expand(4, 2), torch.zeros(1, 2).expand(4, 2),
                torch.zeros(9).as_strided((4, 2), (2, 1)).expand(4, 2)[:, :1].expand(4, 2), torch.zeros(9).as_strided((4, 2), (1, 3))):
        f("scale: ", s=bad)
    f("scale: ", block_rows=128)
    f("block_rows", block_rows=2)
    f("bfloat16", x=x.half())
    f("tensor", q=None)
    refused("arguments", "dc_quantize_f8", x, q, s)


def test_binding_refuses_norms():
    import torch
    n, x, q, s, w = None, torch.zeros(4, 200), f8(4, 256), torch.zeros(4, 2), torch.zeros(200)

    def f(match, x=x, q=q, s=s, weight=n, eps=1e-6, residual=n, out=n):
        refused(match, "dc_rms_norm_f8", x, q, s, weight, eps, residual, out)

    other = torch.zeros(4, 200)
    f("on a GPU")
    f("on a GPU", weight=w, residual=other.bfloat16(), out=x)
    f("on a GPU", residual=other, out=other)
    f("on a GPU", residual=x, out=x)
    f("on a GPU", x=torch.zeros(4, 300)[:, 100:], residual=torch.zeros(4, 201)[:, 1:], out=other.bfloat16())
    f("weight", weight=w[:100])
    f("weight", weight=w.bfloat16())
    f("one shape", residual=other[:, :100])
    f("one shape", out=other[:3])
    f("one shape", out=torch.zeros(200, 4).t())
    f("one shape", residual=other[:1].expand(4, 200))
    f("bfloat16", residual=other.half())
    f("bfloat16", out=other.double())
    f("scale: ", s=torch.zeros(4, 3))
    f("codes: ", q=q[:, :200])
    with pytest.raises(TypeError):
        getattr(L.binding(), "dc_rms_norm_f8")(x, q, s, n, "x", n, n, -1, 0)
    flat = torch.zeros(4 * 200 + 8)
    a, b = flat[: 800].view(4, 200), flat[8:].view(4, 200)
    f("overlap", x=a, out=b)
    f("overlap", residual=a, out=b)
    wide = torch.zeros(4, 512)
    f("on a GPU", x=wide[:, :200], out=wide[:, 200:400], residual=wide[:, 300:500].clone())
    f("overlap", x=wide[:, :200], out=wide[:, 199:399])
    bytes_ = wide.view(torch.uint8).view(torch.float8_e4m3fn)       # [4, 2048]
    f("on a GPU", x=wide[:, :200], q=bytes_[:, 800:1056])
    f("overlap", x=wide[:, :200], q=bytes_[:, 792:1048])
    f("overlap", out=wide[:, :200], q=bytes_[:, 792:1048])
    f("overlap", residual=wide[:, :200], q=bytes_[:, 792:1048])
    f("overlap", x=wide[:, :200], s=wide[:, 199:201])
    f("overlap", weight=wide.view(-1)[:200], s=wide[:, 100:102])
    f("overlap", weight=wide.view(-1)[:200], out=wide[:, 150:350])
    f("overlap", weight=wide.view(-1)[:200], q=bytes_[:, 600:856])
    f("overlap", q=bytes_[:, :256], s=wide[:, 60:62])


def test_binding_refuses_products():
    import torch
    n, x, w, out = None, f8(4, 256), f8(200, 256), torch.zeros(4, 200)
    xs, ws, v = torch.zeros(4, 2), torch.zeros(2, 2), torch.zeros(200)

    def f(match, x=x, xs=xs, w=w, ws=ws, out=out, bias=n, gelu=False, gate=n, residual=n):
        refused(match, "dc_linear_f8", x, xs, w, ws, out, bias, gelu, gate, residual)

    f("on a GPU")
    f("on a GPU", bias=v, gate=v, residual=out)
    f("on a GPU", residual=out)
    f("on a GPU", out=out.bfloat16(), residual=torch.zeros(4, 201).bfloat16()[:, 1:])
    f("on a GPU", xs=torch.zeros(1, 1).expand(4, 2), ws=torch.zeros(2, 1).expand(2, 2))
    f("on a GPU", x=f8(4, 300)[:, 16:272], w=f8(200, 512)[:, :256])
    f("whole blocks", w=w[:, :128])
    f("whole blocks", x=x[:, :200], w=w[:, :200])
    f("whole blocks", x=x.view(torch.uint8))
    f("whole blocks", w=w.view(torch.uint8).view(torch.float8_e5m2))
    f("rows of x, rows of w", out=out[:, :7])
    f("rows of x, rows of w", out=out[:3])
    f("contiguous rows", out=torch.zeros(200, 4).t())
    f("contiguous rows", residual=out[:1].expand(4, 200))
    f("contiguous rows", x=x[:1].expand(4, 256))
    f("x_scale", xs=xs[:3])
    f("x_scale", xs=torch.zeros(2, 4))
    f("x_scale", xs=xs.double())
    f("w_scale", ws=torch.zeros(200, 2))
    f("w_scale", ws=torch.zeros(2, 2).bfloat16())
    f("bias", bias=v[:5])
    f("gate", gate=v.double(), residual=out)
    f("residual", residual=out.bfloat16())
    f("residual", residual=out[:, :7])
    f("bfloat16", out=out.half())
    f("tensor", xs=n)
    wide = torch.zeros(4, 600)
    f("on a GPU", out=wide[:, :200], residual=wide[:, 200:400])
    f("on a GPU", out=wide[:, :200], residual=wide[:, :200])
    f("overlap", out=wide[:, :200], residual=wide[:, 100:300])
    f("overlap", out=wide[:, :200], xs=wide[:, 150:152])
    f("overlap", out=wide[:, :200], ws=wide[:2, 150:152])
    f("overlap", out=wide[:, :200], bias=wide.view(-1)[:200])
    f("overlap", out=wide[:, :200], gate=wide.view(-1)[100:300], residual=out)
    bytes_ = wide.view(torch.uint8).view(torch.float8_e4m3fn)
    f("overlap", out=wide[:, :200], x=bytes_[:, 784:1040])
    f("on a GPU", out=wide[:, :200], x=bytes_[:, 800:1056])


def test_api_refuses_host_tensors():
    import torch
    from paper_2608_16354_amd import api
    x, q, s = torch.zeros(4, 100), f8(4, 128), torch.zeros(4, 1)
    for call in (lambda: api.dc_quantize_f8(x, q, s), lambda: api.dc_rms_norm_f8(x, q, s),
                 lambda: api.dc_linear_f8(q, s, f8(8, 128), torch.zeros(1, 1), torch.zeros(4, 8))):
        with pytest.raises(ValueError, match="on a GPU"):
            call()


def test_product_shapes_take_the_tiles_they_name():
    """The GPU tests' shapes are the ones the library's rule sends to each of its tiles."""
    from tests import test_gpu_f8 as G
    assert {k: G.f8_tile(*k, 256) for k in G.TILE_SHAPES} == G.TILE_SHAPES
    assert {t for k, t in G.TILE_SHAPES.items() if k[3] == "bf16"} == set(G.F8_TILES)
    assert {t for k, t in G.TILE_SHAPES.items() if k[3] == "f32"} == {*G.F8_TILES[1:12], G.F8_TILES[-1]}


def test_products_of_few_k_steps_take_the_tiles_they_name():
    """One to three k-steps: every tile that the rule picks for them, the columns' kernels (one row, two long ones) aside."""
    from tests import test_gpu_f8 as G
    assert {k: G.f8_tile(*k, 256) for k in G.FEW_STEPS} == G.FEW_STEPS
    assert {t for k, t in G.FEW_STEPS.items() if k[3] == "bf16"} == set(G.F8_TILES) - {"64x64 x 2", "32x32 x 8", "column", "column of 2"}
    assert {k[2] for k, t in G.FEW_STEPS.items() if t in ("192x256", "192x128", "128x128", "64x128", "64x64")} == {128, 256, 384}


# ----------------------------------------------------------------------------
# the definitions, by hand
# ----------------------------------------------------------------------------
def test_e4m3_by_hand():
    import torch
    v = [0, 1, 1.0625, 1.1875, -1.0625, 448, 463.9, 1000, 2.0 ** -6, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 0.75 * 2.0 ** -9]
    assert X.e4m3(v).tolist() == [0, 1, 1.0, 1.25, -1.0, 448, 448, 448, 2.0 ** -6, 2.0 ** -9, 0, 2.0 ** -8, 2.0 ** -9]
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    every = every[np.isfinite(every)]
    assert len(every) == 254 and np.array_equal(X.e4m3(every), every) and every.max() == X.E4M3_TOP
    between = np.random.default_rng(0).uniform(-448, 448, 20000) * 2.0 ** -np.random.default_rng(1).integers(0, 18, 20000)
    nearest = np.abs(between[:, None] - every[None]).min(1)
    assert np.array_equal(np.abs(X.e4m3(between) - between), nearest)


def test_blocks_by_hand():
    x = np.zeros((3, 130), np.float32)
    x[0, :2] = 448, 1.0625
    x[0, 128] = 7
    x[1, 129] = np.nan
    q, s = X.e4m3_blocks(x)
    assert q.shape == (3, 256) and s.tolist()[0] == [1.0, 7 / 448] and s[2].tolist() == [0, 0]
    assert q[0, :3].tolist() == [448, 1.0, 0] and q[0, 128] == 448 and np.isnan(s[1, 1]) and not q[1:].any()
    q, s = X.e4m3_blocks(x[[0, 2]], 128)
    assert s.shape == (1, 2) and np.array_equal(X.e4m3_values(q, s, 128)[0, [0, 128]], [448.0, 7.0])


def test_products_by_hand():
    x, w = np.ones((2, 256)), np.ones((3, 256))
    w[1, 128:] = -1
    y, size = X.linear_f8(x, [[1, 2], [0.5, 0.25]], w, [[1, 3]], bias=[0, 1, 2], residual=np.ones((2, 3)), gate=[1, 2, 1])
    assert y.tolist() == [[1 + 128 * 7, 1 + 2 * (1 - 128 * 5), 1 + 2 + 128 * 7], [1 + 160, 1 + 2 * (1 - 32), 3 + 160]]
    assert size.tolist() == [[896] * 3, [160] * 3]
    assert np.allclose(X.rms_norm([[3.0, 4.0]], [1, 2], 0.0), [[3 / math.sqrt(12.5), 8 / math.sqrt(12.5)]])
