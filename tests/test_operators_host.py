"""The rotary, int8 and quantised-cache entry points refuse bad arguments on the host: every call below
ends before any device work (the pointers are never dereferenced), and the definitions they are tested
against hold on small cases worked out by hand."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import ext as X
from paper_2608_16354_amd import _lib as L

FAKE = 0x100000
ARG, SHAPE, DTYPE, WS = L.DC_ERR_ARG, L.DC_ERR_SHAPE, L.DC_ERR_DTYPE, L.DC_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    return L.load()


def cfg(dtype=1, heads=4, head_dim=64, lat=(4, 16, 16), n_txt=16):
    d = heads * head_dim
    return L.ModelCfg(2, d, heads, head_dim, 4 * d, 16, *lat, 2, n_txt, dtype, 1e-6)


def idx(*v):
    return (C.c_int32 * max(len(v), 1))(*v), len(v)


def axes(dim=(16, 24, 24), theta=1e4, start=(0.0, 0.0, 0.0), step=(1.0, 1.0, 1.0)):
    return L.RopeAxes((C.c_int32 * 3)(*dim), theta, (C.c_double * 3)(*start), (C.c_double * 3)(*step))


@pytest.mark.parametrize("bad", [dict(dim=(16, 24, 26)), dict(dim=(15, 24, 24)), dict(dim=(-2, 24, 24)),
                                 dict(theta=0.0), dict(theta=math.nan), dict(theta=math.inf),
                                 dict(start=(math.nan, 0, 0)), dict(step=(0, math.inf, 0))])
def test_rope_table_refuses_axes(lib, bad):
    c = cfg()
    assert lib.dc_rope_table(C.byref(c), C.byref(axes(**bad)), None, FAKE, None) == ARG


def test_rope_table_refuses_pointers(lib):
    c, a = cfg(), axes()
    assert lib.dc_rope_table(C.byref(c), None, None, FAKE, None) == ARG
    assert lib.dc_rope_table(C.byref(c), C.byref(a), None, None, None) == ARG
    assert lib.dc_rope_table(C.byref(c), C.byref(a), None, FAKE + 8, None) == ARG
    assert lib.dc_rope_table(C.byref(c), C.byref(a), FAKE + 4, FAKE, None) == ARG
    assert lib.dc_rope_table(None, C.byref(a), None, FAKE, None) == ARG


def qk(q=FAKE, k=FAKE, eps=1e-6, table=FAKE, interleaved=1):
    return L.QkCfg(q, k, eps, table, interleaved)


@pytest.mark.parametrize("case", [
    dict(qk=qk(eps=0.0)), dict(qk=qk(eps=math.nan)), dict(qk=qk(interleaved=2)), dict(qk=qk(table=FAKE + 8)), dict(qk=qk(q=FAKE + 4)), dict(qk=qk(k=FAKE + 8)),
    dict(ld_in=504), dict(ld_out=504), dict(ld_in=516), dict(ld_out=517), dict(src=FAKE + 8), dict(dst=FAKE + 8),
    dict(src=None), dict(dst=None), dict(dst=FAKE, ld_out=768), dict(idx=(1, 1)), dict(idx=(-1,)), dict(idx=(64,))])
def test_qk_norm_rope_refuses(lib, case):
    c = cfg()
    a = dict(qk=qk(), src=FAKE, ld_in=512, dst=2 * FAKE, ld_out=512, idx=(0,))
    a.update(case)
    arr, n = idx(*a["idx"])
    assert lib.dc_qk_norm_rope(C.byref(c), C.byref(a["qk"]), a["src"], a["ld_in"], a["dst"], a["ld_out"], 1.0, arr, n,
                               None) == ARG


@pytest.mark.parametrize("more", [dict(lat=(4, -16, 16)), dict(lat=(4, 16, -16)), dict(lat=(1, -16, -16)),
                                  dict(lat=(1 << 16, 1 << 16, 1 << 16)), dict(n_txt=2**31 - 1)])
def test_token_counts_outside_32_bits_are_refused(lib, more):
    c = cfg(**more)
    arr, n = idx(0)
    assert lib.dc_rope_table(C.byref(c), C.byref(axes()), None, FAKE, None) == SHAPE
    assert lib.dc_qk_norm_rope(C.byref(c), C.byref(qk()), FAKE, 512, FAKE, 512, 1.0, arr, n, None) == SHAPE
    assert lib.dc_cache_apply_q(C.byref(c), 8, FAKE, FAKE, FAKE, FAKE, arr, n, None) == SHAPE
    assert lib.dc_block_ext_workspace_bytes(C.byref(c), 1) == 0


def test_qk_norm_rope_of_no_samples_is_a_no_op(lib):
    arr, n = idx()
    assert lib.dc_qk_norm_rope(C.byref(cfg()), C.byref(qk()), FAKE, 512, FAKE, 512, 1.0, arr, n, None) == L.DC_OK


@pytest.mark.parametrize("args,code", [
    ((FAKE, 2, 64, 4, 64, FAKE, 128, FAKE), DTYPE), ((FAKE, 1, 63, 4, 64, FAKE, 128, FAKE), ARG),
    ((FAKE, 1, 64, 4, 64, FAKE, 127, FAKE), ARG), ((FAKE, 1, 129, 4, 129, FAKE, 255, FAKE), ARG),
    ((FAKE, 1, 64, -1, 64, FAKE, 128, FAKE), ARG), ((FAKE, 1, 64, 1 << 24, 64, FAKE, 128, FAKE), ARG),
    ((FAKE, 1, 64, 4, 0, FAKE, 128, FAKE), ARG), ((FAKE, 1, 1 << 24, 4, 1 << 24, FAKE, 1 << 24, FAKE), ARG),
    ((FAKE, 0, 2**31 - 1, 1, 2**31 - 1, FAKE, 1 << 31, FAKE), ARG), ((None, 1, 64, 4, 64, FAKE, 128, FAKE), ARG),
    ((FAKE, 1, 64, 4, 64, None, 128, FAKE), ARG), ((FAKE, 1, 64, 4, 64, FAKE, 128, None), ARG),
    ((FAKE + 1, 1, 64, 4, 64, FAKE, 128, FAKE), ARG), ((FAKE + 2, 0, 64, 4, 64, FAKE, 128, FAKE), ARG),
    ((FAKE, 0, 64, 4, 64, FAKE, 128, FAKE + 2), ARG), ((None, 0, 64, 0, 64, None, 128, None), L.DC_OK)])
def test_quantize_rows_refuses(lib, args, code):
    assert lib.dc_quantize_rows(*args, None) == code


def linear(**more):
    a = dict(rows=4, out_features=32, in_features=128, x=FAKE, x_scale=FAKE, ld_x=128, w=FAKE, w_scale=FAKE, ld_w=128,
             bias=FAKE, gelu=0, gate=None, residual=None, ld_residual=0, out=FAKE, out_dtype=0, ld_out=32)
    a.update(more)
    return L.LinearI8Args(**a)


GATED = dict(gate=FAKE, residual=FAKE, ld_residual=32, out=2 * FAKE)


@pytest.mark.parametrize("more,code", [
    (dict(out_dtype=2), DTYPE), (dict(rows=-1), ARG), (dict(out_features=0), ARG), (dict(gelu=2), ARG),
    (dict(gate=FAKE), ARG), (dict(residual=FAKE), ARG), (dict(GATED, gelu=1), ARG), (dict(GATED, out_dtype=1), ARG),
    (dict(GATED, ld_residual=31), ARG), (dict(GATED, out=FAKE, ld_out=64), ARG), (dict(ld_out=31), ARG),
    (dict(x=None), ARG), (dict(x_scale=None), ARG), (dict(w=None), ARG), (dict(w_scale=None), ARG), (dict(out=None), ARG),
    (dict(x=FAKE + 8), ARG), (dict(w=FAKE + 8), ARG), (dict(in_features=64), SHAPE), (dict(in_features=192), SHAPE),
    (dict(in_features=131072, ld_x=131072, ld_w=131072), SHAPE), (dict(ld_x=120), SHAPE), (dict(ld_w=136), SHAPE),
    (dict(ld_x=(1 << 22) + 16), SHAPE), (dict(rows=(1 << 24) - 1, out_features=1 << 20, ld_out=1 << 20), SHAPE),
    (dict(rows=1 << 24), ARG), (dict(out_features=1 << 24, ld_out=1 << 24), ARG), (dict(out=FAKE + 2), ARG),
    (dict(out=FAKE + 1, out_dtype=1), ARG), (dict(x_scale=FAKE + 2), ARG), (dict(w_scale=FAKE + 1), ARG),
    (dict(bias=FAKE + 2), ARG), (dict(GATED, gate=FAKE + 2), ARG), (dict(GATED, residual=FAKE + 3), ARG),
    (dict(rows=0, x=None, out=None), L.DC_OK)])
def test_linear_i8_refuses(lib, more, code):
    a = linear(**more)
    assert lib.dc_linear_i8(C.byref(a), None) == code


def test_linear_i8_refuses_null(lib):
    assert lib.dc_linear_i8(None, None) == ARG


@pytest.mark.parametrize("f", ["dc_cache_store_q", "dc_cache_apply_q"])
def test_quantised_cache_refuses(lib, f):
    call, c = getattr(lib, f), cfg()
    arr, n = idx(0)
    for bits in (0, 2, 16, -8):
        assert call(C.byref(c), bits, FAKE, FAKE, FAKE, FAKE, arr, n, None) == ARG
    for hole in range(4):
        p = [FAKE] * 4
        p[hole] = None
        assert call(C.byref(c), 8, *p, arr, n, None) == ARG
        p[hole] = FAKE + 8
        assert call(C.byref(c), 4, *p, arr, n, None) == ARG
    arr, n = idx(2, 2)
    assert call(C.byref(c), 8, FAKE, FAKE, FAKE, FAKE, arr, n, None) == ARG
    arr, n = idx()
    assert call(C.byref(c), 8, FAKE, FAKE, FAKE, FAKE, arr, n, None) == L.DC_OK


def test_block_ext_refuses(lib):
    arr, n = idx(0)

    def call(c, qk_cfg=None, i8=None, w=None, ws=FAKE, nbytes=None):
        e = L.BlockExt()
        if qk_cfg is not None:
            e.qk = C.pointer(qk_cfg)
        if i8 is not None:
            e.i8 = C.pointer(i8)
        nbytes = lib.dc_block_ext_workspace_bytes(C.byref(c), 1) if nbytes is None else nbytes
        return lib.dc_block_forward_ext(C.byref(c), C.byref(w or L.BlockWeights(*[FAKE] * 9)), C.byref(e), FAKE, FAKE, arr,
                                        n, ws, nbytes, None)

    c = cfg()
    plain = lib.dc_workspace_bytes(C.byref(c), 1)
    assert lib.dc_block_ext_workspace_bytes(C.byref(c), 1) >= plain + 272 * 1024 + 272 * 4
    assert lib.dc_block_ext_workspace_bytes(C.byref(c), 0) == 0
    i8 = L.BlockWeightsI8(*[FAKE] * 8)
    assert call(c, qk_cfg=qk(), nbytes=plain) == WS
    assert call(c, i8=i8, nbytes=plain) == WS
    assert call(c, i8=i8, ws=None) == WS
    assert call(c, qk_cfg=qk(eps=-1.0)) == ARG
    for hole in range(8):
        p = [FAKE] * 8
        p[hole] = None
        assert call(c, i8=L.BlockWeightsI8(*p)) == ARG
    assert call(c, i8=L.BlockWeightsI8(*[FAKE + 8] * 8)) == ARG
    for off in range(1, 8, 2):
        p = [FAKE] * 8
        p[off] = FAKE + 2
        assert call(c, i8=L.BlockWeightsI8(*p)) == ARG
    assert call(cfg(dtype=0), i8=i8) == DTYPE
    # int8 products do not read the matrices of the model dtype, but need its biases
    no_bias = L.BlockWeights(None, None, None, FAKE, None, FAKE, None, FAKE, None)
    assert call(c, i8=i8, w=no_bias) == ARG
    no_matrix = L.BlockWeights(None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None)
    assert call(c, qk_cfg=qk(), w=no_matrix) == ARG


@pytest.mark.parametrize("f,lat,n_txt,int8", [
    (131072, (4, 16, 16), 16, True),            # the down product's K
    (65536, (64, 512, 512), 0, True),           # 4,194,304 tokens: the up product's outputs
    (1 << 20, (4, 128, 128), 0, False),         # bf16: the down product's operand of 2^34 values
])
def test_block_refuses_its_products_before_it_starts(lib, f, lat, n_txt, int8):
    """A block that one of its products cannot run is refused before h is written."""
    c = cfg(lat=lat, n_txt=n_txt)
    c.mlp_hidden = f
    arr, n = idx(0)
    i8 = L.BlockWeightsI8(*[FAKE] * 8)
    e = L.BlockExt(None, C.pointer(i8) if int8 else None)
    blk = L.BlockWeights(*[FAKE] * 9)
    nbytes = lib.dc_block_ext_workspace_bytes(C.byref(c), 1)
    assert nbytes
    assert lib.dc_block_forward_ext(C.byref(c), C.byref(blk), C.byref(e), FAKE, FAKE, arr, n, FAKE, nbytes, None) == SHAPE
    if not int8:
        assert lib.dc_block_forward(C.byref(c), C.byref(blk), FAKE, FAKE, arr, n, FAKE, nbytes, None) == SHAPE


def test_a_text_only_model_has_empty_tables_and_caches(lib):
    """Without video tokens the table, codes and scales are empty: their (NULL) addresses are not read."""
    c = cfg(lat=(4, 0, 16))
    arr, n = idx(0)
    assert lib.dc_rope_table(C.byref(c), C.byref(axes()), None, None, None) == L.DC_OK
    assert lib.dc_cache_store_q(C.byref(c), 8, FAKE, FAKE, None, None, arr, n, None) == L.DC_OK
    assert lib.dc_cache_apply_q(C.byref(c), 4, FAKE, None, None, FAKE, arr, n, None) == L.DC_OK
    assert lib.dc_cache_apply_q(C.byref(c), 4, None, None, None, FAKE, arr, n, None) == ARG


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("hole", ["w_pe", "b_pe", "pos"])
def test_patch_embedding_refuses_a_missing_table(lib, dtype, hole):
    """A rotary model has no additive position table: a NULL one is refused, not read."""
    c = cfg(dtype=dtype)
    w = L.ModelWeights()
    for name in ("w_pe", "b_pe", "pos"):
        setattr(w, name, None if name == hole else FAKE)
    nbytes = lib.dc_workspace_bytes(C.byref(c), 1)
    for samples, code in (((0,), ARG), ((), L.DC_OK)):
        arr, n = idx(*samples)
        assert lib.dc_patch_embed(C.byref(c), C.byref(w), FAKE, FAKE, FAKE, arr, n, FAKE, nbytes, None) == code


def test_sampler_ext_refuses(lib):
    from paper_2608_16354_amd import api
    from paper_2608_16354_amd import inputs as I
    w = I.WORKLOADS["dit-tiny-f32"]
    c = api.model_cfg(w.model)
    blocks = (L.BlockWeights * w.model.n_blocks)()
    weights = L.ModelWeights()
    weights.blocks = C.cast(blocks, C.POINTER(L.BlockWeights))
    sig = np.ascontiguousarray(I.sigmas(w.K))
    cp = api._CProblem(I.scene_problem(w, w.motions[0]))

    def create(x, nbytes):
        bufs = L.Buffers(*[FAKE] * 9, nbytes)
        h = C.c_void_p()
        rc = lib.dc_sampler_create_ext(C.byref(c), C.byref(weights), 1, C.byref(cp.c),
                                       sig.ctypes.data_as(C.POINTER(C.c_double)), C.byref(bufs), None, C.byref(x), None,
                                       C.byref(h))
        assert not h.value
        return rc

    plain, full = lib.dc_workspace_bytes(C.byref(c), 1), lib.dc_block_ext_workspace_bytes(C.byref(c), 1)
    ext = (L.BlockExt * 2)()
    assert create(L.SamplerExt(None, None, 5, FAKE), full) == ARG
    assert create(L.SamplerExt(None, None, 8, None), full) == ARG
    assert create(L.SamplerExt(None, None, 4, FAKE + 8), full) == ARG
    assert create(L.SamplerExt(ext, None, 0, None), plain) == WS
    assert create(L.SamplerExt(None, ext, 0, None), full) == ARG       # no low expert
    bad = qk(eps=0.0)
    ext[1].qk = C.pointer(bad)
    assert create(L.SamplerExt(ext, None, 0, None), full) == ARG
    i8 = L.BlockWeightsI8(*[FAKE] * 8)
    ext[1] = L.BlockExt(None, C.pointer(i8))
    assert create(L.SamplerExt(ext, None, 0, None), full) == DTYPE     # an fp32 model


# ----------------------------------------------------------------------------
# the binding: host tensors, which it refuses last, so that every other check is seen here
# ----------------------------------------------------------------------------
def refused(match, name, *args):
    with pytest.raises(ValueError, match=match):
        getattr(L.binding(), name)(*args, -1, 0)


def test_binding_refuses_rows():
    import torch
    x, q, s = torch.zeros(4, 100), torch.zeros(4, 128, dtype=torch.int8), torch.zeros(4)
    f = "dc_quantize_rows"
    refused("on a GPU", f, x, q, s)
    refused("on a GPU", f, x[:, 1:], q, s)
    refused("on a GPU", f, x.bfloat16()[:1], q[:1], s[:1])
    for bad in (q[:, :64], q[:3], q.float(), q.to(torch.uint8)):
        refused("q: ", f, x, bad, s)
    for bad in (x.t(), x[:1].expand(4, 100), x[0], x[:, ::2]):
        refused("x: ", f, bad, q, s)
    for bad in (s.double(), torch.zeros(5), torch.zeros(8)[::2], torch.zeros(4, 1)):
        refused("scale: ", f, x, q, bad)
    refused("bfloat16", f, x.half(), q, s)
    refused("tensor", f, x, q, None)
    refused("tensor", f, [1.0], q, s)
    refused("arguments", f, x, q)


def test_binding_refuses_products():
    import torch
    q, s = torch.zeros(4, 128, dtype=torch.int8), torch.zeros(4)
    w, ws, out, n = torch.zeros(8, 128, dtype=torch.int8), torch.zeros(8), torch.zeros(4, 8), None

    def f(match, x=q, xs=s, w=w, ws=ws, out=out, bias=n, gelu=False, gate=n, residual=n):
        refused(match, "dc_linear_i8", x, xs, w, ws, out, bias, gelu, gate, residual)

    f("on a GPU")
    f("on a GPU", bias=ws, gate=ws, residual=out)
    f("on a GPU", out=torch.zeros(4, 12)[:, 3:11])
    f("equally long", w=w[:, :64])
    f("equally long", x=q.to(torch.uint8))
    f("rows of x, rows of w", out=out[:, :7])
    f("rows of x, rows of w", out=out[:3])
    f("contiguous rows", out=torch.zeros(8, 4).t())
    f("contiguous rows", residual=out[:1].expand(4, 8), gate=ws)
    f("x_scale", xs=ws)
    f("w_scale", ws=s)
    f("bias", bias=s)
    f("gate", gate=ws.double(), residual=out)
    f("residual", gate=ws, residual=out[:, :7])
    f("residual", gate=ws, residual=out.bfloat16())
    f("bfloat16", out=out.half())
    f("tensor", xs=None)


def test_binding_refuses_caches():
    import torch
    c = cfg()
    h, k8, sc = torch.zeros(2, 272, 256), torch.zeros(2, 256, 256, dtype=torch.int8), torch.zeros(2, 256, 4)
    k4 = torch.zeros(2, 256, 128, dtype=torch.uint8)
    for f in ("dc_cache_store_q", "dc_cache_apply_q"):
        refused("on a GPU", f, c, 8, h, h, k8, sc, [0, 1])
        refused("on a GPU", f, c, 4, h, h, k4, sc, np.array([1]))
        refused("on a GPU", f, c, 4, h, h, k4, sc, ())
        for idx_ in ([2], [-1], [0, 1, 2], list(range(65)), [0.5], "x", 3):
            with pytest.raises((ValueError, TypeError)):
                getattr(L.binding(), f)(c, 8, h, h, k8, sc, idx_, -1, 0)
        for bits, codes in ((4, k8), (8, k4), (8, k8.to(torch.uint8)), (8, k8[:, :255]), (8, k8[:, :, :255]), (8, k8[0])):
            refused("codes: ", f, c, bits, h, h, codes, sc, [0])
        for bad in (sc[:, :, :3], sc.double(), sc.transpose(1, 2)):
            refused("scales: ", f, c, 8, h, h, k8, bad, [0])
        for bad in (h[:, :271], h.bfloat16(), h[:, :, :255], h.transpose(0, 1)):
            refused("h_in", f, c, 8, bad, h, k8, sc, [0])
            refused("h_in", f, c, 8, h, bad, k8, sc, [0])
        refused("bits", f, c, 6, h, h, k8, sc, [0])
        refused("cfg", f, axes(), 8, h, h, k8, sc, [0])
        refused("patch", f, L.ModelCfg(2, 256, 4, 64, 1024, 16, 4, 16, 16, 0, 16, 0, 1e-6), 8, h, h, k8, sc, [0])
        # batches of different sizes: the smallest counts
        refused("idx", f, c, 8, h, h, k8[:1], sc, [1])
        refused("idx", f, c, 8, h, h[:1], k8, sc, [1])


def test_binding_refuses_norms_and_tables():
    import torch
    c = cfg()
    b = torch.zeros(2, 272, 768, dtype=torch.bfloat16)
    o, wt, t = torch.zeros(2, 272, 512, dtype=torch.bfloat16), torch.zeros(64), torch.zeros(256, 32, 2)

    def f(match, x=b, out=o, idx_=(0, 1), wq=wt, wk=wt, table=t):
        refused(match, "dc_qk_norm_rope", c, x, out, idx_, wq, wk, 1e-6, table, True, 1.0)

    f("on a GPU")
    f("on a GPU", wq=None, wk=None, table=None)
    f("on a GPU", x=b[:1], idx_=[0])
    for bad in (b.float(), b[:, :, :500], b[:, :271], b[0], b[:, :, ::2][:, :, :384], b[:, :1].expand(2, 272, 768)):
        f("x and out", x=bad)
        f("x and out", out=bad)
    f("idx", out=o[:1])
    f("q_weight", wq=torch.zeros(63))
    f("k_weight", wk=wt.double())
    for bad in (t[:255], t[:, :31], t.double(), t[..., :1]):
        f("table", table=bad)
        refused("table", "dc_rope_table", c, axes(), None, bad)
    refused("on a GPU", "dc_rope_table", c, axes(), None, t)
    refused("on a GPU", "dc_rope_table", c, axes(), torch.zeros(256, 3, dtype=torch.float64), t)
    for bad in (torch.zeros(256, 3), torch.zeros(255, 3, dtype=torch.float64), torch.zeros(3, 256, dtype=torch.float64).t()):
        refused("pos", "dc_rope_table", c, axes(), bad, t)
    refused("axes", "dc_rope_table", c, c, None, t)
    refused("tensor", "dc_rope_table", c, axes(), None, None)


def test_binding_takes_single_tokens_of_any_stride():
    """A model of one token: its rows are the samples, a dimension of one has no stride of its own."""
    import torch
    c = cfg(lat=(1, 2, 2), n_txt=0)
    buf, out = torch.zeros(3, 5, 768, dtype=torch.bfloat16), torch.zeros(3, 1, 512, dtype=torch.bfloat16)

    def f(match, x, out, idx_):
        refused(match, "dc_qk_norm_rope", c, x, out, idx_, None, None, 1e-6, None, True, 1.0)

    for st in (0, 3, 512, 768):
        one = buf.as_strided((1, 1, 768), (7, st, 1))
        f("on a GPU", one, out[:1], [0])
        f("on a GPU", out[:1], one, [0])
        f("on a GPU", buf.as_strided((3, 1, 768), (3840, st, 1)), out, [0, 2])
    f("on a GPU", buf[:, 2:3], out, [1])
    f("x and out", buf.as_strided((3, 1, 768), (504, 768, 1)), out, [0])            # samples that overlap
    f("x and out", buf[:1, :1].expand(3, 1, 768), out, [0])


def test_binding_refuses_a_list_that_shrinks_under_it():
    """An index that takes the list apart while it is read: nothing is read behind the list's end."""
    import torch
    c, samples = cfg(), []
    h, codes, scales = torch.zeros(2, 272, 256), torch.zeros(2, 256, 256, dtype=torch.int8), torch.zeros(2, 256, 4)

    class Index:
        def __index__(self):
            samples.clear()
            return 0

    samples += [Index(), 1, 1]
    refused("idx", "dc_cache_apply_q", c, 8, h, h, codes, scales, samples)


def test_binding_refuses_overlaps():
    """What is written overlaps nothing that is read, but for the places that may be the same: other columns of a
    buffer's rows, or other rows, are taken."""
    import torch
    c, n = cfg(), None
    buf = torch.zeros(2, 272, 1024, dtype=torch.bfloat16)

    def qk_(match, x, out):
        refused(match, "dc_qk_norm_rope", c, x, out, [0], n, n, 1e-6, n, True, 1.0)

    qk_("on a GPU", buf[..., :512], buf[..., :512])             # in place
    qk_("on a GPU", buf[..., :512], buf[..., 512:])
    qk_("on a GPU", buf[..., 512:], buf[..., :512])
    qk_("on a GPU", buf[:1], buf[1:])
    qk_("on a GPU", buf[1:], buf[:1])
    qk_("overlap", buf[..., :512], buf[..., 8:520])
    qk_("overlap", buf[..., 256:768], buf[..., :512])
    qk_("on a GPU", buf, buf[..., 512:])                        # 512 of x's columns are read
    qk_("overlap", buf, buf[..., 504:])
    flat = buf.view(-1)
    rows_ = flat[: 272 * 512].view(1, 272, 512)
    qk_("overlap", buf[:1, :, :512], rows_)                     # rows of another length in the same place
    qk_("overlap", flat[8: 8 + 272 * 512].view(1, 272, 512), rows_)
    qk_("on a GPU", flat[272 * 512: 2 * 272 * 512].view(1, 272, 512), rows_)

    def quant(match, x, q, s):
        refused(match, "dc_quantize_rows", x, q, s)

    raw = torch.zeros(4, 1024, dtype=torch.int8)
    s = torch.zeros(4)
    floats = raw.view(torch.float32)                            # [4, 256]
    quant("on a GPU", floats[:, 128:], raw[:, :128], s)
    quant("on a GPU", floats[:, 32:132], raw, s)                # the 128 columns that are written lie before x
    quant("overlap", floats[:, 31:131], raw, s)
    quant("overlap", floats, raw, s)
    quant("overlap", floats[:2], raw.view(8, 512)[2:4], s[:2])
    quant("on a GPU", floats[:2], raw[2:], s[:2])
    quant("on a GPU", floats[:1, :8], raw[0, 128:].unsqueeze(0)[:, :128], s[:1])
    quant("overlap", floats, torch.zeros(4, 256, dtype=torch.int8), floats[0, :4])

    x, w = torch.zeros(4, 128, dtype=torch.int8), torch.zeros(8, 128, dtype=torch.int8)
    out, ws, wide = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4, 20)

    def lin(match, x=x, xs=s, w=w, ws=ws, out=out, bias=n, gate=n, residual=n):
        refused(match, "dc_linear_i8", x, xs, w, ws, out, bias, False, gate, residual)

    lin("on a GPU", out=wide[:, :8], residual=wide[:, 8:16], gate=ws)
    lin("on a GPU", out=wide[:, :8], residual=wide[:, :8], gate=ws)
    lin("overlap", out=wide[:, :8], residual=wide[:, 4:12], gate=ws)
    lin("overlap", out=wide[1:, :8], x=x[1:], xs=s[1:], residual=wide[:3, :8], gate=ws)
    for name, t in (("x", x), ("w", w)):
        lin("overlap", **{name: t, "out": t.view(torch.float32)[:4, :8]})
    vec = torch.zeros(32)
    for name in ("ws", "bias"):
        lin("overlap", out=vec.view(4, 8), **{name: vec[5:13]})
    lin("overlap", out=vec.view(4, 8), gate=vec[:8], residual=out)
    lin("overlap", out=vec.view(4, 8), xs=vec[28:])


def test_api_refuses_host_tensors():
    import torch
    from paper_2608_16354_amd import api
    with pytest.raises(ValueError, match="on a GPU"):
        api.dc_quantize_rows(torch.zeros(4, 100), torch.zeros(4, 128, dtype=torch.int8), torch.zeros(4))


def test_rope_axes_are_the_struct():
    from paper_2608_16354_amd import api
    got = api.rope_axes((16, 24, 20), 100, start=np.array([1, 2.5, -3]), step=[0.5, 4, 5])
    want = axes((16, 24, 20), 100.0, (1.0, 2.5, -3.0), (0.5, 4.0, 5.0))
    assert bytes(got) == bytes(want)
    for bad in (dict(dim=(16, 24)), dict(dim=(16, 24, 24.5)), dict(dim=(1, 2, 3), start=(0, 0)), dict(dim=(1, 2, 3), theta="x")):
        with pytest.raises(ValueError, match="three numbers"):
            api.rope_axes(**bad)


def test_extensions_belong_to_a_shape_and_a_device():
    """An extension holds tensors of its model's sizes: another model, or a tensor elsewhere, is refused."""
    import types
    import torch
    from paper_2608_16354_amd import api

    def model(**more):
        c = cfg(**more)
        return types.SimpleNamespace(cfg=c, blocks=[dict(b_qkv=torch.zeros(4))] * c.n_blocks)

    dm, w = model(), [torch.ones(64)] * 2
    e = api.BlockExt(dm, q_weight=w, k_weight=w, table=torch.zeros(256, 32, 2))
    assert e.of(dm) is e and e.of(model()) is e
    for other in (model(heads=6), model(lat=(4, 16, 18)), model(n_txt=17), model(dtype=0)):
        with pytest.raises(ValueError, match="another shape"):
            e.of(other)
        with pytest.raises(ValueError, match="another shape"):
            api.dc_block_forward_ext(other, 0, e, None, None, [0], None)
    for bad in (dict(q_weight=[torch.ones(64, device="meta")] * 2), dict(table=torch.zeros(256, 32, 2, device="meta")),
                dict(k_weight=[torch.ones(63)] * 2), dict(table=torch.zeros(255, 32, 2))):
        with pytest.raises(ValueError, match="is wanted"):
            api.BlockExt(dm, **bad)
    with pytest.raises(IndexError):
        api.BlockExt(dm, q_weight=w[:1])


def test_extensions_belong_to_their_device():
    """Equal shapes on another device: the addresses an extension holds are not that model's."""
    import types
    import torch
    from paper_2608_16354_amd import api

    def model(device):
        return types.SimpleNamespace(cfg=cfg(), blocks=[dict(b_qkv=torch.zeros(4, device=device))] * 2)

    here, elsewhere = model("cpu"), model("meta")
    e = api.BlockExt(here)
    assert e.of(model("cpu")) is e
    with pytest.raises(ValueError, match="another device"):
        e.of(elsewhere)
    with pytest.raises(ValueError, match="another device"):
        api.dc_block_forward_ext(elsewhere, 0, e, None, None, [0], None)


def test_extensions_keep_their_tensors():
    """The library holds addresses, so the tensors live as long as the extension, whatever becomes of the caller's list."""
    import gc
    import types
    import weakref
    import torch
    from paper_2608_16354_amd import api
    dm = types.SimpleNamespace(cfg=cfg(), blocks=[dict(b_qkv=torch.zeros(4))] * 2)
    wq, wk, table = [torch.ones(64) for _ in range(2)], [torch.ones(64) for _ in range(2)], torch.zeros(256, 32, 2)
    held = [weakref.ref(v) for v in (*wq, *wk, table)]
    e = api.BlockExt(dm, q_weight=wq, k_weight=wk, table=table)
    wq.clear()
    wk[:] = [None, None]
    del table
    gc.collect()
    assert all(r() is not None for r in held)
    del e
    gc.collect()
    assert all(r() is None for r in held)


def test_product_shapes_take_the_tiles_they_name():
    """The GPU tests' shapes are the ones the library's rule sends to each of its tiles."""
    from tests import test_gpu_operators as G
    assert {k: G.i8_tile(*k, 256) for k in G.TILE_SHAPES} == G.TILE_SHAPES
    assert set(G.TILE_SHAPES.values()) == set(G.I8_TILES)


def test_qkv_models_take_every_tile():
    """The models whose QKV rows are tested on the GPU take each tile that the int8 QKV product can take."""
    from tests import test_gpu_extended_step as E
    from tests import test_gpu_operators as G
    from tests.gpu_util import _native
    models = {**E.QKV_TILES, **E.QKV_WIDE}
    for tile, m in models.items():
        assert G.I8_TILES[_native("_ZN2dc7i8_tileEiiiib", m.n_tok, 3 * m.hidden, m.hidden // 128, 256, False)] == tile
    assert set(models) == {t for t in G.I8_TILES if not t.startswith("32x32")}


# ----------------------------------------------------------------------------
# the definitions, by hand
# ----------------------------------------------------------------------------
def test_codes_by_hand():
    q, s = X.codes(np.array([[127.0, -63.5, 0.4, 62.5], [0, 0, 0, 0], [1, np.nan, 0, 0], [np.inf, 1, 0, 0]]), 127)
    assert q.tolist() == [[127, -64, 0, 62], [0] * 4, [0] * 4, [0] * 4]      # ties go to the even code
    assert s[0] == 1 and s[1] == 0 and np.isnan(s[2:]).all()
    q, s = X.cache_codes(np.concatenate([np.full(64, -3.5), np.full(64, 0.5), [7.0] + [1.0] * 63])[None], 4)
    assert q[0, 0] == -7 and q[0, 64] == 7 and q[0, 128] == 7 and q[0, 129] == 1
    assert s[0].tolist() == [0.5, np.float32(0.5) / np.float32(7), 1.0]


def test_rotation_by_hand():
    t = X.rope_table(np.array([[math.pi / 2, 0.0, 0.0]]), (2, 0, 2), 100.0, 3)
    assert np.allclose(t[0], [[0, 1], [1, 0], [1, 0]])
    x = np.arange(1.0, 7.0).reshape(1, 1, 6)
    assert np.allclose(X.qk_norm_rope(x, None, 0, t, True), [[[-2, 1, 3, 4, 5, 6]]])
    assert np.allclose(X.qk_norm_rope(x, None, 0, t, False), [[[-4, 2, 3, 1, 5, 6]]])
    y = X.qk_norm_rope(np.full((1, 1, 4), 3.0), np.arange(4.0), 0.0, None, True, 2.0)
    assert np.allclose(y, [[[0, 2, 4, 6]]])
