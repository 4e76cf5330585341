"""Extended blocks and samples: rotary positions, query/key norms, int8 products and the quantised cache as
they run together.

Blocks against the float64 oracle; samples against the same public calls made one by one, bit for bit."""
import numpy as np
import pytest

from oracle import dit
from oracle import ext as X
from paper_2608_16354_amd import inputs as I
from tests.gpu_util import _native, compute_units, mod_input, rel_l2, say, t
from tests.test_gpu_kernels import _OneBlock

pytestmark = pytest.mark.gpu


def _shape(d, heads, hd, f, lat, n_txt, dtype, blocks=1):
    return I.ModelShape(blocks, d, heads, hd, f, 16, *lat, 2, n_txt, dtype)


BLOCKS = {
    "bf16-64": _shape(256, 4, 64, 1024, (3, 10, 12), 21, "bf16"),
    "bf16-72-odd": _shape(1152, 16, 72, 4608, (2, 6, 10), 7, "bf16"),
    "bf16-narrow-mlp": _shape(384, 6, 64, 128, (5, 14, 18), 13, "bf16"),
    "bf16-1556": _shape(640, 10, 64, 2560, (3, 34, 58), 77, "bf16"),
    "f32": _shape(256, 4, 64, 1024, (3, 10, 12), 5, "f32"),
}


@pytest.fixture(scope="module")
def api():
    from paper_2608_16354_amd import api as A
    A.L.load()
    return A


def qk_weights(m, key=0):
    return [(1 + I.normal((m.head_dim,), 0.2, (8000 + key, i))).astype(np.float32) for i in range(2)]


def axis_dims(m):
    a = 2 * (m.head_dim // 8)
    return a, a, m.head_dim - 2 * a


def make_table(api, m, dev):
    import torch
    table = torch.empty((m.n_v, m.head_dim // 2, 2), device=dev)
    api.dc_rope_table(api.model_cfg(m), api.rope_axes(axis_dims(m), 100.0), None, table)
    return table


@pytest.mark.parametrize("name", list(BLOCKS))
@pytest.mark.parametrize("mode", ["qk", "int8", "both"])
def test_block(api, dev, name, mode):
    import torch
    m = BLOCKS[name]
    if m.dtype == "f32" and mode != "qk":
        pytest.skip("int8 products are for bf16 models")
    W = I.Weights(m, 140)
    dm = api.DeviceModel(_OneBlock(W, 0), dev)
    ws = api.Workspace(m, 2, dev, ext=True)
    h = I.hidden_state(m, (70,))
    mod = mod_input(m, (71,))
    wq, wk = qk_weights(m)
    il = m.head_dim == 64
    table = make_table(api, m, dev)
    kw = dict(q_weight=[t(wq, dev)], k_weight=[t(wk, dev)], table=table, interleaved=il) if mode != "int8" else {}
    ext = api.BlockExt(dm, int8=mode != "qk", **kw)
    dh = torch.full((2, m.n_tok, m.hidden), 4.0, device=dev)
    dh[1] = t(h, dev)
    say("extended block", name, mode)
    api.dc_block_forward_ext(dm, 0, ext, t(mod, dev), dh, [1], ws)
    torch.cuda.synchronize()
    got = dh[1].cpu().numpy()
    assert (dh[0] == 4).all()
    qk = None
    if mode != "int8":
        grid = X.grid_positions(m.lat_t, m.hp, m.wp)
        qk = dict(q_weight=wq, k_weight=wk, eps=1e-6, interleaved=il,
                  table=X.rope_table(grid, axis_dims(m), 100.0, m.head_dim // 2))
    P, mod64, h64 = dit.Params(W), mod.astype(np.float64), h.astype(np.float64)
    want = X.block(P, 0, mod64, h64, qk=qk, int8=mode != "qk")
    err = rel_l2(got - h, want - h)
    say(name, mode, "update rel-L2", err)
    if mode == "qk":
        # fp32: 2^-24 a rounding over sums of up to 1024 terms; bf16: 2^-9 of each operand, as dc_block_forward's tests
        assert err < (2e-5 if m.dtype == "f32" else 1e-2)
        return
    # A row's codes are steps of its largest magnitude / 127: with 3 to 6 standard deviations to the largest,
    # 3 / 127 / sqrt(12) = 0.7 % to 1.4 % of a row.  Where an operand is off by bf16's 2^-9 (attention's rows, the MLP's
    # hidden ones) its codes fall on either side of a border, so two right evaluations differ by up to that noise in each
    # of two operands of two products: 2 x 1.4 %.
    assert err < 2.8e-2
    assert rel_l2(got - h, X.block(P, 0, mod64, h64, qk=qk) - h) < 4e-2        # four products' own noise


def test_block_without_extensions_is_the_block(api, dev):
    import torch
    m = BLOCKS["bf16-64"]
    dm = api.DeviceModel(_OneBlock(I.Weights(m, 140), 0), dev)
    h, mod = t(I.hidden_state(m, (70,))[None], dev), t(mod_input(m, (71,)), dev)
    a, b = h.clone(), h.clone()
    api.dc_block_forward(dm, 0, mod, a, [0], api.Workspace(m, 1, dev))
    api.dc_block_forward_ext(dm, 0, api.BlockExt(dm), mod, b, [0], api.Workspace(m, 1, dev))
    assert torch.equal(a, b)
    b.copy_(h)
    api.dc_block_forward_ext(dm, 0, None, mod, b, [0], api.Workspace(m, 1, dev))
    assert torch.equal(a, b)


def _legal(K, h_max, b):
    a = np.array([(k + b) % (h_max + 1) != 0 for k in range(K)], np.uint8)
    a[0] = 0
    return a


SAMPLES = {
    "bf16": _shape(256, 4, 64, 512, (3, 10, 12), 5, "bf16", blocks=2), "f32": _shape(256, 4, 64, 512, (3, 10, 12), 5, "f32", blocks=2),
    # the reuse head's other widths, three tiles of tokens to a workgroup, and a width whose reuse applies the cache first
    "bf16-1152": _shape(1152, 16, 72, 1152, (3, 10, 12), 5, "bf16", blocks=2), "bf16-1920": _shape(1920, 30, 64, 1920, (1, 14, 14), 5, "bf16", blocks=2),
    "bf16-long": _shape(128, 2, 64, 128, (8, 64, 78), 5, "bf16", blocks=2), "bf16-2304": _shape(2304, 36, 64, 128, (1, 6, 6), 3, "bf16", blocks=2),
}


@pytest.mark.parametrize("bits", [0, 8, 4])
@pytest.mark.parametrize("name,mode", [("bf16", "both"), ("bf16", "none"), ("f32", "qk"), ("bf16-1152", "none"), ("bf16-1920", "none"),
                                       ("bf16-long", "none"), ("bf16-2304", "none")])
def test_sample_is_its_calls(api, dev, bits, name, mode):
    """Two scenes with staggered reuses and guidance: the sampler's latent against the public calls in order."""
    import torch
    m, K, B, w = SAMPLES[name], 6, 2, 2.5
    W = I.Weights(m, 150)
    dm = api.DeviceModel(W, dev)
    ext = None
    if mode != "none":
        pairs = [qk_weights(m, l) for l in range(2)]
        ext = api.BlockExt(dm, q_weight=[t(p[0], dev) for p in pairs], k_weight=[t(p[1], dev) for p in pairs],
                           table=make_table(api, m, dev), interleaved=False, int8=mode == "both")
    wl = I.Workload(0, "s", m, B, K, 2, None, "inf", 0.5, I.NO_VETO)
    problems = [I.scene_problem(wl, I.Motion(6.0, 0.25)).replace(legal=_legal(K, 2, b)) for b in range(B)]
    x1 = torch.from_numpy(np.stack([I.latent(m, 150, b) for b in range(B)]))
    txt = torch.from_numpy(np.stack([I.text(m, 150, b) for b in range(B)]))
    null = torch.zeros_like(txt)
    sig = I.sigmas(K)
    say("extended sample", bits, name, mode)
    smp = api.Sampler(dm, problems, sig, x1, txt, guidance=(w, null), ext=ext, cache_bits=bits)
    realized, _ = smp.run()
    torch.cuda.synchronize()
    assert realized.sum() > 0 and realized.sum() < K * B

    bufs = api.SamplerBuffers(m, 2 * B, K, dev, ext=True, cache_bits=bits)       # entries B + b: the unconditional branch
    cfg, ws = dm.cfg, bufs.ws
    x = x1.to(dev)
    mod = bufs.mod
    api.dc_time_modulation(dm, sig[:K], mod, ws)
    for k in range(K):
        both = torch.cat([txt, null]).to(dev)
        xx = torch.cat([x, x])
        api.dc_patch_embed(dm, xx, both, bufs.h_in, list(range(2 * B)), ws)
        fresh = [b for b in range(B) if not realized[k, b]]
        fresh += [B + b for b in fresh]
        kept = [b for b in range(2 * B) if b not in fresh]
        for b in fresh:
            bufs.h[b].copy_(bufs.h_in[b])
        for l in range(2):
            if ext is None:
                api.dc_block_forward(dm, l, mod[k, l], bufs.h, fresh, ws)
            else:
                api.dc_block_forward_ext(dm, l, ext, mod[k, l], bufs.h, fresh, ws)
        if bits:
            api.dc_cache_store_q(cfg, bits, bufs.h, bufs.h_in, bufs.resid, bufs.cache_scales, fresh)
            api.dc_cache_apply_q(cfg, bits, bufs.h_in, bufs.resid, bufs.cache_scales, bufs.h, kept)
        else:
            api.dc_cache_store(cfg, bufs.h, bufs.h_in, bufs.resid, fresh)
            api.dc_cache_apply(cfg, bufs.h_in, bufs.resid, bufs.h, kept)
        ds = float(sig[k + 1] - sig[k])
        for b in range(B):
            v = x[b: b + 1].clone()
            api.dc_head_euler(dm, mod[k, 2], bufs.h[b: b + 1], v, np.float32(ds * w), [0], ws)
            api.dc_head_euler(dm, mod[k, 2], bufs.h[B + b: B + b + 1], v, np.float32(ds * (1.0 - w)), [0], ws)
            x[b] = v[0]
    torch.cuda.synchronize()
    got, want = smp.x.cpu().numpy(), x.cpu().numpy()
    say("sample", bits, name, mode, "max difference", np.abs(got - want).max())
    assert np.isfinite(got).all() and np.array_equal(got, want)
    smp.close()


def test_sample_of_two_experts_takes_each_ones_extensions(api, dev):
    """With a low-noise expert, its steps run ext_low: equal weights and extensions on both sides of the switch give
    the one-expert sample, other norms on the low side another one."""
    import torch
    m = _shape(256, 4, 64, 512, (2, 6, 8), 3, "f32", blocks=2)
    K = 4
    dm = api.DeviceModel(I.Weights(m, 160), dev)
    table = make_table(api, m, dev)
    ones = [torch.ones(64, device=dev)] * 2
    e1 = api.BlockExt(dm, q_weight=ones, k_weight=ones, table=table)
    e2 = api.BlockExt(dm, q_weight=[3 * o for o in ones], k_weight=ones, table=table)
    wl = I.Workload(0, "s", m, 1, K, 2, None, "inf", 0.5, I.NO_VETO)
    p = I.scene_problem(wl, I.Motion(6.0, 0.25)).replace(legal=np.zeros(K, np.uint8), segment=np.array([0, 0, 1, 1], np.int32))
    x1, txt = torch.from_numpy(I.latent(m, 160, 0)[None]), torch.from_numpy(I.text(m, 160, 0)[None])

    def run(low):
        smp = api.Sampler(dm, [p], I.sigmas(K), x1, txt, ext=e1, ext_low=low, low_expert=(dm, 3) if low else None)
        smp.run()
        x = smp.x.cpu().numpy()
        smp.close()
        return x

    say("two experts with extensions")
    one, same, other = run(None), run(e1), run(e2)
    assert np.array_equal(one, same) and not np.array_equal(one, other)


def test_two_captured_blocks_share_a_workspace(api, dev):
    """Blocks with norms, rotation and int8 products as two graphs on one workspace, replayed in turn between eager
    work, against the eager calls."""
    import torch
    m = _shape(256, 4, 64, 1024, (3, 10, 12), 21, "bf16", blocks=2)
    dm = api.DeviceModel(I.Weights(m, 170), dev)
    wq, wk = qk_weights(m)
    ext = api.BlockExt(dm, q_weight=[t(wq, dev)] * 2, k_weight=[t(wk, dev)] * 2, table=make_table(api, m, dev), int8=True)
    mod = t(mod_input(m, (72,)), dev)
    ws, ws_e = api.Workspace(m, 1, dev, ext=True), api.Workspace(m, 1, dev, ext=True)
    h, e = (torch.zeros((1, m.n_tok, m.hidden), device=dev) for _ in range(2))
    gen = torch.Generator(dev).manual_seed(5)
    graphs, stream = [], torch.cuda.Stream()
    torch.cuda.synchronize()
    for l in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[l], stream=stream):
            api.dc_block_forward_ext(dm, l, ext, mod, h, [0], ws)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        h.copy_(torch.randn(h.shape, device=dev, generator=gen))
        e.copy_(h)
        for l in order:
            graphs[l].replay()
            api.dc_block_forward_ext(dm, l, ext, mod, e, [0], ws_e)
        torch.cuda.synchronize()
        assert torch.isfinite(e).all() and torch.equal(h, e), order


QKV_TILES = {       # the int8 QKV product's tile on 256 compute units: the model that takes it
    "64x64": _shape(256, 4, 64, 128, (3, 10, 12), 21, "bf16"), "128x64": _shape(1152, 18, 64, 128, (1, 38, 40), 1, "bf16"),
    "128x128": _shape(1152, 18, 64, 128, (1, 34, 68), 1, "bf16"), "192x128": _shape(768, 12, 64, 128, (4, 28, 64), 5, "bf16"),
    "256x128": _shape(1152, 16, 72, 128, (4, 28, 64), 5, "bf16"), "256x192": _shape(1536, 24, 64, 128, (4, 28, 64), 5, "bf16"),
    "384x192": _shape(1536, 24, 64, 128, (3, 68, 58), 77, "bf16"),
}


@pytest.mark.parametrize("tile", list(QKV_TILES))
def test_int8_qkv_rows(api, dev, tile):
    """Q, K and V transposed as the block leaves them in its workspace, against the product of the codes.  The LN's fp32
    roundings move a code over a border about once in 10^4: six such codes of a row, each of at most 127 of a weight's
    steps, the two scales' roundings, and bf16's half step."""
    import torch
    from tests.test_gpu_operators import I8_TILES
    m = QKV_TILES[tile]
    N, d, ldv = m.n_tok, m.hidden, -(-m.n_tok // 64) * 64
    assert I8_TILES[_native("_ZN2dc7i8_tileEiiiib", N, 3 * d, d // 128, compute_units(dev), False)] == tile
    W = I.Weights(m, 180)
    dm = api.DeviceModel(_OneBlock(W, 0), dev)
    ext, ws = api.BlockExt(dm, int8=True), api.Workspace(m, 1, dev, ext=True)
    ws.buf.fill_(0xFF)                                       # NaN wherever nothing is written
    h, mod = I.hidden_state(m, (71,)), mod_input(m, (73,))
    say("int8 QKV", tile, N, d)
    api.dc_block_forward_ext(dm, 0, ext, t(mod, dev), t(h[None], dev), [0], ws)
    torch.cuda.synchronize()
    at = ws.ptr.value - ws.buf.data_ptr() + -(-2 * N * d // 256) * 256

    def held(rows, cols):
        nonlocal at
        v = ws.buf[at: at + 2 * rows * cols].view(torch.bfloat16).view(rows, cols).float().cpu().numpy()
        at += -(-2 * rows * cols // 256) * 256
        return v

    qk, vt = held(ldv + 64, 2 * d)[:N], held(d, ldv)
    x8, xs = X.codes(dit.modulate(h.astype(np.float64), mod[0].astype(np.float64), mod[1].astype(np.float64), m.ln_eps), 127)
    w8, wsc = X.codes(dm.blocks[0]["w_qkv"].float().cpu().numpy(), 127)
    step = xs[:, None].astype(np.float64) * wsc.astype(np.float64)
    want = (x8.astype(np.float64) @ w8.astype(np.float64).T) * step + dm.blocks[0]["b_qkv"].cpu().numpy()
    tol = 6 * 127 * step
    q_scale = 1.4426950408889634 / np.sqrt(m.head_dim)
    want[:, :d] *= q_scale
    tol[:, :d] *= q_scale
    tol += (2.0 ** -8 + 1e-5) * (np.abs(want) + tol)
    got = np.concatenate([qk, vt[:, :N].T], 1)
    err = np.abs(got - want)
    say(tile, "largest share of the tolerance", (err / tol).max())
    assert np.isfinite(got).all() and (err <= tol).all(), np.argwhere(err > tol)[:4]
    assert not vt[:, N:].any()


QKV_WIDE = {"320x256": _shape(1152, 16, 72, 128, (6, 56, 64), 77, "bf16")}       # the tile with five strips of rows to a wave


@pytest.mark.parametrize("tile", list(QKV_WIDE))
def test_int8_qkv_rows_of_wide_tiles(api, dev, monkeypatch, tile):
    monkeypatch.setitem(QKV_TILES, tile, QKV_WIDE[tile])
    test_int8_qkv_rows(api, dev, tile)
