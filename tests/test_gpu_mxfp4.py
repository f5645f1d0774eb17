"""Microscaled 4-bit operands: quantisation and its way back bit for bit, the product against 64-bit arithmetic.

The product's terms are exact (e2m1 x e2m1 x a power of two), so outputs whose every partial sum fits 24 bits have to be the
rounded exact sum, bit for bit.  Others may lose up to 2^-23 of the magnitudes per addition (the accumulator may cut instead of
rounding), and 2^-8 of themselves with the rounding to bf16; the activation's own error is far below that."""
import numpy as np
import pytest
import torch

from oracle import mxfp4
from paper_2411_00288_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _f64(t):
    return t.detach().cpu().double().numpy()


def _randn(seed, *shape):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV)


def _check_quantised(x):
    c = x.shape[-1]
    codes, scales = api.ssconv_quantize_mxfp4(x)
    back = api.ssconv_dequantize_mxfp4(codes, scales, c)
    rows = x.numel() // c
    q, e = mxfp4.quantize(_f64(x).reshape(rows, c))
    blocks = q.shape[1]
    image = scales.cpu().numpy()
    at = np.array([[mxfp4.scale_image_index(r, b, blocks) for b in range(blocks)] for r in range(rows)])
    assert (image[at].astype(np.int64) - 127 == e).all()
    others = np.ones(image.size, bool)
    others[at.ravel()] = False
    assert (image[others] == 0).all()                           # padding: a scale that is a number
    got = codes.cpu().numpy().reshape(rows, -1)
    fine = np.repeat(e != 128, 16, axis=1)                      # (what a block that is NaN holds does not matter)
    assert (got[fine] == mxfp4.code_bytes(q)[fine]).all()
    want = mxfp4.values(q, e, c)
    assert back.shape == x.shape and np.array_equal(_f64(back).reshape(rows, c), want, equal_nan=True)


@pytest.mark.parametrize("rows", [1, 2, 31, 127, 128, 129, 300])
@pytest.mark.parametrize("c", [8, 24, 32, 40, 96, 128, 136, 520])
def test_quantised_values(rows, c):
    x = _randn(rows * c, rows, c) * torch.exp(2 * _randn(c, rows, 1))
    x[:, : c // 8] *= 50
    _check_quantised(x.bfloat16())


@pytest.mark.parametrize("rows", [33, 128, 1000])
@pytest.mark.parametrize("c", [48, 56, 64, 72, 80, 88, 104])
def test_quantised_rows_of_less_than_an_image(rows, c):
    _check_quantised((_randn(rows * c, rows, c) * torch.exp(2 * _randn(c, rows, 1))).bfloat16())


def test_quantised_shapes_of_more_axes():
    x = _randn(3, 2, 5, 7, 64).bfloat16()
    codes, scales = api.ssconv_quantize_mxfp4(x)
    assert codes.shape == (2, 5, 7, 32)
    _check_quantised(x)


def test_every_bf16_value_is_rounded_to_the_nearest_code():
    # each of the 65,536 bit patterns beside a largest magnitude that makes its scale 2^0, 2^1 and 2^-3
    bits = torch.arange(65536, dtype=torch.int32, device=DEV).to(torch.int16).view(torch.bfloat16)
    for top in (4.0, 15.0, 0.5):
        x = bits.clone().view(-1, 32)
        x = torch.where(x.float().abs() <= top, x, torch.zeros_like(x))
        x[:, 0] = top
        _check_quantised(x.contiguous())


def test_extremes_and_non_numbers():
    x = torch.zeros(8, 64, dtype=torch.bfloat16, device=DEV)
    tiny = torch.tensor([1], dtype=torch.int16, device=DEV).view(torch.bfloat16)      # the smallest magnitude
    x[0, 5] = tiny
    x[1, :] = 3.3895e38
    x[2, 40] = float("inf")
    x[3, 1] = float("-inf")
    x[4, 33] = float("nan")
    x[5, 0], x[5, 1] = 1e-38, -3e-39
    x[6, :32] = -0.0
    x[7, 2], x[7, 3] = 3e38, tiny
    _check_quantised(x)


def test_no_rows():
    codes, scales = api.ssconv_quantize_mxfp4(torch.empty(0, 40, dtype=torch.bfloat16, device=DEV))
    assert codes.shape == (0, 32) and scales.numel() == 0
    assert api.ssconv_dequantize_mxfp4(codes, scales, 40).shape == (0, 40)
    with pytest.raises(api.SsconvError):
        api.ssconv_quantize_mxfp4(torch.empty(4, 0, dtype=torch.bfloat16, device=DEV))


def test_large_quantisation_in_pieces():
    rows, c = 70_001, 200
    x = _randn(9, rows, c).bfloat16()
    codes, scales = api.ssconv_quantize_mxfp4(x)
    back = api.ssconv_dequantize_mxfp4(codes, scales, c)
    for r in range(0, rows, 16384):
        part = x[r:r + 16384].contiguous()
        pc, ps = api.ssconv_quantize_mxfp4(part)
        assert torch.equal(pc, codes[r:r + 16384]) and torch.equal(api.ssconv_dequantize_mxfp4(pc, ps, c), back[r:r + 16384])


def _layer(rows, cin, cout, act="none", bias=True, exact=False, seed=0, y=None, **k):
    """(y, its exact value before rounding, sum of the terms' magnitudes)."""
    if exact:      # values of the grid with blocks of equal scale: every partial sum is a multiple of 1/4 below 2^22 / 4
        grid = torch.tensor([0.0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV)
        g = torch.Generator(device=DEV).manual_seed(seed)

        def values(n, m):
            v = grid[torch.randint(0, 8, (n, m), generator=g, device=DEV)] * (1 - 2 * torch.randint(0, 2, (n, m), generator=g, device=DEV))
            v[:, ::32] = 4.0
            return v.bfloat16()

        x, w = values(rows, cin), values(cout, cin)
        b = torch.randint(-64, 65, (cout,), generator=g, device=DEV).float() if bias else None
    else:
        x = (_randn(seed, rows, cin) * torch.exp(_randn(seed + 1, rows, 1))).bfloat16()
        w = (_randn(seed + 2, cout, cin) / cin ** 0.5).bfloat16()
        b = _randn(seed + 3, cout) if bias else None
    desc = api.make_desc(rows, 1, 1, cin, cout, 1, 1, bias=bias, relu=act == "relu", gelu=act == "gelu")
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    xq, wq = api.ssconv_quantize_mxfp4(x), api.ssconv_quantize_mxfp4(w)
    out = api.ssconv_forward_dense_mxfp4(desc, *xq, *wq, b, y=y, dev_status=status, **k).view(rows, cout)
    xv, wv = api.ssconv_dequantize_mxfp4(*xq, cin).double(), api.ssconv_dequantize_mxfp4(*wq, cin).double()
    want, mag = xv @ wv.t(), xv.abs() @ wv.abs().t()
    if bias:
        want, mag = want + b.double(), mag + b.double().abs()
    assert int(status) == 0
    return out, want, mag


def _activated(v, act):
    if act == "relu":
        return v.clamp(min=0)
    return v * torch.special.ndtr(v) if act == "gelu" else v


def _check_layer(rows, cin, cout, act="none", **k):
    out, want, mag = _layer(rows, cin, cout, act, **k)
    v = _activated(want, act)
    # (both activations have slopes below 1.13)
    tol = 1.13 * (cin + 1) * 2.0 ** -23 * mag + (2.0 ** -8 + 1e-5) * v.abs() + 1e-6
    worst = ((out.double() - v).abs() / tol).max()
    assert worst <= 1.0, float(worst)


@pytest.mark.parametrize("rows", [1, 5, 127, 128, 129, 1000])
@pytest.mark.parametrize("cin,cout", [(8, 8), (32, 64), (64, 192), (72, 200), (96, 384), (128, 128), (136, 136), (256, 1000), (264, 72), (520, 328), (1096, 960)])
def test_sums_that_fit_come_out_exactly(rows, cin, cout):
    out, want, _ = _layer(rows, cin, cout, exact=True, seed=rows + cin)
    assert torch.equal(out, want.float().bfloat16())


@pytest.mark.parametrize("rows,cin,cout", [(300, 512, 2048), (5000, 72, 264), (20_000, 256, 200), (148 * 128, 64, 192), (148 * 128 + 1, 64, 128), (37, 4096, 64)])
def test_many_tiles_come_out_exactly(rows, cin, cout):
    out, want, _ = _layer(rows, cin, cout, exact=True, seed=cin)
    assert torch.equal(out, want.float().bfloat16())


# (long K and many tiles: pairs of thread blocks; 157, 129 and 313 tiles of rows leave the last pair half empty)
@pytest.mark.parametrize("rows,cin,cout", [(16_384, 4096, 256), (20_000, 4040, 960), (33_000, 3880, 392), (16_500, 4096, 392), (40_001, 4000, 584)])
def test_products_on_pairs_of_blocks_come_out_exactly(rows, cin, cout):
    out, want, _ = _layer(rows, cin, cout, exact=True, seed=cin)
    assert torch.equal(out, want.float().bfloat16())


@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("rows,cin,cout", [(49, 768, 768), (1, 2048, 1000), (3136, 96, 384), (777, 392, 88), (130, 4096, 520), (16_385, 4072, 208)])
def test_layers(rows, cin, cout, act):
    _check_layer(rows, cin, cout, act, seed=7)


@pytest.mark.parametrize("cin", [96, 320])
def test_without_a_bias(cin):
    _check_layer(333, cin, 136, bias=False)


def test_scales_of_every_block_and_row_are_its_own():
    # one value per (row, block) pair and an identity-like weight: each output is one element times its two scales
    rows, blocks = 260, 12
    cin = 32 * blocks
    e = torch.randint(-20, 20, (rows, blocks), generator=torch.Generator().manual_seed(1))
    x = torch.zeros(rows, cin)
    x[:, ::32] = 1.5 * torch.exp2(e.double()).float()
    f = torch.randint(-20, 20, (blocks,), generator=torch.Generator().manual_seed(2))
    w = torch.zeros(208, cin)
    for b in range(blocks):
        w[17 * b + 3, 32 * b] = 3.0 * 2.0 ** int(f[b])
    xq, wq = api.ssconv_quantize_mxfp4(x.bfloat16().to(DEV)), api.ssconv_quantize_mxfp4(w.bfloat16().to(DEV))
    y = api.ssconv_forward_dense_mxfp4(api.make_desc(rows, 1, 1, cin, 208, 1, 1, bias=False), *xq, *wq).view(rows, 208).cpu()
    want = torch.zeros(rows, 208, dtype=torch.float64)
    for b in range(blocks):
        want[:, 17 * b + 3] = 4.5 * torch.exp2((e[:, b] + f[b]).double())
    assert torch.equal(y.double(), want)


def test_nan_reaches_its_row_and_channel_alone():
    x, w = _randn(1, 200, 160).bfloat16(), _randn(2, 264, 160).bfloat16()
    x[130, 40], w[200, 150] = float("nan"), float("inf")
    desc = api.make_desc(200, 1, 1, 160, 264, 1, 1, bias=False)
    y = api.ssconv_forward_dense_mxfp4(desc, *api.ssconv_quantize_mxfp4(x), *api.ssconv_quantize_mxfp4(w)).view(200, 264)
    bad = torch.zeros(200, 264, dtype=torch.bool, device=DEV)
    bad[130], bad[:, 200] = True, True
    assert torch.equal(y.isnan(), bad)


def test_nothing_is_written_past_the_output():
    for rows, cout in ((1, 8), (129, 200), (640, 72)):
        buf = torch.full((rows * cout + 4096,), 7.0, dtype=torch.bfloat16, device=DEV)
        out, want, _ = _layer(rows, 64, cout, exact=True, y=buf[:rows * cout].view(rows, 1, 1, cout))
        assert torch.equal(out, want.float().bfloat16()) and (buf[rows * cout:] == 7.0).all()


def test_images_keep_their_shape():
    x, w = _randn(5, 3, 9, 11, 40).bfloat16(), _randn(6, 56, 40).bfloat16()
    desc = api.make_desc(3, 9, 11, 40, 56, 1, 1, bias=False)
    xq, wq = api.ssconv_quantize_mxfp4(x), api.ssconv_quantize_mxfp4(w)
    y = api.ssconv_forward_dense_mxfp4(desc, *xq, *wq)
    assert y.shape == (3, 9, 11, 56)
    flat = api.ssconv_forward_dense_mxfp4(api.make_desc(297, 1, 1, 40, 56, 1, 1, bias=False), *xq, *wq)
    assert torch.equal(y.view(-1, 56), flat.view(-1, 56))


def test_captured_and_on_another_stream():
    x, w, b = _randn(1, 500, 96).bfloat16(), _randn(2, 200, 96).bfloat16(), _randn(3, 200)
    desc = api.make_desc(500, 1, 1, 96, 200, 1, 1, bias=True, gelu=True)
    wq = api.ssconv_quantize_mxfp4(w)

    def layer(stream=None):
        return api.ssconv_forward_dense_mxfp4(desc, *api.ssconv_quantize_mxfp4(x, stream=stream), *wq, b, stream=stream)

    want = layer()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    beside = layer(side)
    torch.cuda.synchronize()
    assert torch.equal(beside, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer()
    x.copy_(x.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y.flip(0), want)


def test_refusals():
    x, w = _randn(1, 10, 64).bfloat16(), _randn(2, 16, 64).bfloat16()
    xq, wq = api.ssconv_quantize_mxfp4(x), api.ssconv_quantize_mxfp4(w)
    d = api.make_desc(10, 1, 1, 64, 16, 1, 1, bias=False)
    with pytest.raises(ValueError):
        api.ssconv_forward_dense_mxfp4(d, xq[0][:5], xq[1], *wq)
    with pytest.raises(ValueError):
        api.ssconv_forward_dense_mxfp4(d, *wq, *xq)
    with pytest.raises(api.SsconvError):
        api.ssconv_forward_dense_mxfp4(api.make_desc(10, 1, 1, 64, 16, 1, 1, bias=True), *xq, *wq)
    with pytest.raises(api.SsconvError):
        api.ssconv_quantize_mxfp4(_randn(1, 4, 20).bfloat16())
    with pytest.raises(ValueError):
        api.ssconv_quantize_mxfp4(x.t())
    with pytest.raises(TypeError):
        api.ssconv_quantize_mxfp4(x.float())
    with pytest.raises(ValueError):
        api.ssconv_dequantize_mxfp4(xq[0], xq[1], 96)
