"""Tensors of more than 2^31 elements through the many-tensor, residual-and-norm and 4-bit calls: their last rows are what a call on
those rows alone gives."""
import pytest
import torch

from paper_2411_00288_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FAR = 1 << 31


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def test_norm_clip_and_update_of_a_far_tensor():
    n, tail = FAR + 12_345, 10_001
    g = torch.Generator(device=DEV).manual_seed(1)
    grad = torch.zeros(n, device=DEV)
    grad[-tail:] = _randn(g, tail)
    alone = grad[-tail:].clone()
    norm, inf = api.ssconv_grad_norm([grad]), api.ssconv_grad_norm([grad], api.GRAD_NORM_INF)
    assert abs(float(norm) - float(alone.double().norm())) <= 2.0 ** -20 * float(norm) and float(inf) == float(alone.abs().max())
    api.ssconv_clip_grads([grad], norm, 0.5)
    api.ssconv_clip_grads([alone], norm, 0.5)
    assert torch.equal(grad[-tail:], alone) and not grad[:-tail].any()
    theta, m, v = (torch.zeros(n, device=DEV) for _ in range(3))
    small = [torch.zeros(tail, device=DEV) for _ in range(3)]
    api.ssconv_adamw_multi([theta], [grad], [m], [v], 1)
    api.ssconv_adamw_multi([small[0]], [alone], [small[1]], [small[2]], 1)
    assert all(torch.equal(a[-tail:], b) for a, b in zip((theta, m, v), small))


@pytest.mark.parametrize("c,per", [(4096, 0), (96, 0), (96, 1000)])
def test_far_rows_of_the_end_of_a_block(c, per):
    tail = 2000
    rows = (FAR // c + 1000) // tail * tail + tail
    g = torch.Generator(device=DEV).manual_seed(2)
    x, b, dh, dy = (torch.zeros(rows, c, dtype=torch.bfloat16, device=DEV) for _ in range(4))
    for t in (x, b, dh, dy):
        t[-tail:] = _randn(g, tail, c).bfloat16()
    gates = 1 if per == 0 else rows // per
    gate = 0.5 + 0.1 * _randn(g, gates, c)
    affine = dict(post_gamma=1 + 0.1 * _randn(g, c), pre_gamma=1 + 0.1 * _randn(g, c))

    def run(rows, gate, *tensors):
        d = api.make_resnorm(rows, c, rows_per_gate=per, post=api.NORM_LAYER, pre=api.NORM_RMS)
        h, y, stats = api.ssconv_residual_norm(d, tensors[0], tensors[1], gate=gate, want_stats=True, **affine)
        r = api.ssconv_residual_norm_backward(d, *tensors[:2], stats, *tensors[2:], gate=gate, **affine)
        return h, y, r

    h, y, r = run(rows, gate, x, b, dh, dy)
    h1, y1, r1 = run(tail, gate[-(tail // per):] if per else gate, *(t[-tail:].clone() for t in (x, b, dh, dy)))
    for far, near in ((h, h1), (y, y1), (r.dx, r1.dx), (r.db, r1.db)):
        assert torch.equal(far[-tail:], near)
    if per:
        torch.testing.assert_close(r.dgate[-(tail // per):], r1.dgate, rtol=1e-4, atol=1e-2)   # (other units, another order)
    torch.testing.assert_close(r.dpre_gamma, r1.dpre_gamma, rtol=1e-4, atol=1e-2)


def test_far_rows_in_four_bits():
    rows, cin, cout, tail = FAR // 1024 + 130, 40, 1024, 500
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.zeros(rows, cin, dtype=torch.bfloat16, device=DEV)
    x[-tail:] = _randn(g, tail, cin).bfloat16()
    wq, bias = api.ssconv_quantize_mxfp4(_randn(g, cout, cin).bfloat16()), _randn(g, cout)

    def run(x):
        return api.ssconv_forward_dense_mxfp4(api.make_desc(x.shape[0], 1, 1, cin, cout, 1, 1), *api.ssconv_quantize_mxfp4(x), *wq, bias).view(-1, cout)

    assert torch.equal(run(x)[-tail:], run(x[-tail:].clone()))
    del x
    wide = torch.zeros(FAR // 4096 + 33, 4096, dtype=torch.bfloat16, device=DEV)
    wide[-40:] = _randn(g, 40, 4096).bfloat16()
    codes, scales = api.ssconv_quantize_mxfp4(wide)
    back = api.ssconv_dequantize_mxfp4(codes, scales, 4096)
    near = api.ssconv_quantize_mxfp4(wide[-40:].clone())
    assert torch.equal(codes[-40:], near[0]) and torch.equal(back[-40:], api.ssconv_dequantize_mxfp4(*near, 4096)) and not back[:-40].any()
