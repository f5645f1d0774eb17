"""The calls around the convolutions together: a training step of two residual blocks, a mask-learning step that ends in one update
of all layers' choice weights, and a ConvNeXt-shaped block in 4 bits."""
import os
import subprocess
import sys
import threading

import numpy as np
import pytest
import torch

from oracle import optim
from paper_2411_00288_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


class Blocks:
    """h_{i+1} = h_i + gate_i * norm(conv_i(n_i)), n_i = pre_i(h_i) from the block before: fp32 parameters, bf16 weights for the calls."""

    def __init__(self, n=2, hw=9, c=48, k=3, blocks=2):
        g = torch.Generator(device=DEV).manual_seed(5)
        self.rows, self.c, self.blocks = n * hw * hw, c, blocks
        self.conv = api.make_desc(n, hw, hw, c, c, k, k, 1, k // 2, bias=False)
        self.norm = api.make_resnorm(self.rows, c, rows_per_gate=0, post=api.NORM_LAYER, pre=api.NORM_LAYER, eps=1e-5)
        self.params = []
        for _ in range(blocks):
            self.params += [_randn(g, c, k, k, c) / (k * c ** 0.5), 0.5 + 0.1 * _randn(g, c), 1 + 0.1 * _randn(g, c), 0.1 * _randn(g, c),
                            1 + 0.1 * _randn(g, c), 0.1 * _randn(g, c)]
        self.x = _randn(g, n, hw, hw, c).bfloat16()
        self.dy = _randn(g, n, hw, hw, c).bfloat16()
        self.m = [torch.zeros_like(p) for p in self.params]
        self.v = [torch.zeros_like(p) for p in self.params]

    def step(self, t, max_norm):
        """Forward, backward, clip, update; returns (last norm's output, gradients, their norm)."""
        h, y, kept = self.x, self.x, []
        for i in range(self.blocks):
            w, gate, *affine = self.params[6 * i:6 * i + 6]
            wb = w.bfloat16()
            b = api.ssconv_forward_dense(self.conv, y, wb)
            names = dict(zip(("post_gamma", "post_beta", "pre_gamma", "pre_beta"), affine), gate=gate)
            h_next, y_next, stats = api.ssconv_residual_norm(self.norm, h, b, want_stats=True, **names)
            kept.append((h, y, b, wb, stats, names))
            h, y = h_next, y_next
        out, grads, dh, dy = y, [None] * len(self.params), None, self.dy
        for i in reversed(range(self.blocks)):
            h, y, b, wb, stats, names = kept[i]
            r = api.ssconv_residual_norm_backward(self.norm, h, b, stats, dh, dy, **names)
            grads[6 * i] = api.ssconv_wgrad(self.conv, y, r.db)
            grads[6 * i + 1:6 * i + 6] = [r.dgate, r.dpost_gamma, r.dpost_beta, r.dpre_gamma, r.dpre_beta]
            dh, dy = r.dx, api.ssconv_dgrad(self.conv, r.db, wb)
        norm = api.ssconv_grad_norm(grads)
        api.ssconv_adamw_multi(self.params, grads, self.m, self.v, t, lr=1e-2, weight_decay=0.0, norm=norm, max_norm=max_norm)
        return out, grads, norm

    def exact(self):
        """The same forward pass and its gradients in 64 bits, by automatic differentiation; the weights as the calls see them."""
        leaves = [p.double().requires_grad_() for p in self.params]
        h = y = self.x.double()
        eps = float(np.float32(1e-5))

        def layer(v, gamma, beta):
            d = v - v.mean(-1, keepdim=True)
            return d / torch.sqrt((d * d).mean(-1, keepdim=True) + eps) * gamma + beta

        for i in range(self.blocks):
            w, gate, pg, pb, qg, qb = leaves[6 * i:6 * i + 6]
            seen = w + (self.params[6 * i].bfloat16().double() - w).detach()
            b = torch.nn.functional.conv2d(y.permute(0, 3, 1, 2), seen.permute(0, 3, 1, 2), padding=1).permute(0, 2, 3, 1)
            h = h + gate * layer(b, pg, pb)
            y = layer(h, qg, qb)
        return y.detach(), torch.autograd.grad((y * self.dy.double()).sum(), leaves)


def test_a_training_step_of_two_blocks():
    """bf16 between the calls: every tensor that is stored on the way (four per block and direction) adds a rounding of 2^-9 of its
    values on average; through two blocks a gradient stays within 16 of them, 2^-5, of the exact one in norm."""
    net = Blocks()
    y, want = net.exact()
    before = [p.clone() for p in net.params]
    out, grads, norm = net.step(1, max_norm=0.5)
    assert (out.double() - y).norm() <= 2.0 ** -6 * y.norm()
    for got, g in zip(grads, want):
        assert (got.double() - g).norm() <= 2.0 ** -5 * g.norm()
    host = [g.cpu().double().numpy() for g in grads]
    n = optim.grad_norm(host)
    assert abs(float(norm) - n) <= 6 * 2.0 ** -24 * n
    factor = optim.clip_factor(n, 0.5)
    for p0, p1, g in zip(before, net.params, host):
        t, _, _ = optim.adamw(p0.cpu().double().numpy(), g * factor, 0.0, 0.0, 1, 1e-2, 0.9, 0.999, 1e-8, 0.0)
        # (2 u of the parameter, 64 u of a move of at most lr)
        assert (np.abs(p1.cpu().double().numpy() - t) <= 2.0 ** -23 * np.abs(t) + 2.0 ** -18 * 1e-2).all()


def test_the_step_captured_and_replayed_while_eager_steps_go_on():
    one, two = Blocks(), Blocks()
    one.step(1, 0.5)
    two.step(1, 0.5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    saved = [[t.clone() for t in s] for s in (one.params, one.m, one.v)]
    with torch.cuda.graph(graph):
        out, grads, norm = one.step(2, 0.5)
    for s, k in zip((one.params, one.m, one.v), saved):
        for a, b in zip(s, k):
            a.copy_(b)
    graph.replay()
    out2, grads2, norm2 = two.step(2, 0.5)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(norm, norm2)
    assert all(torch.equal(a, b) for a, b in zip(grads, grads2))
    assert all(torch.equal(a, b) for a, b in zip(one.params, two.params))


def test_choice_weights_of_all_layers_in_one_update():
    g = torch.Generator(device=DEV).manual_seed(8)
    layers = [(64, 64, 3), (128, 64, 1), (256, 128, 1), (8, 24, 3)]
    ws = [(_randn(g, co, k, k, ci) / (k * ci ** 0.5)).bfloat16() for co, ci, k in layers]
    logits = [0.01 * _randn(g, w.numel() // 4, 6) for w in ws]
    ups = [_randn(g, *w.shape) for w in ws]
    zs = [api.ssconv_soft_mask(t, None, 0.5, w)[0] for t, w in zip(logits, ws)]
    grads = [api.ssconv_mask_grad(z, 0.5, w, up) for z, w, up in zip(zs, ws, ups)]
    m, v = ([torch.zeros_like(t) for t in logits] for _ in range(2))
    one = [t.clone() for t in logits]
    norm = api.ssconv_grad_norm(grads)
    api.ssconv_adamw_multi(logits, grads, m, v, 1, lr=1.0, norm=norm, max_norm=0.25)
    clipped = api.ssconv_clip_grads(grads, norm, 0.25, out=[torch.empty_like(t) for t in grads])
    assert abs(float(api.ssconv_grad_norm(clipped)) - 0.25) <= 1e-5
    for a, t, c in zip(logits, one, clipped):
        api.ssconv_adamw(t, c, torch.zeros_like(t), torch.zeros_like(t), 1, lr=1.0)
        torch.testing.assert_close(a, t, rtol=4e-6, atol=4e-6)   # (the constants are rounded in another place)


@pytest.mark.parametrize("batch,hw,c", [(3, 14, 96), (1, 7, 192)])
def test_a_convnext_shaped_block_in_four_bits(batch, hw, c):
    """Depthwise, norm, two point-wise layers in 4 bits, layer scale and skip connection with the next norm: each step against 64
    bits on what the step before produced."""
    g = torch.Generator(device=DEV).manual_seed(c)
    rows = batch * hw * hw
    x = _randn(g, batch, hw, hw, c).bfloat16()
    dw = api.make_desc(batch, hw, hw, c, c, 7, 7, 1, 3, bias=True)
    t = api.ssconv_depthwise(dw, x, (0.1 * _randn(g, 7, 7, c)).bfloat16(), 0.1 * _randn(g, c))
    gamma, beta = 1 + 0.1 * _randn(g, c), 0.1 * _randn(g, c)
    t = api.ssconv_layernorm(t, gamma, beta)
    w1, w2 = ((_randn(g, *s) / s[1] ** 0.5).bfloat16() for s in ((4 * c, c), (c, 4 * c)))
    b1, b2 = 0.1 * _randn(g, 4 * c), 0.1 * _randn(g, c)
    for w, b, gelu in ((w1, b1, True), (w2, b2, False)):
        d = api.make_desc(batch, hw, hw, w.shape[1], w.shape[0], 1, 1, bias=True, gelu=gelu)
        xq, wq = api.ssconv_quantize_mxfp4(t), api.ssconv_quantize_mxfp4(w)
        y = api.ssconv_forward_dense_mxfp4(d, *xq, *wq, b)
        v = api.ssconv_dequantize_mxfp4(*xq, w.shape[1]).double().view(rows, -1) @ api.ssconv_dequantize_mxfp4(*wq, w.shape[1]).double().t() + b.double()
        v = v * torch.special.ndtr(v) if gelu else v
        assert (y.double().view(rows, -1) - v).norm() <= 2.0 ** -8 * v.norm()
        t = y
    scale = 0.3 + 0.05 * _randn(g, c)
    h, n, _ = api.ssconv_residual_norm(api.make_resnorm(rows, c, pre=api.NORM_LAYER), x, t, gate=scale, pre_gamma=gamma, pre_beta=beta)
    want = x.double() + scale.double() * t.double()
    assert h.shape == x.shape and (h.double() - want).abs().max() <= 2.0 ** -8 * want.abs().max()
    d = want - want.mean(-1, keepdim=True)
    want = d / torch.sqrt((d * d).mean(-1, keepdim=True) + float(np.float32(1e-6))) * gamma.double() + beta.double()
    assert (n.double() - want).abs().max() <= 2.0 ** -8 * want.abs().max() + 1e-5


def test_a_bias_that_was_updated_just_before_its_layer():
    """AdamW on a 4-bit layer's bias, quantisation of its input and the layer, over and over without waiting: each kernel may start
    while those before it run, and the outputs are those of calls that wait for each other."""
    g = torch.Generator(device=DEV).manual_seed(21)
    rows, cin, cout = 5000, 96, 384
    desc = api.make_desc(rows, 1, 1, cin, cout, 1, 1, bias=True, gelu=True)
    xs = [_randn(g, rows, cin).bfloat16() for _ in range(3)]
    wq = api.ssconv_quantize_mxfp4((_randn(g, cout, cin) / cin ** 0.5).bfloat16())
    grads = [_randn(g, cout) for _ in range(3)]
    start = _randn(g, cout)

    def steps(wait):
        bias, m, v = start.clone(), torch.zeros_like(start), torch.zeros_like(start)
        out = []
        for t in range(24):
            api.ssconv_adamw_multi([bias], [grads[t % 3]], [m], [v], t + 1, lr=0.5)
            wait()
            xq = api.ssconv_quantize_mxfp4(xs[t % 3])
            wait()
            out.append(api.ssconv_forward_dense_mxfp4(desc, *xq, *wq, bias))
            wait()
        return out

    apart = steps(torch.cuda.synchronize)
    together = steps(lambda: None)
    assert all(torch.equal(a, b) for a, b in zip(apart, together))


@pytest.mark.parametrize("own", [True, False], ids=["a_stream", "the_default_stream"])
def test_streams_that_are_not_torchs(own):
    """Any object with `cuda_stream`, as the calls of the convolutions take it."""
    side = torch.cuda.Stream() if own else torch.cuda.default_stream()

    class Raw:
        cuda_stream = side.cuda_stream

    def calls(stream):
        g = torch.Generator(device=DEV).manual_seed(3)
        grads = [_randn(g, 300), _randn(g, 70)]
        theta, m, v = ([torch.zeros_like(t) for t in grads] for _ in range(3))
        x, b, dy = (_randn(g, 40, 96).bfloat16() for _ in range(3))
        w = _randn(g, 64, 96).bfloat16()
        torch.cuda.synchronize()
        norm = api.ssconv_grad_norm(grads, stream=stream)
        clipped = api.ssconv_clip_grads(grads, norm, 0.5, out=[torch.empty_like(t) for t in grads], stream=stream)
        api.ssconv_adamw_multi(theta, grads, m, v, 1, norm=norm, max_norm=0.5, stream=stream)
        d = api.make_resnorm(40, 96)
        h, y, stats = api.ssconv_residual_norm(d, x, b, want_stats=True, stream=stream)
        r = api.ssconv_residual_norm_backward(d, x, b, stats, None, dy, stream=stream)
        xq, wq = api.ssconv_quantize_mxfp4(y, stream=stream), api.ssconv_quantize_mxfp4(w, stream=stream)
        out = api.ssconv_forward_dense_mxfp4(api.make_desc(40, 1, 1, 96, 64, 1, 1, bias=False), *xq, *wq, stream=stream)
        back = api.ssconv_dequantize_mxfp4(*xq, 96, stream=stream)
        assert torch.cuda.current_stream() == torch.cuda.default_stream()
        torch.cuda.synchronize()
        return [norm, *clipped, *theta, *m, *v, h, y, stats, r.dx, r.db, out, back]

    assert all(torch.equal(a, b) for a, b in zip(calls(Raw()), calls(None)))
    assert all(torch.equal(a, b) for a, b in zip(calls(torch.Stream(device=DEV)), calls(None)))


def _all_calls(g, i):
    """Every call once, on extents that differ with i; what each wrote."""
    grads = [_randn(g, n) for n in (300_000 + i, 5, 77)]
    theta, m, v = ([torch.zeros_like(t) for t in grads] for _ in range(3))
    rows, c = 700, (96, 768, 1000, 2048, 5000, 384)[i % 6]
    x, b, dh, dy = (_randn(g, rows, c).bfloat16() for _ in range(4))
    gate, w = _randn(g, 7, c), _randn(g, 264, c).bfloat16()

    def run():
        norm = api.ssconv_grad_norm(grads)
        clipped = api.ssconv_clip_grads(grads, norm, 0.5, out=[torch.empty_like(t) for t in grads])
        api.ssconv_adamw_multi(theta, grads, m, v, 1, norm=norm, max_norm=0.5)
        d = api.make_resnorm(rows, c, rows_per_gate=100, post=1 + i % 2, pre=1 + i // 2 % 2)
        h, y, stats = api.ssconv_residual_norm(d, x, b, gate=gate, want_stats=True)
        r = api.ssconv_residual_norm_backward(d, x, b, stats, dh, dy, gate=gate)
        xq, wq = api.ssconv_quantize_mxfp4(y), api.ssconv_quantize_mxfp4(w)
        out = api.ssconv_forward_dense_mxfp4(api.make_desc(rows, 1, 1, c, 264, 1, 1, bias=False), *xq, *wq)
        return [norm, *clipped, *theta, h, y, stats, r.dx, r.db, r.dgate, *xq, out, api.ssconv_dequantize_mxfp4(*xq, c)]

    return run, (theta, m, v)


def test_calls_of_four_threads_at_once():
    streams = [torch.cuda.Stream() for _ in range(4)]

    def work(k, out):
        with torch.cuda.stream(streams[k]):
            g = torch.Generator(device=DEV).manual_seed(100 + k)
            for i in range(24):
                out.append([t.clone() for t in _all_calls(g, i)[0]()])
            streams[k].synchronize()

    def all_of(at_once):
        outs = [[] for _ in streams]
        threads = [threading.Thread(target=work, args=(k, outs[k])) for k in range(4)]
        for t in threads:
            t.start()
            if not at_once:
                t.join()
        for t in threads:
            t.join()
        return outs

    together, apart = all_of(True), all_of(False)
    for a, b in zip(together, apart):
        assert len(a) == len(b) == 24
        assert all(torch.equal(s, t) for x, y in zip(a, b) for s, t in zip(x, y))


def test_a_process_whose_first_calls_are_recorded():
    """Nothing that the calls set up once per process is closed to a recording."""
    code = """
import torch
from tests.test_gpu_block_step import DEV, _all_calls
run, state = _all_calls(torch.Generator(device=DEV).manual_seed(1), 0)
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    out = run()
graph.replay()
torch.cuda.synchronize()
kept = [t.clone() for t in out]
for tensors in state:
    for t in tensors:
        t.zero_()
assert all(torch.equal(a, b) for a, b in zip(kept, run()))
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
