"""The global gradient norm, clipping and AdamW over many tensors against 64-bit arithmetic.

Tolerances, in units of u = 2^-24 (half a step of fp32): the squares of up to 8 numbers are added in 32 bits (9 roundings at
most, all terms positive, so 9 u relative), their sums in 64 bits; the root halves that and is rounded once: 6 u.  The factor adds
the rounding of norm + 1e-6 and of the quotient: 8 u; a scaled fp32 gradient one more: 9 u; a bf16 one 2^-8."""
import math
import sys

import numpy as np
import pytest
import torch

from oracle import optim
from paper_2411_00288_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def _f64(t):
    return t.detach().cpu().double().numpy()


def _grads(sizes, seed=0, dtypes=(torch.float32,), scale=0.05, offset=0):
    """Tensors of these sizes, types in turn, starting `offset` elements into their buffers."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [(torch.randn(n + offset, generator=g, device=DEV) * scale).to(dtypes[i % len(dtypes)])[offset:] for i, n in enumerate(sizes)]


SETS = {
    "one": [1],
    "none_in_it": [0, 0],
    "some_empty": [5, 0, 1000, 0],
    "odd": [1, 2, 3, 7, 8, 9, 1023, 1025, 2047, 2049],
    "one_block_at_the_line": [1024] * 32,
    "past_one_block": [1024] * 65,
    "ragged": [4097, 63, 8192, 50_003, 12_289],
    "many_small": [1 + 37 * i % 301 for i in range(400)],
    "many_launches": [i % 5 for i in range(1700)],
    "large": [3_000_001, 7, 6_500_000],
}


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16,), (torch.float32, torch.bfloat16)], ids=["f32", "bf16", "both"])
@pytest.mark.parametrize("name", SETS)
def test_norm_and_clipping(name, dtypes, offset):
    grads = _grads(SETS[name], 1, dtypes, offset=offset)
    host = [_f64(g) for g in grads]
    kept = [g.clone() for g in grads]
    for kind, inf in ((api.GRAD_NORM_L2, False), (api.GRAD_NORM_INF, True)):
        norm = api.ssconv_grad_norm(grads, kind)
        want = optim.grad_norm(host, inf)
        got = float(norm)
        assert got == want if inf else abs(got - want) <= 6 * U * want
        max_norm = 0.37 * want if want else 1.0
        out = api.ssconv_clip_grads(grads, norm, max_norm, out=[torch.full_like(g, 9) for g in grads])
        factor = optim.clip_factor(want, np.float64(np.float32(max_norm)))
        for o, g, dtype in zip(out, host, (g.dtype for g in grads)):
            tol = 9 * U if dtype is torch.float32 else 2.0 ** -8
            assert (np.abs(_f64(o) - g * factor) <= tol * np.abs(g * factor) + 2.0 ** -149).all()
    assert all(torch.equal(a, b) for a, b in zip(grads, kept))
    api.ssconv_clip_grads(grads, norm, max_norm)                # in place: the same bits
    assert all(torch.equal(a, b) for a, b in zip(grads, out))


def test_same_bits_every_time():
    grads = _grads([1_000_003, 5, 70_001], 2)
    first = api.ssconv_grad_norm(grads)
    assert all(torch.equal(api.ssconv_grad_norm(grads), first) for _ in range(20))


def test_nothing_is_written_beside_the_tensors():
    flat = torch.full((10_000,), 3.0, device=DEV)
    views = [flat[10:1011], flat[2000:2003], flat[4000:8193]]
    norm = api.ssconv_grad_norm(views)
    api.ssconv_clip_grads(views, norm, 1.0)
    there = torch.zeros(10_000, dtype=torch.bool, device=DEV)
    for a, b in ((10, 1011), (2000, 2003), (4000, 8193)):
        there[a:b] = True
    assert (flat[~there] == 3.0).all() and (flat[there] < 3.0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", [3e38, 1e30, 1e-30, 2.0 ** -120])
def test_no_overflow_and_no_loss_on_the_way(value, dtype):
    g = torch.full((3000,), value, device=DEV).to(dtype)
    want = float(g[0].double()) * math.sqrt(3000)
    got = float(api.ssconv_grad_norm([g]))
    assert got == math.inf if want > 3.4028236e38 else abs(got - want) <= 6 * U * want


@pytest.mark.parametrize("kind", [api.GRAD_NORM_L2, api.GRAD_NORM_INF])
@pytest.mark.parametrize("n", [40, 200_000])
def test_infinities_and_nan(kind, n):
    for bad, check in ((math.inf, math.isinf), (-math.inf, math.isinf), (math.nan, math.isnan)):
        g = torch.ones(n, device=DEV)
        g[n // 2] = bad
        norm = api.ssconv_grad_norm([g], kind)
        assert check(float(norm))
        out = api.ssconv_clip_grads([g], norm, 1.0)[0]
        if math.isnan(bad):
            assert out.isnan().all()
        else:
            assert out[n // 2].isnan() and (out[:n // 2] == 0).all()


def test_gradients_within_the_norm_keep_their_bits():
    g = _grads([777, 5000], 4, (torch.bfloat16, torch.float32))
    kept = [t.clone() for t in g]
    norm = api.ssconv_grad_norm(g)
    out = api.ssconv_clip_grads(g, norm, 1e9, out=[torch.empty_like(t) for t in g])
    api.ssconv_clip_grads(g, norm, 1e9)
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(kept, out, g))


def _state(sizes, seed, dtypes):
    g = torch.Generator(device=DEV).manual_seed(seed)
    theta = [torch.randn(n, generator=g, device=DEV) for n in sizes]
    m = [0.01 * torch.randn(n, generator=g, device=DEV) for n in sizes]
    v = [(0.01 * torch.randn(n, generator=g, device=DEV)).square() for n in sizes]
    return theta, _grads(sizes, seed + 1, dtypes), m, v


def _check_update(before, after, grads, factor, step, hyper):
    """m: two products and a sum, with the factor (8 u) and both constants rounded: 12 u of the terms' magnitudes.  v: the square of
    the scaled gradient (18 u), constants, products, sum: 24 u, all terms positive.  The update divides m c1 by sqrt(v c2) + eps:
    12 + 2 (c1 and its product) + 12 + 2 (root, halved) + 3 (sum, quotient): 32 u of lr times its magnitude; decay adds 3."""
    for (t0, m0, v0), (t1, m1, v1), g in zip(before, after, grads):
        t0, m0, v0, t1, m1, v1, g = (_f64(a) for a in (t0, m0, v0, t1, m1, v1, g))
        g = g * factor
        lr, b1, b2, eps, decay = hyper
        t, m, v = optim.adamw(t0, g, m0, v0, step, *hyper)
        m_mag = b1 * np.abs(m0) + (1 - b1) * np.abs(g)
        assert (np.abs(m1 - m) <= 12 * U * m_mag + 2.0 ** -148).all()
        assert (np.abs(v1 - v) <= 24 * U * v + 2.0 ** -148).all()
        move = m_mag / (1 - b1 ** step) / (np.sqrt(v / (1 - b2 ** step)) + eps)
        assert (np.abs(t1 - t) <= 2 * U * np.abs(t0) + 32 * U * lr * (move + decay * np.abs(t0))).all()


@pytest.mark.parametrize("clip", [None, 0.4, 1e6])
@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16, torch.float32)], ids=["f32", "both"])
@pytest.mark.parametrize("name", ["one", "some_empty", "odd", "ragged", "many_small", "many_launches"])
def test_adamw_of_many_tensors(name, dtypes, clip):
    theta, g, m, v = _state(SETS[name], 11, dtypes)
    before = [tuple(t.clone() for t in s) for s in zip(theta, m, v)]
    norm = None if clip is None else api.ssconv_grad_norm(g)
    hyper = (1e-2, 0.9, 0.999, 1e-8, 1e-2)
    api.ssconv_adamw_multi(theta, g, m, v, 5, *hyper, norm=norm, max_norm=1.0 if clip is None else clip)
    factor = 1.0 if clip is None else optim.clip_factor(optim.grad_norm([_f64(t) for t in g]), float(np.float32(clip)))
    _check_update(before, list(zip(theta, m, v)), g, factor, 5, hyper)


def test_adamw_of_unaligned_tensors():
    sizes = [4099, 10, 333]
    theta, g, m, v = _state([n + 1 for n in sizes], 12, (torch.float32, torch.bfloat16))
    theta, g, m = [t[1:] for t in theta], [t[1:] for t in g], [t[1:] for t in m]
    v = [t[:-1] for t in v]
    before = [tuple(t.clone() for t in s) for s in zip(theta, m, v)]
    hyper = (1e-2, 0.9, 0.99, 1e-6, 0.0)
    api.ssconv_adamw_multi(theta, g, m, v, 1, *hyper)
    _check_update(before, list(zip(theta, m, v)), g, 1.0, 1, hyper)


def test_one_call_is_what_a_call_per_tensor_is():
    theta, g, m, v = _state([100_001, 64, 4096], 13, (torch.float32,))
    one = [[t.clone() for t in s] for s in (theta, m, v)]
    api.ssconv_adamw_multi(theta, g, m, v, 3, lr=0.5, beta2=0.75)
    for i in range(3):
        api.ssconv_adamw(one[0][i], g[i], one[1][i], one[2][i], 3, lr=0.5, beta2=0.75)
        # (1 - beta in 64 bits here, in 32 there: 0.1 by 2^-25 / 0.1, on top of each side's own roundings)
        for a, b in zip((theta[i], m[i], v[i]), (one[0][i], one[1][i], one[2][i])):
            torch.testing.assert_close(a, b, rtol=2e-6, atol=2e-6)


@pytest.mark.parametrize("sizes", [[300, 20], [400_000, 9, 33]])
def test_captured_replayed_and_on_another_stream(sizes):
    side = torch.cuda.Stream()
    theta, g, m, v = _state(sizes, 14, (torch.float32,))
    other = [[t.clone() for t in s] for s in (theta, g, m, v)]

    def step(theta, g, m, v, stream=None):
        norm = api.ssconv_grad_norm(g, stream=stream)
        api.ssconv_adamw_multi(theta, g, m, v, 2, norm=norm, max_norm=0.5, stream=stream)
        return norm

    side.wait_stream(torch.cuda.current_stream())
    step(*other, stream=side)
    graph = torch.cuda.CUDAGraph()
    kept = [[t.clone() for t in s] for s in (theta, g, m, v)]
    with torch.cuda.graph(graph):
        norm = step(theta, g, m, v)
    for s, k in zip((theta, g, m, v), kept):
        for a, b in zip(s, k):
            a.copy_(b)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for s, o in zip((theta, m, v), (other[0], other[2], other[3])) for a, b in zip(s, o))
    g[0].mul_(3.0)                                              # new gradients, the same graph
    graph.replay()
    torch.cuda.synchronize()
    want = optim.grad_norm([_f64(t) for t in g])
    assert abs(float(norm) - want) <= 6 * U * want


def test_two_graphs_keep_their_own_scratch():
    sets = [_grads([500_000, 77], 20 + i, scale=0.1 * (i + 1)) for i in range(2)]
    graphs, norms = [], []
    for g in sets:
        api.ssconv_grad_norm(g)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            norms.append(api.ssconv_grad_norm(g))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(50):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for g, n in zip(sets, norms):
        want = optim.grad_norm([_f64(t) for t in g])
        assert abs(float(n) - want) <= 6 * U * want


def test_refusals():
    g = _grads([10, 20])
    norm = api.ssconv_grad_norm(g)
    with pytest.raises(ValueError):
        api.ssconv_grad_norm([torch.zeros(4, 4, device=DEV).t()[1:]])
    with pytest.raises(TypeError):
        api.ssconv_grad_norm([torch.zeros(4, device=DEV, dtype=torch.float16)])
    with pytest.raises(TypeError):
        api.ssconv_clip_grads(g, norm, 1.0, out=[t.bfloat16() for t in g])
    with pytest.raises(ValueError):
        api.ssconv_clip_grads(g, norm, 1.0, out=g[:1])
    with pytest.raises(ValueError):
        api.ssconv_clip_grads(g, norm, 1.0, out=g[::-1])
    with pytest.raises(ValueError):
        api.ssconv_clip_grads(g, torch.zeros(2, device=DEV), 1.0)
    with pytest.raises(api.SsconvError):
        api.ssconv_clip_grads([g[0], g[0]], norm, 1.0)
    with pytest.raises(TypeError):
        api.ssconv_adamw_multi([t.bfloat16() for t in g], g, g, g, 1)
    with pytest.raises(api.SsconvError):
        api.ssconv_adamw_multi(g, g, g, g, 1)
    with pytest.raises(ValueError):
        api.ssconv_adamw_multi(g, g, g, g, 0)
    with pytest.raises(api.SsconvError):
        api.ssconv_grad_norm(g, ws=torch.empty(8, dtype=torch.uint8, device=DEV))


def test_bounds_at_the_ends():
    """max_norm = 0 leaves zeros, an infinite one leaves the gradients (NaN if the norm is infinite too)."""
    g = torch.randn(1000, device="cuda")
    norm = api.ssconv_grad_norm([g])
    out = [torch.empty_like(g)]
    api.ssconv_clip_grads([g], norm, 0.0, out=out)
    assert torch.equal(out[0], g * 0)
    api.ssconv_clip_grads([g], norm, math.inf, out=out)
    assert torch.equal(out[0], g)
    api.ssconv_clip_grads([g], torch.full_like(norm, math.inf), math.inf, out=out)
    assert out[0].isnan().all()


def test_tensors_that_only_a_generator_gives():
    """Nobody but the call holds them: their memory must not be handed out again before it is made."""
    g = _grads([4096, 100, 70_000], 31)
    want = api.ssconv_grad_norm(g)
    for _ in range(10):
        assert torch.equal(api.ssconv_grad_norm(t.clone() for t in g), want)
        scaled = api.ssconv_clip_grads((t.clone() for t in g), want, 0.5)
        assert all(torch.equal(a, b) for a, b in zip(scaled, api.ssconv_clip_grads(g, want, 0.5, out=(torch.empty_like(t) for t in g))))
        assert len(scaled) == 3
    theta, m, v = ([torch.zeros_like(t) for t in g] for _ in range(3))
    one = [[t.clone() for t in s] for s in (theta, m, v)]
    api.ssconv_adamw_multi(theta, g, m, v, 1, norm=want, max_norm=0.5)
    api.ssconv_adamw_multi(iter(one[0]), (t.clone() for t in g), iter(one[1]), iter(one[2]), 1, norm=want, max_norm=0.5)
    assert all(torch.equal(a, b) for s, o in zip((theta, m, v), one) for a, b in zip(s, o))


def _chunks(count, tensors, ragged):
    """Extents of `tensors` tensors that are cut into `count` chunks of 2048; ragged: the last chunk of each has one element."""
    per = [count // tensors + (i < count % tensors) for i in range(tensors)]
    return [2048 * k - 2047 * ragged for k in per]


# where another form of the norm is taken: 32, 64 and 128 chunks are the warps of one, two and four blocks of a cluster, 256 the last ones
# that one launch takes, 32 and 384 tensors the most of a kernel's argument; 1184 blocks make a launch of 148 SMs, and from
# 1184 * 4096 and 1184 * 8192 elements on chunks are longer
LIMITS = {f"{c}_chunks_of_{t}{'_ragged' if r else ''}": _chunks(c, t, r)
          for c in (32, 33, 64, 65, 128, 129, 256, 257) for t in (1, 32) for r in (False, True) if c >= t}
LIMITS.update({f"{t}_tensors": [2049 + i for i in range(t - 1)] + [5] for t in (31, 32, 33, 383, 384, 385, 768, 769)})
LIMITS.update({f"{t}_tensors_between_empty_ones": [0, 0] + [100 + i for i in range(t)] + [0, 0, 0] for t in (32, 33, 384, 385)})
LIMITS.update({f"{n}_elements": [n - 3, 3] for n in (1184 * 2048, 1184 * 2048 + 4, 1184 * 4096 - 1, 1184 * 4096, 1184 * 8192 - 1, 1184 * 8192)})


@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.float32, torch.bfloat16)], ids=["f32", "both"])
@pytest.mark.parametrize("name", LIMITS)
def test_at_the_limits_of_the_forms(name, dtypes):
    grads = _grads(LIMITS[name], 3, dtypes)
    grads[-1].mul_(50)                                          # (the last chunk counts)
    host = [_f64(g) for g in grads]
    for kind, inf in ((api.GRAD_NORM_L2, False), (api.GRAD_NORM_INF, True)):
        want, got = optim.grad_norm(host, inf), float(api.ssconv_grad_norm(grads, kind))
        assert got == want if inf else abs(got - want) <= 6 * U * want
    norm = api.ssconv_grad_norm(grads)
    factor = optim.clip_factor(optim.grad_norm(host), 0.5)
    for o, g, dtype in zip(api.ssconv_clip_grads(grads, norm, 0.5, out=[torch.full_like(g, 9) for g in grads]), host, (g.dtype for g in grads)):
        assert (np.abs(_f64(o) - g * factor) <= (9 * U if dtype is torch.float32 else 2.0 ** -8) * np.abs(g * factor) + 2.0 ** -149).all()
    theta, m, v = ([torch.ones(n, device=DEV) for n in LIMITS[name]] for _ in range(3))
    before = [tuple(t.clone() for t in s) for s in zip(theta, m, v)]
    hyper = (1e-2, 0.9, 0.999, 1e-8, 1e-2)
    api.ssconv_adamw_multi(theta, grads, m, v, 5, *hyper, norm=norm, max_norm=0.5)
    _check_update(before, list(zip(theta, m, v)), grads, factor, 5, hyper)


@pytest.mark.parametrize("count", [3, 32, 33, 100])
def test_calls_hold_no_tensor_afterwards(count):
    g = _grads([7] * count, 32)
    norm = api.ssconv_grad_norm(g)

    def references():
        return [sys.getrefcount(t) for t in g]

    before = references()
    api.ssconv_grad_norm(g)
    api.ssconv_clip_grads(g, norm, 0.5, out=[torch.empty_like(t) for t in g])
    for bad in (torch.zeros(7), torch.zeros(8, device=DEV), torch.zeros(7, device=DEV, dtype=torch.float16), None):
        with pytest.raises((TypeError, ValueError)):
            api.ssconv_clip_grads(g, norm, 0.5, out=g[:-1] + [bad])
    with pytest.raises(ValueError):
        api.ssconv_clip_grads(g, norm, 0.5, out=g[:-1])
    assert references() == before
