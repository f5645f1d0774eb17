"""The oracles of the many-tensor, residual-and-norm and 4-bit calls against closed forms and differences."""
import numpy as np
import pytest

from oracle import mxfp4, optim, resnorm


def test_mxfp4_grid_ties_and_saturation():
    x = np.zeros((1, 64))
    x[0, :12] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.9, -0.75, -5.0]   # scale 1: the largest is in [4, 8)
    codes, e = mxfp4.quantize(x)
    v = mxfp4.values(codes, e, 64)
    assert e.tolist() == [[0, -127]]
    assert v[0, :12].tolist() == [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, 6.0, -1.0, -4.0]


@pytest.mark.parametrize("k", [-130, -126, -125, -3, 0, 5, 127])
def test_mxfp4_scale_is_the_power_of_two_below(k):
    x = np.zeros((1, 32))
    x[0, 3] = 1.5 * 2.0 ** k
    codes, e = mxfp4.quantize(x)
    assert e[0, 0] == max(k - 2, -127)
    if k >= -125:
        assert mxfp4.values(codes, e, 32)[0, 3] == x[0, 3]


def test_mxfp4_not_a_number():
    x = np.ones((2, 40))
    x[1, 35] = np.inf
    v = mxfp4.values(*mxfp4.quantize(x), 40)
    assert np.isfinite(v[0]).all() and np.isfinite(v[1, :32]).all() and np.isnan(v[1, 32:]).all()


def test_mxfp4_scale_images_hold_every_scale_once():
    rows, blocks = 300, 6
    at = {mxfp4.scale_image_index(r, b, blocks) for r in range(rows) for b in range(blocks)}
    assert len(at) == rows * blocks and max(at) < 3 * 2 * 512
    assert mxfp4.scale_image_index(33, 5, blocks) == 512 + 16 + 4 + 1


@pytest.mark.parametrize("post", [0, 1, 2])
@pytest.mark.parametrize("pre", [0, 1, 2])
@pytest.mark.parametrize("rows_per_gate", [0, 1, 2, 5])
def test_resnorm_gradients_are_differences(post, pre, rows_per_gate):
    r = np.random.RandomState(3)
    rows, c, eps, scale = 5, 8, 1e-3, 0.5
    x, b, dh, dy = (r.randn(rows, c) for _ in range(4))
    gates = 1 if rows_per_gate == 0 else -(-rows // rows_per_gate)
    gate = r.randn(gates, c)
    params = [1 + 0.1 * r.randn(c), r.randn(c), 1 + 0.1 * r.randn(c), r.randn(c)]

    def loss(x, b, gate, *params):
        f = resnorm.forward(x, b, gate, rows_per_gate, post, pre, params, scale, eps)
        return (f["h"] * dh).sum() + (0.0 if f["y"] is None else (f["y"] * dy).sum())

    f = resnorm.forward(x, b, gate, rows_per_gate, post, pre, params, scale, eps)
    g = resnorm.backward(f, dh, dy, rows_per_gate, post, pre, params, scale)
    leaves = [x, b, gate, *params]
    for i, name in enumerate(["dx", "db", "dgate", "dpost_gamma", "dpost_beta", "dpre_gamma", "dpre_beta"]):
        if name not in g:
            continue
        for at in np.ndindex(leaves[i].shape):
            moved = []
            for step in (1e-5, -1e-5):
                t = [v.copy() for v in leaves]
                t[i][at] += step
                moved.append(loss(*t))
            want = g[name].reshape(leaves[i].shape)[at]
            assert abs((moved[0] - moved[1]) / 2e-5 - want) <= 1e-6 * (1 + abs(want))


def test_norm_clip_and_update_by_hand():
    grads = [np.array([3.0, 0.0]), np.zeros(0), np.array([-4.0])]
    assert optim.grad_norm(grads) == 5.0 and optim.grad_norm(grads, inf=True) == 4.0 and optim.grad_norm([]) == 0.0
    assert optim.clip_factor(5.0, 10.0) == 1.0 and abs(optim.clip_factor(5.0, 1.0) - 0.2) < 1e-7
    theta, m, v = optim.adamw(np.array([1.0]), np.array([2.0]), np.zeros(1), np.zeros(1), 1, 0.1, 0.9, 0.999, 0.0, 0.5)
    assert abs(m[0] - 0.2) < 1e-15 and abs(v[0] - 0.004) < 1e-15 and abs(theta[0] - (1.0 - 0.1 * (1.0 + 0.5))) < 1e-12
