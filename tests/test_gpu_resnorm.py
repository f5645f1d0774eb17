"""The end of a block (norms before and after, gate, scaled residual) and its gradients against 64-bit arithmetic.

Tolerances, in units of u = 2^-24.  A sum along a row of C channels adds at most 16 numbers per thread, then 5 levels of a warp
and 16 warps: its error is at most 40 u of the sum of magnitudes.  A mean is off by 42 u of the row's largest magnitude, so is a
centred value; its square and their mean by 128 u relative to the mean square, 1/deviation by 68 u with its own two units: a
normalised value by 128 u of (|v - mean| + the row's largest magnitude) / deviation.  Whatever is stored as bf16 is off by 2^-8 of
itself in addition.  Sums over rows carry their terms' errors and at most one u per row."""
import itertools

import numpy as np
import pytest
import torch

from oracle import resnorm
from paper_2411_00288_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
NONE, LAYER, RMS = api.NORM_NONE, api.NORM_LAYER, api.NORM_RMS


def _f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


class Case:
    def __init__(self, rows, c, rows_per_gate=0, gate=True, post=LAYER, pre=LAYER, affine=True, scale=0.5, eps=1e-6, seed=0, mean=0.25):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def randn(*shape):
            return torch.randn(shape, generator=g, device=DEV)

        self.desc = api.make_resnorm(rows, c, rows_per_gate=rows_per_gate, post=post, pre=pre, scale=scale, eps=eps)
        self.rows, self.c, self.rpg, self.post, self.pre, self.scale, self.eps = rows, c, rows_per_gate, post, pre, scale, eps
        self.x, self.b = (randn(rows, c) + mean).bfloat16(), (2 * randn(rows, c) + mean).bfloat16()
        self.dh, self.dy = randn(rows, c).bfloat16(), randn(rows, c).bfloat16() if pre != NONE else None
        gates = 1 if rows_per_gate == 0 else -(-rows // rows_per_gate)
        self.gate = (0.3 + 0.5 * randn(gates, c)) if gate else None
        self.params = [None] * 4
        if affine and post != NONE:
            self.params[:2] = [1 + 0.1 * randn(c), 0.1 * randn(c)]
        if affine and pre != NONE:
            self.params[2:] = [1 + 0.1 * randn(c), 0.1 * randn(c)]

    def named(self):
        return dict(zip(("post_gamma", "post_beta", "pre_gamma", "pre_beta"), self.params), gate=self.gate)

    def forward(self, **k):
        return api.ssconv_residual_norm(self.desc, self.x, self.b, want_stats=True, **self.named(), **k)

    def backward(self, stats, dh="own", **k):
        return api.ssconv_residual_norm_backward(self.desc, self.x, self.b, stats, self.dh if dh == "own" else dh, self.dy, **self.named(), **k)

    def exact(self):
        gate = None if self.gate is None else _f64(self.gate)
        return resnorm.forward(_f64(self.x), _f64(self.b), gate, self.rpg, self.post, self.pre, [_f64(p) for p in self.params], self.scale,
                               np.float64(np.float32(self.eps)))

    def magnitudes(self, f):
        """Bounds of what the roundings of p, h, y, bhat and hhat are relative to."""
        mag = {}
        p = np.abs(_f64(self.b))
        one = [np.ones(self.c) if q is None else np.abs(_f64(q)) for q in self.params]
        zero = [np.zeros(self.c) if q is None else np.abs(_f64(q)) for q in self.params]
        mag["bhat"] = p
        if self.post != NONE:
            mag["bhat"] = (2 * p + p.max(-1, keepdims=True)) * f["rb"]
            p = mag["bhat"] * one[0] + zero[1]
        mag["p"] = p
        mag["h"] = self.scale * np.abs(_f64(self.x)) + np.abs(f["gate"]) * p
        if self.pre != NONE:
            mag["hhat"] = (2 * mag["h"] + mag["h"].max(-1, keepdims=True)) * f["rh"]
            mag["y"] = mag["hhat"] * one[2] + zero[3]
        return mag


def _near(got, want, mag, units, stored_bf16=True):
    got = _f64(got)
    tol = units * U * mag + (2.0 ** -8 * np.abs(want) if stored_bf16 else 0.0) + 2.0 ** -130
    assert got.shape == want.shape and np.isfinite(got).all()
    worst = np.max(np.abs(got - want) / tol)
    assert worst <= 1.0, worst


def _check_forward(case, h, y, stats, f, mag):
    _near(h, f["h"], mag["h"], 256)
    if case.pre == NONE:
        assert y is None
    else:
        _near(y, f["y"], mag["y"], 512)


def _check_backward(case, g, f, mag, with_dh=True):
    dh, dy = _f64(case.dh) if with_dh else np.zeros((case.rows, case.c)), _f64(case.dy)
    want = resnorm.backward(f, dh if with_dh else None, dy, case.rpg, case.post, case.pre, [_f64(p) for p in case.params], case.scale)

    def through(t, hat, r):
        return r * (t + t.mean(-1, keepdims=True) + hat * (t * hat).mean(-1, keepdims=True))

    d = np.abs(dh)
    if case.pre != NONE:
        gamma = np.ones(case.c) if case.params[2] is None else np.abs(_f64(case.params[2]))
        d = d + through(np.abs(dy) * gamma, np.maximum(mag["hhat"], np.abs(f["hhat"])), f["rh"])
    _near(g.dx, want["dx"], case.scale * d, 1024)
    db = dp = d * np.abs(f["gate"])
    if case.post != NONE:
        gamma = np.ones(case.c) if case.params[0] is None else np.abs(_f64(case.params[0]))
        db = through(dp * gamma, mag["bhat"], f["rb"])
    _near(g.db, want["db"], db, 2048)

    def summed(got, want, terms, units, groups=None):
        if got is None:
            return
        total = terms.sum(0) if groups is None else np.add.reduceat(terms, np.arange(0, terms.shape[0], groups), axis=0)
        got = got if groups else got.reshape(-1)
        _near(got, want, total, units + min(case.rows, groups or case.rows), stored_bf16=False)

    assert (g.dgate is None) == (case.gate is None)
    summed(g.dgate, want["dgate"], d * mag["p"], 1400, case.rpg or None)
    if case.post != NONE:
        summed(g.dpost_gamma, want["dpost_gamma"], dp * mag["bhat"], 1400)
        summed(g.dpost_beta, want["dpost_beta"], dp, 1100)
    if case.pre != NONE:
        summed(g.dpre_gamma, want["dpre_gamma"], np.abs(dy) * mag["hhat"], 600)
        summed(g.dpre_beta, want["dpre_beta"], np.abs(dy), 0)


def _check(case):
    h, y, stats = case.forward()
    f = case.exact()
    mag = case.magnitudes(f)
    _check_forward(case, h, y, stats, f, mag)
    _check_backward(case, case.backward(stats), f, mag)
    if case.pre != NONE:
        _check_backward(case, case.backward(stats, dh=None), f, mag, with_dh=False)


@pytest.mark.parametrize("post,pre", list(itertools.product([NONE, LAYER, RMS], repeat=2)))
@pytest.mark.parametrize("c", [8, 24, 96, 256, 264, 384, 512, 520, 768, 1000, 1024, 1032])
def test_norms_of_every_kind_and_width(c, post, pre):
    _check(Case(37, c, post=post, pre=pre, seed=c))


# (past four rows per SM the rows of up to 768 channels are dealt to warps with several pieces per lane)
@pytest.mark.parametrize("post,pre", [(NONE, LAYER), (RMS, NONE), (LAYER, RMS), (LAYER, LAYER), (NONE, NONE)])
@pytest.mark.parametrize("c", [8, 16, 40, 48, 64, 88, 96, 120, 128, 192, 256, 264, 320, 384, 512, 520, 680, 768, 776])
def test_many_rows_of_every_width(c, post, pre):
    _check(Case(733, c, rows_per_gate=50 if c % 16 else 0, post=post, pre=pre, seed=c))


@pytest.mark.parametrize("c", [2048, 4096, 4104, 8192])
@pytest.mark.parametrize("post,pre", [(LAYER, RMS), (NONE, LAYER), (RMS, NONE), (LAYER, LAYER)])
def test_wide_rows(c, post, pre):
    _check(Case(5, c, post=post, pre=pre, seed=c))


# (blocks take two rows at a time where there are many)
@pytest.mark.parametrize("c", [1544, 2048, 3584, 4096])
@pytest.mark.parametrize("rows,per", [(1201, 0), (1202, 7), (1999, 1), (1201, 600)])
def test_many_wide_rows(c, rows, per):
    _check(Case(rows, c, rows_per_gate=per, post=LAYER, pre=RMS, seed=rows + c))


@pytest.mark.parametrize("c", [8, 24, 2504])
@pytest.mark.parametrize("post,pre", [(RMS, LAYER), (LAYER, NONE)])
def test_sums_over_few_images(c, post, pre):
    _check(Case(1300, c, rows_per_gate=433, post=post, pre=pre, seed=c))


@pytest.mark.parametrize("rows", [1, 2, 3, 31, 33, 257, 3001])
@pytest.mark.parametrize("c", [8, 40, 136, 776])
def test_numbers_of_rows(rows, c):
    _check(Case(rows, c, seed=rows))


@pytest.mark.parametrize("c", [16, 96, 512, 528])
@pytest.mark.parametrize("rows,per", [(1, 1), (50, 1), (700, 1), (2500, 2), (2500, 3), (61 * 17, 17), (100, 49), (3000, 1000), (3001, 1000), (20, 500), (6000, 5999)])
def test_gates_per_image(rows, per, c):
    _check(Case(rows, c, rows_per_gate=per, post=LAYER, pre=RMS, seed=rows + c))


@pytest.mark.parametrize("c", [64, 640])
@pytest.mark.parametrize("per", [0, 7])
def test_without_gates_or_parameters(c, per):
    _check(Case(50, c, rows_per_gate=per, gate=False))
    _check(Case(50, c, rows_per_gate=per, affine=False))
    _check(Case(50, c, rows_per_gate=per, gate=False, affine=False, post=NONE, pre=NONE))


@pytest.mark.parametrize("c", [96, 768])
@pytest.mark.parametrize("mean", [0.0, 100.0])
def test_means_far_from_zero(c, mean):
    _check(Case(64, c, mean=mean, gate=False, scale=1.0))


@pytest.mark.parametrize("c", [32, 800])
def test_rows_without_spread_and_of_zeros(c):
    case = Case(6, c, post=LAYER, pre=LAYER, eps=1e-3)
    case.b[0] = 0
    case.b[1] = 3.0
    case.x[2] = 0
    _check(case)


def test_more_rows_than_the_grid_takes_at_once():
    for c, per in ((32, 0), (96, 3), (1032, 0)):
        rows = 200_000 if c < 1000 else 5000
        case = Case(rows, c, rows_per_gate=per, post=RMS, pre=LAYER)
        h, y, stats = case.forward()
        f = case.exact()
        mag = case.magnitudes(f)
        _check_forward(case, h, y, stats, f, mag)
        _check_backward(case, case.backward(stats), f, mag)


@pytest.mark.parametrize("c", [48, 1000])
@pytest.mark.parametrize("into", ["x", "b"])
def test_in_place(c, into):
    case = Case(300, c)
    h, y, stats = case.forward()
    x, b = case.x.clone(), case.b.clone()
    other = {"x": b, "b": x}[into]
    h2, y2, s2 = api.ssconv_residual_norm(case.desc, x, b, want_stats=True, h={"x": x, "b": b}[into], y=other, **case.named())
    assert torch.equal(h, h2) and torch.equal(y, y2) and torch.equal(stats, s2)


def test_only_the_second_norm_or_only_the_sum():
    case = Case(40, 96)
    h, y, _ = case.forward()
    y2 = torch.empty_like(y)
    f = api.lib().ssconv_residual_norm
    pg, pb, qg, qb = (p.data_ptr() for p in case.params)
    rc = f(api.ctypes.byref(case.desc), case.x.data_ptr(), case.b.data_ptr(), case.gate.data_ptr(), pg, pb, qg, qb, None, y2.data_ptr(), None,
           torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(y, y2)


@pytest.mark.parametrize("c", [96, 768])
@pytest.mark.parametrize("kept", range(7))
def test_each_gradient_by_itself(c, kept):
    case = Case(123, c, rows_per_gate=10)
    stats = case.forward()[2]
    whole = case.backward(stats)
    names = ["dx", "db", "dgate", "dpost_gamma", "dpost_beta", "dpre_gamma", "dpre_beta"]
    out = [None] * 7
    out[kept] = torch.empty_like(getattr(whole, names[kept]))
    ws = torch.empty(api.ssconv_residual_norm_ws_bytes(case.desc), dtype=torch.uint8, device=DEV)
    f = api.lib().ssconv_residual_norm_backward
    rc = f(api.ctypes.byref(case.desc), *(t.data_ptr() for t in (case.x, case.b, stats, case.dh, case.dy, case.gate, *case.params[:3])),
           *(None if t is None else t.data_ptr() for t in out), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(out[kept], getattr(whole, names[kept]))


def test_nan_stays_in_its_row():
    for c in (96, 1000):
        case = Case(9, c)
        case.b[4, 3] = float("nan")
        h, y, stats = case.forward()
        bad = torch.arange(9, device=DEV) == 4
        assert y[bad].isnan().all() and y[~bad].isfinite().all() and h[~bad].isfinite().all()
        g = case.backward(stats)
        assert g.dx[bad].isnan().all() and g.dx[~bad].isfinite().all() and g.db[~bad].isfinite().all()


def test_no_rows():
    desc = api.make_resnorm(0, 64, post=LAYER, pre=RMS)
    x = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    gamma = torch.ones(64, device=DEV)
    h, y, stats = api.ssconv_residual_norm(desc, x, x, post_gamma=gamma, pre_gamma=gamma, want_stats=True)
    g = api.ssconv_residual_norm_backward(desc, x, x, stats, x, x, gate=gamma, post_gamma=gamma, pre_gamma=gamma, pre_beta=gamma)
    assert h.shape == x.shape and g.dpost_beta is None
    assert all((t == 0).all() for t in (g.dgate, g.dpost_gamma, g.dpre_gamma, g.dpre_beta))


@pytest.mark.parametrize("c,per", [(96, 0), (96, 49), (1000, 7)])
def test_captured_and_on_another_stream(c, per):
    case = Case(490, c, rows_per_gate=per)
    h, y, stats = case.forward()
    want = case.backward(stats)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h2, y2, s2 = case.forward(stream=side)
    got = case.backward(s2, stream=side)
    torch.cuda.synchronize()
    same = [(h, h2), (y, y2), (stats, s2)] + [(getattr(want, k), getattr(got, k)) for k in vars(want)]
    assert all(torch.equal(a, b) for a, b in same)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h3, y3, s3 = case.forward()
        g3 = case.backward(s3)
    case.x.copy_(case.x.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    f = case.exact()
    mag = case.magnitudes(f)
    _check_forward(case, h3, y3, s3, f, mag)
    _check_backward(case, g3, f, mag)


def test_gradients_are_the_same_every_time():
    case = Case(20_011, 96, rows_per_gate=300)
    stats = case.forward()[2]
    first = case.backward(stats)
    for _ in range(5):
        again = case.backward(stats)
        assert all(torch.equal(getattr(first, k), getattr(again, k)) for k in vars(first))


def test_refusals():
    case = Case(12, 64)
    with pytest.raises(ValueError):
        api.ssconv_residual_norm(case.desc, case.x[:6], case.b)
    with pytest.raises(ValueError):
        api.ssconv_residual_norm(case.desc, case.x, case.b, gate=torch.ones(2, 64, device=DEV))
    with pytest.raises(ValueError):
        api.ssconv_residual_norm(case.desc, case.x, case.b, pre_gamma=torch.ones(32, device=DEV))
    with pytest.raises(TypeError):
        api.ssconv_residual_norm(case.desc, case.x, case.b, gate=torch.ones(64, device=DEV, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        api.ssconv_residual_norm(case.desc, case.x.t().contiguous().t(), case.b)
    stats = case.forward()[2]
    with pytest.raises(api.SsconvError):
        api.ssconv_residual_norm_backward(case.desc, case.x, case.b, None, case.dh, case.dy)
    with pytest.raises(api.SsconvError):
        api.ssconv_residual_norm_backward(case.desc, case.x, case.b, stats, case.dh, None)
    with pytest.raises(api.SsconvError):
        case.backward(stats, ws=torch.empty(64, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("per", [40, 41, 1 << 31, (1 << 63) - 1])
def test_one_row_of_gates_for_more_rows_than_there_are(per):
    one, all_rows = Case(40, 96, rows_per_gate=per), Case(40, 96)
    assert all(torch.equal(s, t) for s, t in zip((one.x, one.b, one.gate, *one.params), (all_rows.x, all_rows.b, all_rows.gate, *all_rows.params)))
    for a, b in zip(one.forward(), all_rows.forward()):
        assert torch.equal(a, b)
    stats = one.forward()[2]
    a, b = one.backward(stats), all_rows.backward(stats)
    assert a.dgate.shape == (1, 96)
    _check(one)
    assert torch.equal(a.dx, b.dx) and torch.equal(a.db, b.db)
