"""Refusals and sizes of the many-tensor, residual-and-norm and 4-bit calls, which need no GPU: nothing is launched."""
import ctypes

import pytest
import torch

from paper_2411_00288_b200 import api

NULL, BAD, SHAPE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


def _arrays(*lists):
    return [(ctypes.c_void_p * max(1, len(v)))(*v) for v in lists]


def _counts(*n):
    return (ctypes.c_int64 * max(1, len(n)))(*n)


def _types(*t):
    return (ctypes.c_int32 * max(1, len(t)))(*t)


def _norm(g, n, types=None, tensors=None, kind=0, norm=4, ws=8, ws_bytes=1 << 20):
    a, = _arrays(g)
    f = api.lib().ssconv_grad_norm
    return f(a, n, types, len(g) if tensors is None else tensors, kind, norm, ws, ws_bytes, None)


def test_grad_norm_refuses():
    assert _norm([16], _counts(4), kind=2) == BAD
    assert _norm([16], _counts(-1)) == BAD
    assert _norm([16], _counts(4), tensors=-1) == BAD
    assert _norm([16], _counts(4), types=_types(7)) == BAD
    assert _norm([None], _counts(4)) == NULL
    assert _norm([16], _counts(4), norm=None) == NULL
    assert _norm([18], _counts(4)) == ALIGN                      # half an element
    assert _norm([17], _counts(4), types=_types(1)) == ALIGN
    assert _norm([16], _counts(4), norm=6) == ALIGN
    assert _norm([16], _counts(4), ws=12) == ALIGN
    assert _norm([16], _counts((1 << 40) + 1)) == SHAPE
    assert _norm([16, 16], _counts(1 << 40, 1 << 40)) == SHAPE
    assert _norm([16], _counts(4), ws=None) == WORKSPACE
    assert _norm([16], _counts(4), ws_bytes=8) == WORKSPACE


def test_grad_norm_scratch_grows_with_launches():
    one, many = api.ssconv_grad_norm_ws_bytes(1), api.ssconv_grad_norm_ws_bytes(5000)
    assert 0 < one < many and one % 8 == 0
    assert api.ssconv_grad_norm_ws_bytes(0) > 0
    with pytest.raises(api.SsconvError):
        api.ssconv_grad_norm_ws_bytes(-1)


def _clip(g, out, n, types=None, norm=4, max_norm=1.0):
    a, b = _arrays(g, out)
    f = api.lib().ssconv_clip_grads
    return f(a, b, n, types, len(g), norm, max_norm, None)


def test_clip_refuses():
    assert _clip([], [], _counts()) == 0                         # nothing to do
    assert _clip([16], [16], _counts(4), max_norm=-1.0) == BAD
    assert _clip([16], [16], _counts(4), max_norm=float("nan")) == BAD
    assert _clip([16], [16], _counts(4), norm=None) == NULL
    assert _clip([16], [None], _counts(4)) == NULL
    assert _clip([16], [18], _counts(4)) == ALIGN
    # written twice, or written where another tensor is read
    assert _clip([16, 16], [16, 16], _counts(4, 4)) == BAD
    assert _clip([16, 64], [128, 140], _counts(4, 4)) == BAD
    assert _clip([16, 64], [64, 128], _counts(4, 4)) == BAD
    assert _clip([16], [20], _counts(4)) == BAD


def _adamw(theta, g, m, v, n, types=None, step=1, beta1=0.9, beta2=0.999, eps=1e-8, norm=None, max_norm=1.0):
    a = _arrays(theta, g, m, v)
    f = api.lib().ssconv_adamw_multi
    return f(*a, n, types, len(theta), step, 1.0, beta1, beta2, eps, 0.0, norm, max_norm, None)


def test_adamw_multi_refuses():
    ok = ([64], [128], [192], [256])
    assert _adamw([], [], [], [], _counts()) == 0
    assert _adamw(*ok, _counts(4), step=0) == BAD
    assert _adamw(*ok, _counts(4), beta1=1.0) == BAD
    assert _adamw(*ok, _counts(4), beta2=-0.1) == BAD
    assert _adamw(*ok, _counts(4), eps=float("nan")) == BAD
    assert _adamw(*ok, _counts(4), norm=4, max_norm=-1.0) == BAD
    assert _adamw(*ok, _counts(4), norm=6) == ALIGN
    assert _adamw([64], [128], [192], [258], _counts(4)) == ALIGN
    assert _adamw([64], [130], [192], [256], _counts(4)) == ALIGN
    assert _adamw([64], [128], [192], [None], _counts(4)) == NULL
    assert _adamw([64], [128], [192], [192], _counts(4)) == BAD
    assert _adamw([64], [64], [192], [256], _counts(4)) == BAD   # gradients are read, not written
    assert _adamw([64, 64], [128, 160], [192, 224], [256, 288], _counts(4, 4)) == BAD


def _desc(**k):
    return api.make_resnorm(**{**dict(rows=8, C=64), **k})


def _forward(d, x=16, b=16, gate=None, params=(None,) * 4, h=16, y=32, stats=None):
    f = api.lib().ssconv_residual_norm
    return f(ctypes.byref(d) if d else None, x, b, gate, *params, h, y, stats, None)


def test_residual_norm_refuses():
    assert _forward(None) == NULL
    assert _forward(_desc(rows=0)) == 0
    for bad in (dict(rows=-1), dict(C=0), dict(C=-8), dict(rows_per_gate=-1), dict(post=3), dict(pre=-1), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert _forward(_desc(**bad)) == BAD
    for shape in (dict(C=12), dict(C=8200), dict(rows=(1 << 30) + 1)):
        assert _forward(_desc(**shape)) == SHAPE
    assert _forward(_desc(), x=None) == NULL
    assert _forward(_desc(), b=None) == NULL
    assert _forward(_desc(), y=None) == NULL
    assert _forward(_desc(pre=0), h=None, y=None) == NULL
    assert _forward(_desc(pre=0)) == BAD                         # y of no norm
    assert _forward(_desc(), h=32) == BAD                        # h and y in one buffer
    n = 2 * 8 * 64                                               # bytes of a tensor
    assert _forward(_desc(), x=4096, b=8192, h=4096 + 16, y=65536) == BAD
    assert _forward(_desc(), x=4096, b=8192, h=65536, y=8192 - 16) == BAD
    assert _forward(_desc(), x=4096, b=8192, h=65536, y=65536 + n - 16) == BAD
    assert _forward(_desc(), x=24) == ALIGN
    assert _forward(_desc(), gate=24) == ALIGN
    assert _forward(_desc(), params=(None, None, 24, None)) == ALIGN
    assert _forward(_desc(), stats=24) == ALIGN


def _backward(d, x=16, b=16, stats=16, dh=16, dy=16, gate=None, params=(None,) * 3, dx=16, db=16, sums=(None,) * 5, ws=16, ws_bytes=1 << 30):
    f = api.lib().ssconv_residual_norm_backward
    return f(ctypes.byref(d) if d else None, x, b, stats, dh, dy, gate, *params, dx, db, *sums, ws, ws_bytes, None)


def test_residual_norm_backward_refuses():
    assert _backward(None) == NULL
    assert _backward(_desc(rows=0), x=None, ws=None) == 0
    assert _backward(_desc(C=20)) == SHAPE
    assert _backward(_desc(), dy=None) == NULL
    assert _backward(_desc(pre=0), dh=None, dy=None) == NULL
    assert _backward(_desc(), stats=None) == NULL
    assert _backward(_desc(), b=None) == NULL
    assert _backward(_desc(), sums=(None, 16, None, None, None)) == BAD   # a gradient of a norm that is not there
    assert _backward(_desc(pre=0, post=1), sums=(None, None, None, None, 16)) == BAD
    far = dict(x=4096, b=8192, dh=16384, dy=32768, dx=65536, db=131072)
    for name in ("dx", "db"):
        for other in ("x", "b", "dh", "dy", "dx", "db"):
            if other != name:
                assert _backward(_desc(), **{**far, name: far[other]}) == BAD
                assert _backward(_desc(), **{**far, name: far[other] + 16}) == BAD
    assert _backward(_desc(), dx=8) == ALIGN
    assert _backward(_desc(), **far, ws=None) == WORKSPACE
    assert _backward(_desc(), **far, ws_bytes=16) == WORKSPACE


@pytest.mark.parametrize("rows,rows_per_gate,c", [(1, 0, 8), (7, 7, 96), (7, 100, 96), (1 << 20, 1, 8), (401408, 0, 96), (401408, 3136, 96),
                                                  (25088, 196, 384), (12345, 77, 8192), (1 << 30, 0, 8), (1 << 30, 5, 8)])
def test_residual_norm_scratch_is_bounded(rows, rows_per_gate, c):
    need = api.ssconv_residual_norm_ws_bytes(_desc(rows=rows, C=c, rows_per_gate=rows_per_gate))
    assert 0 < need <= 148 * 16 * 6 * c * 4 + 4 * c * min(rows, 148 * 64)
    assert api.ssconv_residual_norm_ws_bytes(_desc(rows=0)) == 0


def test_mxfp4_sizes():
    assert api.ssconv_sizes_mxfp4(0, 32) == (0, 0)
    assert api.ssconv_sizes_mxfp4(1, 8) == (16, 512)
    assert api.ssconv_sizes_mxfp4(129, 136) == (129 * 80, 2 * 2 * 512)
    for rows, c in ((-1, 32), (4, 0)):
        with pytest.raises(api.SsconvError) as e:
            api.ssconv_sizes_mxfp4(rows, c)
        assert e.value.status == BAD
    for rows, c in ((4, 12), (1 << 31, 32)):
        with pytest.raises(api.SsconvError) as e:
            api.ssconv_sizes_mxfp4(rows, c)
        assert e.value.status == SHAPE


def test_mxfp4_refuses():
    lib = api.lib()
    assert lib.ssconv_quantize_mxfp4(None, 0, 32, None, None, None) == 0
    assert lib.ssconv_quantize_mxfp4(16, 4, 32, 16, None, None) == NULL
    assert lib.ssconv_quantize_mxfp4(8, 4, 32, 16, 16, None) == ALIGN
    assert lib.ssconv_quantize_mxfp4(16, 4, 20, 16, 16, None) == SHAPE
    assert lib.ssconv_dequantize_mxfp4(16, 8, 4, 32, 16, None) == ALIGN
    assert lib.ssconv_dequantize_mxfp4(16, 16, 4, 32, None, None) == NULL

    def forward(bias=16, x=16, y=16, **k):
        d = api.make_desc(**{**dict(N=2, H=7, W=7, C_in=64, C_out=64, KH=1, KW=1), **k})
        return lib.ssconv_forward_dense_mxfp4(ctypes.byref(d), x, 16, 16, 16, bias, y, None, None)

    for shape in (dict(KH=3, KW=3, pad=1), dict(stride=2), dict(pad=1), dict(C_in=12), dict(C_out=12), dict(KW=2)):
        assert forward(**shape) == SHAPE
    assert forward(relu=True, gelu=True) == BAD
    assert forward(bias=None) == NULL
    assert forward(x=None) == NULL
    assert forward(x=8) == ALIGN
    assert forward(y=8) == ALIGN
    assert lib.ssconv_forward_dense_mxfp4(None, 16, 16, 16, 16, None, 16, None, None) == NULL


def test_python_calls_refuse_what_is_not_on_the_gpu():
    x = torch.zeros(4, 32, dtype=torch.bfloat16)
    f = torch.zeros(8)
    with pytest.raises(ValueError):
        api.ssconv_quantize_mxfp4(x)
    with pytest.raises(TypeError):
        api.ssconv_quantize_mxfp4(x.float())
    with pytest.raises(ValueError):
        api.ssconv_residual_norm(api.make_resnorm(4, 32), x, x)
    with pytest.raises(TypeError):
        api.ssconv_residual_norm(api.make_resnorm(4, 32), x.float(), x)
    with pytest.raises(ValueError):
        api.ssconv_residual_norm(api.make_resnorm(5, 32), x, x)   # other extents
    with pytest.raises(ValueError):
        api.ssconv_grad_norm([f])
    with pytest.raises(ValueError):
        api.ssconv_grad_norm([])
    with pytest.raises(ValueError):
        api.ssconv_clip_grads([f], f[:1], 1.0)
    with pytest.raises(TypeError):
        api.ssconv_adamw_multi([1], [2], [3], [4], 1)
    with pytest.raises(ValueError):
        api.ssconv_dequantize_mxfp4(x.view(torch.uint8), f.view(torch.uint8), 40)


def test_refuses_overlaps_of_what_is_written():
    """Every written buffer against every other one of its call; launches nothing, so any addresses will do."""
    f = api.lib()
    K = 1 << 20
    assert _norm([K], _counts(4), norm=K + 12, ws=64 * K) == BAD        # the norm inside a gradient
    assert _norm([K], _counts(4), norm=2 * K, ws=K - 8) == BAD          # the scratch reaches into one
    assert _norm([K], _counts(4), norm=64 * K + 4, ws=64 * K) == BAD    # the norm inside the scratch
    g, out = _arrays([K], [2 * K])
    assert f.ssconv_clip_grads(g, out, _counts(4), None, 1, 2 * K + 4, 1.0, None) == BAD
    theta, g, m, v = _arrays([K], [2 * K], [3 * K], [4 * K])
    assert f.ssconv_adamw_multi(theta, g, m, v, _counts(4), None, 1, 1, 1.0, 0.9, 0.999, 1e-8, 0.0, 3 * K + 4, 1.0, None) == BAD

    d = ctypes.byref(api.make_resnorm(64, 64, rows_per_gate=16, post=api.NORM_LAYER, pre=api.NORM_RMS))
    forward = [(i + 1) * K for i in range(10)]                           # x, b, gate, gammas and betas, h, y, stats
    backward = [(i + 1) * K for i in range(16)]                          # x, b, stats, dh, dy, gate, gammas, outputs, ws
    last = {"gate": 4 * 64 * 4 - 16, "row": 4 * 64 - 16, "stats": 64 * 16 - 16, "rows": 2 * 64 * 64 - 16}
    inputs = ["rows", "rows", "gate", "row", "row", "row", "row"]
    for written in (7, 8, 9):
        for other in range(10):
            if other == written:
                continue
            a = list(forward)
            size = (inputs + ["rows", "rows", "stats"])[other]
            a[written] = a[other] + last[size]                           # its first 16 bytes are the other's last ones
            assert f.ssconv_residual_norm(d, *a, None) == BAD, (written, other)
    kinds = ["rows", "rows", "stats", "rows", "rows", "gate", "row", None, "row", "rows", "rows", "gate", "row", "row", "row", "row"]
    for written in range(9, 16):
        for other in range(16):
            if other == written or kinds[other] is None:                 # (post_beta has no part in the gradients)
                continue
            a = list(backward)
            a[written] = a[other] + last[kinds[other]]
            assert f.ssconv_residual_norm_backward(d, *a, 64 * K, 1 << 30, None) == BAD, (written, other)
    for other in range(7):
        a = list(backward)
        a[other] = 64 * K + 16                                           # inside the scratch
        assert f.ssconv_residual_norm_backward(d, *a, 64 * K, 1 << 30, None) == BAD, other

    for call in (lambda a: f.ssconv_quantize_mxfp4(a[0], 4, 64, a[1], a[2], None), lambda a: f.ssconv_dequantize_mxfp4(a[1], a[2], 4, 64, a[0], None)):
        ends = (4 * 64 * 2 - 16, 4 * 32 - 16)
        assert call([K, K + ends[0], 3 * K]) == BAD
        assert call([K, 2 * K, K + ends[0]]) == BAD
    assert f.ssconv_quantize_mxfp4(K, 4, 64, 2 * K, 2 * K + 4 * 32 - 16, None) == BAD
    desc = ctypes.byref(api.make_desc(1, 2, 2, 64, 64, 1, 1, bias=True))
    base = [K, 2 * K, 3 * K, 4 * K, 5 * K, 6 * K, 7 * K]                 # codes and scales of x and w, bias, y, dev_status
    ends = [4 * 32, 512, 64 * 32, 512, 64 * 4, 4 * 64 * 2]
    for other in range(5):
        a = list(base)
        a[5] = a[other] + ends[other] - 16
        assert f.ssconv_forward_dense_mxfp4(desc, *a, None) == BAD, other
    for other in range(6):
        a = list(base)
        a[6] = a[other] + ends[other] - 4
        assert f.ssconv_forward_dense_mxfp4(desc, *a, None) == BAD, other


@pytest.mark.parametrize("order", ["ascending", "descending", "interleaved", "shuffled"])
def test_adamw_finds_one_overlap_among_many_tensors(order):
    """4 lists of 97 tensors, 4096 bytes apart, of which one reaches into its neighbour: refused wherever it is."""
    lists, count = 4, 97
    at = [(1 << 30) + 4096 * i for i in range(lists * count)]
    if order == "interleaved":
        rows = [at[k::lists] for k in range(lists)]
    else:
        if order == "descending":
            at.reverse()
        elif order == "shuffled":
            at = [at[(37 * i + 11) % len(at)] for i in range(len(at))]
        rows = [at[k * count:(k + 1) * count] for k in range(lists)]
    assert len({a for r in rows for a in r}) == lists * count
    f = api.lib().ssconv_adamw_multi
    for which in range(lists):
        for i in (0, 1, 48, count - 1):
            moved = [list(r) for r in rows]
            step = 4096 if moved[which][i] + 4096 in at else -4096
            if which == 1 and moved[which][i] + step in rows[1]:         # (two gradients, both only read)
                continue
            moved[which][i] += step * (4096 - 16) // 4096
            theta, g, m, v = _arrays(*moved)
            assert f(theta, g, m, v, _counts(*[1024 - 4] * count), None, count, 1, 1.0, 0.9, 0.999, 1e-8, 0.0, None, 1.0, None) == BAD


def test_mxfp4_sizes_of_the_longest_rows():
    """ceil(C / 32) and ceil(C / 128) up to the last C of 31 bits."""
    for c in (2147483520, 2147483528, 2147483608, 2147483616, 2147483640):
        for rows in (1, 127, 4000):
            assert api.ssconv_sizes_mxfp4(rows, c) == (rows * -(-c // 32) * 16, -(-rows // 128) * -(-c // 128) * 512)
    for rows, c in ((128 * 128 + 1, 2147483640), (2147483392, 128 * 129)):  # 2^31 scale images and more
        with pytest.raises(api.SsconvError) as e:
            api.ssconv_sizes_mxfp4(rows, c)
        assert e.value.status == SHAPE


def test_kinds_of_norm_beyond_31_bits_are_refused():
    with pytest.raises(ValueError, match="kind"):
        api.ssconv_grad_norm([], kind=1 << 32)


def test_plan_of_the_4_bit_product():
    def plan(rows, cin, cout, sms=148, pairs=70, **k):
        return api.ssconv_plan_mxfp4(api.make_desc(rows, 1, 1, cin, cout, 1, 1, **k), sms, pairs)

    assert plan(1, 2048, 1000) == dict(columns=64, pair=False, ctas=16)
    assert plan(401408, 96, 384) == dict(columns=192, pair=False, ctas=148)
    assert plan(6000, 4096, 1536) == dict(columns=192, pair=True, ctas=140)
    assert plan(401408, 96, 384, sms=100, pairs=50) == dict(columns=192, pair=False, ctas=100)
    for bad, status in ((dict(sms=-1), BAD), (dict(pairs=0), BAD), (dict(rows=0), BAD), (dict(cin=12), SHAPE), (dict(relu=True, gelu=True), BAD)):
        with pytest.raises(api.SsconvError) as e:
            plan(**{**dict(rows=4, cin=64, cout=64), **bad})
        assert e.value.status == status
    assert api.lib().ssconv_plan_mxfp4(None, 148, 70, None, None, None) == NULL
    d = ctypes.byref(api.make_desc(4, 1, 1, 64, 64, 1, 1))
    assert api.lib().ssconv_plan_mxfp4(d, 148, 70, None, None, None) == 0
    assert api.lib().ssconv_plan_mxfp4(ctypes.byref(api.make_desc(4, 3, 3, 64, 64, 3, 3, pad=1)), 148, 70, None, None, None) == SHAPE
