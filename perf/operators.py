"""The operators around a network's convolutions that are timed and compared with their plain forms, as a training step or a
4-bit forward pass calls them.

Kinds of case
  clip       the norm over all gradients of a step, and the gradients scaled down to it
  adamw      the same norm, then AdamW on every tensor with the clipped gradients
  resnorm    the end of a block: norm of its output, gate, scaled residual, the next block's norm; forward, or a training step
  quantize   activations to microscaled 4-bit values (blocks of 32 channels) and back
  pointwise  a 1x1 convolution in 4 bits: activations quantised on the way in, weights quantised once
"""
import itertools
import math
import random

import torch

own = False

DEV = "cuda:0"
CLIP_EPS = 1e-6
EPS = 1e-6
BETA1, BETA2, ADAM_EPS, DECAY, LR, STEP = 0.9, 0.999, 1e-8, 1e-4, 1e-2, 7
BLOCK = 32                       # channels of one scale


def _clip(name, tensors, total, dtype="f32", norm="l2", max_norm=1.0):
    return dict(name=name, kind="clip", tensors=tensors, total=total, dtype=dtype, norm=norm, max_norm=max_norm)


def _adamw(name, tensors, total, dtype="f32", max_norm=1.0):
    return dict(name=name, kind="adamw", tensors=tensors, total=total, dtype=dtype, max_norm=max_norm)


def _resnorm(name, images, pixels, c, gate, post, pre, train, scale=1.0):
    return dict(name=name, kind="resnorm", images=images, pixels=pixels, c=c, gate=gate, post=post, pre=pre, train=train, scale=scale)


def _quantize(name, rows, c):
    return dict(name=name, kind="quantize", rows=rows, c=c)


def _pointwise(name, rows, cin, cout, act):
    return dict(name=name, kind="pointwise", rows=rows, cin=cin, cout=cout, act=act)


def listed():
    return [
        # biases and norm scales of a few layers: a call's latency
        _clip("clip_24_small", 24, 9_001),
        # the choice weights of the ResNet-50-shaped stack's 52 masked layers
        _clip("clip_r50_choices", 52, 35_168_256),
        # a few small layers' choice weights, and all of the stack's
        _adamw("adamw_20_small", 20, 300_007),
        _adamw("adamw_r50_choices", 52, 35_168_256),
        # one image's last stage: the end of a block, forward only
        _resnorm("resnorm_b1_c768", 1, 49, 768, "shared", "none", "layer", False),
        # a training step: first stage at the benchmark's batch, layer scale and the norm after it
        _resnorm("resnorm_train_c96_b128", 128, 3136, 96, "shared", "none", "layer", True),
        # a training step with both norms and a gate per image; ragged extents
        _resnorm("resnorm_train_images_c1000", 61, 197, 1000, "image", "rms", "rms", True, 0.5),
        # activations of one image, and of the first stage at the benchmark's batch
        _quantize("quantize_49x768", 49, 768),
        _quantize("quantize_401408x96", 401_408, 96),
        # the classifier of one image: latency; a block's expansion at the benchmark's batch; a large generic product
        _pointwise("pointwise_1x2048_1000", 1, 2048, 1000, "none"),
        _pointwise("pointwise_25088x384_1536", 25_088, 384, 1536, "gelu"),
        _pointwise("pointwise_8192x4096_4096", 8192, 4096, 4096, "relu"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _channels(rng, lo, hi, step=8):
    return max(lo, _log_int(rng, lo, hi) // step * step)


def draw(rng):
    have = [{k: v for k, v in c.items() if k != "name"} for c in listed()]
    while True:
        c = _draw(rng)
        if c not in have:
            return c


def _draw(rng):
    kind = rng.choice(["clip", "adamw", "resnorm", "resnorm", "quantize", "pointwise", "pointwise"])
    if kind in ("clip", "adamw"):
        tensors = _log_int(rng, 1, 200)
        c = dict(kind=kind, tensors=tensors, total=_log_int(rng, tensors, 35_000_000), dtype=rng.choice(["f32", "f32", "bf16"]),
                 max_norm=rng.choice([0.5, 1.0, 100.0]))
        if kind == "clip":
            c["norm"] = rng.choice(["l2", "l2", "inf"])
        return c
    if kind == "resnorm":
        ch = _channels(rng, 8, 4096)
        rows = _log_int(rng, 1, max(1, 38_000_000 // ch))
        images = _log_int(rng, 1, min(rows, 256))
        return dict(kind=kind, images=images, pixels=max(1, rows // images), c=ch, gate=rng.choice(["none", "shared", "image"]),
                    post=rng.choice(["none", "layer", "rms"]), pre=rng.choice(["none", "layer", "rms", "layer"]),
                    train=rng.random() < 0.6, scale=rng.choice([1.0, 0.5]))
    if kind == "quantize":
        ch = _channels(rng, 8, 4096)
        return dict(kind=kind, rows=_log_int(rng, 1, 38_000_000 // ch), c=ch)
    cin, cout = _channels(rng, 8, 4096), _channels(rng, 8, 4096)
    most = min(100_000_000_000 // (cin * cout), 30_000_000 // max(cin, cout))
    return dict(kind=kind, rows=_log_int(rng, 1, most), cin=cin, cout=cout, act=rng.choice(["none", "relu", "gelu"]))


# ----------------------------------------------------------------------------- inputs
def _sizes(c):
    """Extents of the case's tensors: spread over four decades, as biases and weights are, none empty, `total` in all."""
    r = random.Random(c["tensors"] * 1_000_003 + c["total"])
    share = [10.0 ** r.uniform(0, 4) for _ in range(c["tensors"])]
    spare = c["total"] - c["tensors"]
    sizes = [1 + int(spare * s / sum(share)) for s in share]
    sizes[0] += c["total"] - sum(sizes)
    return sizes


def _arena(sizes, dtype):
    """One zeroed buffer and a view of it per tensor, each at a multiple of 64 bytes."""
    step = 64 // torch.empty((), dtype=dtype).element_size()
    *starts, end = itertools.accumulate((-(-n // step) * step for n in sizes), initial=0)
    flat = torch.zeros(end, dtype=dtype, device=DEV)
    return flat, [flat[s:s + n] for s, n in zip(starts, sizes)]


def _mx_scale(v):
    """The scale of each block of 32 of v [..., 32]: 2^(floor(log2(largest magnitude)) - 2), at least 2^-127.  (A number over its
    own mantissa is its power of two exactly.)"""
    top = v.abs().amax(-1, keepdim=True).double()
    mantissa, _ = torch.frexp(top)
    return torch.where(top > 0, top / mantissa / 8, torch.zeros_like(top)).clamp(min=2.0 ** -127).float()


def _mx_values(x):
    """The microscaled 4-bit values of x [rows, c], in 32 bits: e2m1 elements (nearest, ties to the even code, at most 6)
    times their block's power of two."""
    rows, c = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -c % BLOCK)).view(rows, -1, BLOCK)
    scale = _mx_scale(v)
    a = v.abs() / scale
    q = 0.5 * ((a > 0.25).float() + (a >= 0.75).float() + (a > 1.25).float() + (a >= 1.75).float()) + (a > 2.5).float() + (a >= 3.5).float() + 2.0 * (a > 5.0).float()
    return (torch.copysign(q, v) * scale).view(rows, -1)[:, :c]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind = case["kind"]

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    if kind in ("clip", "adamw"):
        sizes = _sizes(case)
        dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        flat, grads = _arena(sizes, dtype)
        flat.normal_(0.0, 0.05, generator=g)
        if kind == "clip":
            out_flat, out = _arena(sizes, dtype)
            return dict(case=case, grads=grads, out=out, out_flat=out_flat)
        t_flat, theta = _arena(sizes, torch.float32)
        m_flat, m = _arena(sizes, torch.float32)
        v_flat, v = _arena(sizes, torch.float32)
        t_flat.normal_(generator=g)
        m_flat.normal_(0.0, 0.01, generator=g)
        v_flat.normal_(0.0, 0.01, generator=g).square_()
        return dict(case=case, grads=grads, theta=theta, m=m, v=v, flats=(t_flat, m_flat, v_flat))
    if kind == "resnorm":
        rows, c = case["images"] * case["pixels"], case["c"]
        s = dict(case=case, x=(randn(rows, c) + 0.25).to(torch.bfloat16), b=(randn(rows, c) * 2).to(torch.bfloat16), gate=None, post=(None, None), pre=(None, None))
        if case["gate"] != "none":
            s["gate"] = 0.3 + 0.1 * (randn(c) if case["gate"] == "shared" else randn(case["images"], c))
        for k in ("post", "pre"):
            if case[k] != "none":
                s[k] = (1.0 + 0.1 * randn(c), 0.1 * randn(c) if case[k] == "layer" else None)
        if case["train"]:
            s["dh"] = randn(rows, c).to(torch.bfloat16)
            s["dy"] = randn(rows, c).to(torch.bfloat16) if case["pre"] != "none" else None
        if own:
            from paper_2411_00288_b200 import api
            kinds = dict(none=api.NORM_NONE, layer=api.NORM_LAYER, rms=api.NORM_RMS)
            s["desc"] = api.make_resnorm(rows, c, rows_per_gate=case["pixels"] if case["gate"] == "image" else 0, post=kinds[case["post"]],
                                         pre=kinds[case["pre"]], scale=case["scale"], eps=EPS)
        return s
    if kind == "quantize":
        return dict(case=case, x=(randn(case["rows"], case["c"]) * torch.exp(randn(case["rows"], 1))).to(torch.bfloat16))
    rows, cin, cout = case["rows"], case["cin"], case["cout"]
    w = (randn(cout, cin) / math.sqrt(cin)).to(torch.bfloat16)
    s = dict(case=case, x=randn(rows, cin).to(torch.bfloat16), bias=0.1 * randn(cout))
    if own:
        from paper_2411_00288_b200 import api
        s["desc"] = api.make_desc(rows, 1, 1, cin, cout, 1, 1, bias=True, relu=case["act"] == "relu", gelu=case["act"] == "gelu")
        s["w_codes"], s["w_scales"] = api.ssconv_quantize_mxfp4(w)
    else:
        s["w"] = _mx_values(w)
    return s


# ----------------------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2411_00288_b200 import api
        return {"clip": _own_clip, "adamw": _own_adamw, "resnorm": _own_resnorm, "quantize": _own_quantize, "pointwise": _own_pointwise}[kind](api, state)
    return {"clip": _plain_clip, "adamw": _plain_adamw, "resnorm": _plain_resnorm, "quantize": _plain_quantize, "pointwise": _plain_pointwise}[kind](state)


def _own_clip(api, s):
    norm = api.ssconv_grad_norm(s["grads"], api.GRAD_NORM_L2 if s["case"]["norm"] == "l2" else api.GRAD_NORM_INF)
    api.ssconv_clip_grads(s["grads"], norm, s["case"]["max_norm"], out=s["out"])
    return dict(norm=norm, out=s["out_flat"])


def _own_adamw(api, s):
    norm = api.ssconv_grad_norm(s["grads"])
    api.ssconv_adamw_multi(s["theta"], s["grads"], s["m"], s["v"], STEP, lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY,
                           norm=norm, max_norm=s["case"]["max_norm"])
    return dict(norm=norm, flats=s["flats"])


def _own_resnorm(api, s):
    train = s["case"]["train"]
    (post_gamma, post_beta), (pre_gamma, pre_beta) = s["post"], s["pre"]
    h, y, stats = api.ssconv_residual_norm(s["desc"], s["x"], s["b"], gate=s["gate"], post_gamma=post_gamma, post_beta=post_beta, pre_gamma=pre_gamma,
                                           pre_beta=pre_beta, want_stats=train)
    if not train:
        return dict(h=h, y=y)
    grads = api.ssconv_residual_norm_backward(s["desc"], s["x"], s["b"], stats, s["dh"], s["dy"], gate=s["gate"], post_gamma=post_gamma,
                                              post_beta=post_beta, pre_gamma=pre_gamma, pre_beta=pre_beta)
    return dict(h=h, y=y, dx=grads.dx, db=grads.db, dgate=grads.dgate, dpost_gamma=grads.dpost_gamma, dpost_beta=grads.dpost_beta,
                dpre_gamma=grads.dpre_gamma, dpre_beta=grads.dpre_beta)


def _own_quantize(api, s):
    codes, scales = api.ssconv_quantize_mxfp4(s["x"])
    return api.ssconv_dequantize_mxfp4(codes, scales, s["case"]["c"])


def _own_pointwise(api, s):
    codes, scales = api.ssconv_quantize_mxfp4(s["x"])
    return api.ssconv_forward_dense_mxfp4(s["desc"], codes, scales, s["w_codes"], s["w_scales"], s["bias"]).view(s["case"]["rows"], -1)


def _plain_norm(case, grads):
    if case.get("norm", "l2") == "l2":
        return torch.stack([g.float().square().sum(dtype=torch.float64) for g in grads]).sum().sqrt().float().view(1)
    return torch.stack([g.float().abs().max() for g in grads]).max().view(1)


def _plain_clip(s):
    norm = _plain_norm(s["case"], s["grads"])
    factor = (s["case"]["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0)
    [o.copy_(g.float() * factor) for o, g in zip(s["out"], s["grads"])]
    return dict(norm=norm, out=s["out_flat"])


def _plain_adamw_one(theta, g, m, v):
    m.mul_(BETA1).add_(g * (1 - BETA1))
    v.mul_(BETA2).add_(g * g * (1 - BETA2))
    theta.sub_(LR * (m / (1 - BETA1 ** STEP) / ((v / (1 - BETA2 ** STEP)).sqrt() + ADAM_EPS) + DECAY * theta))


def _plain_adamw(s):
    norm = _plain_norm(s["case"], s["grads"])
    factor = (s["case"]["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0)
    [_plain_adamw_one(t, g.float() * factor, m, v) for t, g, m, v in zip(s["theta"], s["grads"], s["m"], s["v"])]
    return dict(norm=norm, flats=s["flats"])


def _plain_hat(kind, v):
    """(v normalised, 1 / its deviation) over the last axis."""
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    r = torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS)
    return v * r, r


def _plain_affine(hat, gamma, beta):
    return hat * gamma if beta is None else hat * gamma + beta


def _plain_norm_backward(kind, d, hat, r):
    d0 = d - d.mean(-1, keepdim=True) if kind == "layer" else d
    return r * (d0 - hat * (d * hat).mean(-1, keepdim=True))


def _plain_resnorm(s):
    c = s["case"]
    images, pixels, ch = c["images"], c["pixels"], c["c"]
    x, b = s["x"].float().view(images, pixels, ch), s["b"].float().view(images, pixels, ch)
    gate = None if s["gate"] is None else s["gate"] if c["gate"] == "shared" else s["gate"].view(images, 1, ch)
    p = b
    if c["post"] != "none":
        bhat, rb = _plain_hat(c["post"], b)
        p = _plain_affine(bhat, *s["post"])
    h = c["scale"] * x + (p if gate is None else gate * p)
    y = None
    if c["pre"] != "none":
        hhat, rh = _plain_hat(c["pre"], h)
        y = _plain_affine(hhat, *s["pre"])

    def out(t):
        return None if t is None else t.to(torch.bfloat16).view(images * pixels, ch)

    if not c["train"]:
        return dict(h=out(h), y=out(y))
    r = dict.fromkeys(("dgate", "dpost_gamma", "dpost_beta", "dpre_gamma", "dpre_beta"))
    d = s["dh"].float().view(images, pixels, ch)
    if c["pre"] != "none":
        dy = s["dy"].float().view(images, pixels, ch)
        r["dpre_gamma"] = (dy * hhat).sum((0, 1))
        r["dpre_beta"] = None if s["pre"][1] is None else dy.sum((0, 1))
        d = d + _plain_norm_backward(c["pre"], dy * s["pre"][0], hhat, rh)
    dp = d
    if gate is not None:
        r["dgate"] = (d * p).sum((0, 1)) if c["gate"] == "shared" else (d * p).sum(1)
        dp = d * gate
    db = dp
    if c["post"] != "none":
        r["dpost_gamma"] = (dp * bhat).sum((0, 1))
        r["dpost_beta"] = None if s["post"][1] is None else dp.sum((0, 1))
        db = _plain_norm_backward(c["post"], dp * s["post"][0], bhat, rb)
    return dict(h=out(h), y=out(y), dx=out(c["scale"] * d), db=out(db), **r)


def _plain_quantize(s):
    return _mx_values(s["x"]).to(torch.bfloat16)


def _plain_pointwise(s):
    v = _mx_values(s["x"]) @ s["w"].t() + s["bias"]
    if s["case"]["act"] == "relu":
        v = v.clamp(min=0)
    if s["case"]["act"] == "gelu":
        v = 0.5 * v * (1 + torch.erf(v / math.sqrt(2)))
    return v.to(torch.bfloat16)


# ----------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind in ("clip", "adamw"):
        n, width = case["total"], 4 if case["dtype"] == "f32" else 2
        return dict(bytes=2 * n * width, flops=3 * n) if kind == "clip" else dict(bytes=n * (width + 24), flops=18 * n)
    if kind == "resnorm":
        n = case["images"] * case["pixels"] * case["c"]
        norms = (case["post"] != "none") + (case["pre"] != "none")
        moved = 3 + (case["pre"] != "none") + ((3 + (case["pre"] != "none")) if case["train"] else 0)
        return dict(bytes=2 * n * moved, flops=n * (3 + 8 * norms) * (3 if case["train"] else 1))
    if kind == "quantize":
        return dict(bytes=4 * case["rows"] * case["c"], flops=4 * case["rows"] * case["c"])
    rows, cin, cout = case["rows"], case["cin"], case["cout"]
    return dict(bytes=2 * rows * cin + 17 * cin * cout // 32 + 4 * cout + 2 * rows * cout, flops=2 * rows * cin * cout)


# ----------------------------------------------------------------------------- the definition in 64 bits
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _mx_exact(x):
    """The element of the grid nearest to each |x| / scale (of two equally near ones that with the even code), by search."""
    rows, c = x.shape
    v = torch.zeros(rows, -(-c // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    v[:, :c] = x.double()
    v = v.view(rows, -1, BLOCK)
    powers = torch.tensor([2.0 ** k for k in range(-127, 128)], dtype=torch.float64, device=x.device)
    scale = powers[(torch.searchsorted(4 * powers, v.abs().amax(-1, keepdim=True), right=True) - 1).clamp(min=0)]
    a = v.abs() / scale
    best, far = torch.zeros_like(a), a.clone()
    for code in (2, 4, 6, 1, 3, 5, 7):       # even codes first: an odd one has to be nearer
        d = (a - _GRID[code]).abs()
        best = torch.where(d < far, torch.full_like(best, _GRID[code]), best)
        far = torch.minimum(d, far)
    return (best * scale * torch.sign(v)).view(rows, -1)[:, :c]


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind in ("clip", "adamw"):
        g = torch.cat([t.double() for t in s["grads"]])
        norm = torch.linalg.vector_norm(g, 2 if case.get("norm", "l2") == "l2" else math.inf)
        factor = min(1.0, case["max_norm"] / (float(norm) + CLIP_EPS))
        if kind == "clip":
            out = torch.zeros_like(s["out_flat"], dtype=torch.float64)
            for o, t in zip(s["out"], s["grads"]):
                at = o.storage_offset()
                out[at:at + o.numel()] = t.double() * factor
            return dict(norm=norm.view(1), out=out)
        flats = [f.double() for f in s["flats"]]
        for t, p in zip(s["grads"], s["theta"]):
            at = slice(p.storage_offset(), p.storage_offset() + p.numel())
            gd = t.double() * factor
            theta, m, v = (f[at] for f in flats)
            m_new = BETA1 * m + (1.0 - BETA1) * gd
            v_new = BETA2 * v + (1.0 - BETA2) * gd ** 2
            step = (m_new / (1.0 - BETA1 ** STEP)) / (torch.sqrt(v_new / (1.0 - BETA2 ** STEP)) + ADAM_EPS)
            theta -= LR * (step + DECAY * theta)
            m.copy_(m_new)
            v.copy_(v_new)
        return dict(norm=norm.view(1), flats=tuple(flats))
    if kind == "resnorm":
        return _exact_resnorm(case, s)
    if kind == "quantize":
        return _mx_exact(s["x"])
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = (torch.randn((case["cout"], case["cin"]), generator=g, device=DEV) / math.sqrt(case["cin"])).to(torch.bfloat16)
    v = torch.einsum("rk,ck->rc", _mx_exact(s["x"]), _mx_exact(w)) + s["bias"].double()
    if case["act"] == "relu":
        v = torch.relu(v)
    if case["act"] == "gelu":
        v = v * torch.special.ndtr(v)
    return v


def _exact_resnorm(case, s):
    """Forward by the definition; the gradients by differentiating it."""
    x, b = (s[k].double().requires_grad_(case["train"]) for k in ("x", "b"))
    leaves = {k: None if t is None else t.double().requires_grad_(case["train"]) for k, t in
              dict(gate=s["gate"], post_gamma=s["post"][0], post_beta=s["post"][1], pre_gamma=s["pre"][0], pre_beta=s["pre"][1]).items()}

    def norm(which, v):
        if case[which] == "none":
            return v
        if case[which] == "layer":
            var, mean = torch.var_mean(v, dim=-1, correction=0, keepdim=True)
            hat = (v - mean) / torch.sqrt(var + EPS)
        else:
            hat = v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
        hat = hat * leaves[which + "_gamma"]
        return hat if leaves[which + "_beta"] is None else hat + leaves[which + "_beta"]

    gate = leaves["gate"]
    if case["gate"] == "image":
        gate = gate.repeat_interleave(case["pixels"], 0)
    p = norm("post", b)
    h = case["scale"] * x + (p if gate is None else gate * p)
    y = norm("pre", h) if case["pre"] != "none" else None
    out = dict(h=h.detach(), y=None if y is None else y.detach())
    if not case["train"]:
        return out
    loss = (h * s["dh"].double()).sum() + (0.0 if y is None else (y * s["dy"].double()).sum())
    wanted = dict(dx=x, db=b, **{"d" + k: t for k, t in leaves.items()})
    there = [k for k, t in wanted.items() if t is not None]
    out.update(dict.fromkeys(wanted))
    out.update(zip(there, torch.autograd.grad(loss, [wanted[k] for k in there])))
    return out
