"""The retraining operators that this library's speed is measured on: group
normalisation with an activation (forward and backward, NCHW and channels
last), the gradient norm over many tensors, and the AdamW step over many
tensors with moments in 32 or 8 bits.

``own`` chooses the side: the plain forms in elementary torch operations, or
the calls that a user makes of paper_2003_06513_amd.binding.

  gn_fwd  y = act(gamma * xhat + beta), and the statistics that the backward reads
  gn_bwd  dx, dgamma, dbeta from dy and the kept statistics
  clip    the norm of all gradients and the factor that clips them
  adamw   one step on parameters and moments, with the clip before it or without
"""
import math
import random

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16}
_ELT = {"f32": 4, "f16": 2}
_EPS = 1e-5                      # of the normalisation
_LR, _B1, _B2, _ADAM_EPS, _WD = 1e-3, 0.9, 0.999, 1e-8, 1e-2
_STEPS = 100                     # steps done before the measured one
_MAX_NORM = 1.0
_PAD = 256                       # each tensor begins at a multiple of this in the flat buffers
_VGG = [(3, 64), (64, 64), (64, 128), (128, 128), (128, 256), (256, 256), (256, 256), (256, 512), (512, 512),
        (512, 512), (512, 512), (512, 512), (512, 512)]


def _gn(kind, layout, dtype, n, c, h, w, groups, act, name=None):
    k = {"kind": kind, "layout": layout, "dtype": dtype, "n": n, "c": c, "h": h, "w": w, "groups": groups, "act": act}
    if name:
        k["name"] = name
    return k


def _tensors(kind, net, count, numel, grad, bits=32, copy=False, clip=False, mix=0, name=None):
    k = {"kind": kind, "net": net, "count": count, "numel": numel, "grad": grad, "bits": bits, "copy": copy,
         "clip": clip, "mix": mix}
    if name:
        k["name"] = name
    return k


def listed():
    return [
        # a layer of ResNet-50 on one image: the launch is most of the time
        _gn("gn_fwd", "nchw", "f16", 1, 256, 14, 14, 32, "relu", name="fwd_nchw_256c_14_b1_f16"),
        # a training batch of ResNet-50's first stage, channels last, two channels a group
        _gn("gn_fwd", "nhwc", "f16", 32, 64, 56, 56, 32, "silu", name="fwd_nhwc_64c_56_b32_f16"),
        # a CIFAR batch in single precision, in the layout of the convolutions
        _gn("gn_fwd", "nchw", "f32", 256, 128, 16, 16, 32, "relu", name="fwd_nchw_128c_16_b256_f32"),
        # no size a multiple of anything
        _gn("gn_bwd", "nhwc", "f32", 3, 93, 45, 61, 31, "silu", name="bwd_nhwc_ragged_93c_45x61_b3_f32"),
        # ResNet-50's second stage in the backward pass
        _gn("gn_bwd", "nchw", "f16", 32, 128, 28, 28, 32, "relu", name="bwd_nchw_128c_28_b32_f16"),
        # the largest layer of the library's sweep, channels last
        _gn("gn_bwd", "nhwc", "f16", 64, 512, 28, 28, 32, "relu", name="bwd_nhwc_512c_28_b64_f16"),
        # the gradients of VGG-16's 13 pruned layers: stored values and biases
        _tensors("clip", "vgg16", 26, 0, "f32", name="clip_vgg16_f32"),
        # 64 dense 512 -> 512 layers with half-precision gradients
        _tensors("clip", "dense", 64, 9 * 512 * 512, "f16", name="clip_64x512c_f16"),
        # retraining one pruned layer: values and bias
        _tensors("adamw", "layer", 2, 0, "f32", name="adamw_layer_f32"),
        # retraining the pruned VGG-16 with the clip, half-precision copies for the convolutions
        _tensors("adamw", "vgg16", 26, 0, "f32", copy=True, clip=True, name="adamw_vgg16_clip_copy"),
        # a network of many tensors of very different sizes, moments in 8 bits
        _tensors("adamw", "mixed", 161, 1 << 20, "f32", bits=8, clip=True, mix=7, name="adamw8_161_mixed_clip"),
        # 64 dense 512 -> 512 layers, moments in 8 bits: memory decides
        _tensors("adamw", "dense", 64, 9 * 512 * 512, "f32", bits=8, name="adamw8_64x512c"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("gn_fwd", "gn_bwd", "clip", "adamw"), (3, 3, 1, 3))[0]
    if kind in ("gn_fwd", "gn_bwd"):
        while True:
            n, c, h = _log(rng, 1, 256), _log(rng, 8, 1024), _log(rng, 1, 224)
            w = h if rng.random() < 0.6 else max(1, min(224, int(h * rng.uniform(0.6, 1.7))))
            if rng.random() < 0.5:      # what networks use
                c = 2 ** round(math.log2(c))
                h = w = min((4, 7, 8, 14, 16, 28, 32, 56, 112, 224), key=lambda s: abs(math.log(s / h)))
            if 2000 <= n * c * h * w <= 25_000_000:
                break
        groups = rng.choice([g for g in range(1, min(c, 64) + 1) if c % g == 0])
        if c % 32 == 0 and rng.random() < 0.5:
            groups = 32
        return _gn(kind, rng.choice(("nchw", "nhwc")), rng.choice(("f32", "f16")), n, c, h, w, groups,
                   rng.choice(("none", "relu", "silu")))
    count, numel = _log(rng, 1, 400), _log(rng, 1000, 2_000_000)
    while count * numel > 60_000_000:
        numel //= 2
    grad = rng.choice(("f32", "f16"))
    if kind == "clip":
        return _tensors(kind, "mixed", count, numel, grad, mix=rng.randrange(1 << 16))
    return _tensors(kind, "mixed", count, numel, grad, rng.choice((32, 8)), rng.random() < 0.3, rng.random() < 0.5,
                    rng.randrange(1 << 16))


def _sizes(case):
    """Elements of each tensor: first those that decay (weights), then those
    that do not (biases and norm parameters)."""
    if case["net"] == "layer":                      # 256 -> 256, 60 % of the kernels dropped
        return [4 * (65536 - 39322)], [256]
    if case["net"] == "vgg16":
        keep = [ci * co if i == 0 else ci * co // 3 for i, (ci, co) in enumerate(_VGG)]
        return [4 * k for k in keep], [co for _, co in _VGG]
    if case["net"] == "dense":
        return [case["numel"]] * case["count"], []
    r = random.Random(case["mix"])
    s = [_log(r, 1, case["numel"]) for _ in range(case["count"])]
    cut = (len(s) + 1) // 2
    return s[:cut], s[cut:]


def _places(sizes):
    """Where each tensor begins in a flat buffer, and the buffer's length."""
    at, end = [], 0
    for k in sizes:
        at.append(end)
        end += -(-k // _PAD) * _PAD
    return at, end


def _randn(shape, seed, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _gn_inputs(case, seed):
    n, c, h, w = (case[k] for k in ("n", "c", "h", "w"))
    fmt = torch.channels_last if case["layout"] == "nhwc" else torch.contiguous_format
    dt = _DT[case["dtype"]]
    # what a convolution writes: each channel with a level and a spread of its own
    x = _randn((n, c, h, w), seed) * (0.5 + _randn((c, 1, 1), seed + 1).abs()) + 0.5 * _randn((c, 1, 1), seed + 2)
    s = {"case": case, "x": x.to(dt).contiguous(memory_format=fmt),
         "gamma": 1 + 0.2 * _randn(c, seed + 3), "beta": 0.2 * _randn(c, seed + 4)}
    if case["kind"] == "gn_bwd":
        s["dy"] = (0.1 * _randn((n, c, h, w), seed + 5)).to(dt).contiguous(memory_format=fmt)
        # the statistics that the forward kept
        xg = s["x"].double().unflatten(1, (case["groups"], -1))
        mean = xg.mean((2, 3, 4))
        s["mean"] = mean.float()
        s["rstd"] = ((xg - mean[:, :, None, None, None]).square().mean((2, 3, 4)) + _EPS).rsqrt().float()
    return s


def _tensor_inputs(case, seed):
    decayed, others = _sizes(case)
    sizes = decayed + others
    at, total = _places(sizes)
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for a, k in zip(at, sizes):
        inside[a:a + k] = True
    s = {"case": case, "sizes": sizes, "at": at, "decayed": _places(decayed)[1],
         "g": (2e-3 * _randn(total, seed) * inside).to(_DT[case["grad"]])}
    if case["kind"] == "clip":
        return s
    s["p"] = 0.05 * _randn(total, seed + 1) * inside
    s["steps"] = torch.full((1,), _STEPS, dtype=torch.int64, device="cuda")
    if case["copy"]:
        s["copy"] = s["p"].half()
    if case["bits"] == 32:
        s["m"] = 5e-4 * _randn(total, seed + 2) * inside
        s["v"] = 4e-6 * _randn(total, seed + 3).square() * inside
    else:
        s["m"] = ((40 * _randn(total, seed + 2)).clamp_(-127, 127) * inside).to(torch.int8)
        s["v"] = ((150 + 35 * _randn(total, seed + 3)).clamp_(1, 255) * inside).to(torch.uint8)
        # per block of 256: the largest |m| and the largest v
        s["scale"] = torch.stack((1e-3 * (0.5 * _randn(total // 256, seed + 4)).exp(),
                                  1e-5 * _randn(total // 256, seed + 5).exp()), dim=1).contiguous()
    return s


def _views(flat, s):
    return [flat[a:a + k] for a, k in zip(s["at"], s["sizes"])]


def prepare(case, seed):
    if case["kind"] in ("gn_fwd", "gn_bwd"):
        s = _gn_inputs(case, seed)
        if own:
            # the buffers of a program that runs the layer again and again
            s["out"] = torch.empty_like(s["x"])
            if case["kind"] == "gn_fwd":
                s["mean"], s["rstd"] = (torch.empty((case["n"], case["groups"]), device="cuda") for _ in range(2))
            else:
                s["dgamma"], s["dbeta"] = torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
        return s
    s = _tensor_inputs(case, seed)
    if own:
        from paper_2003_06513_amd import binding as B
        grads = _views(s["g"], s)
        if case["kind"] == "clip":
            s["list"] = B.ParamList(None, grads)
            s["norm"] = torch.empty(2, device="cuda")
        else:
            decayed = len(_sizes(case)[0])
            opt = B.AdamW(_views(s["p"], s), grads, lr=_LR, betas=(_B1, _B2), eps=_ADAM_EPS,
                          weight_decay=[_WD if i < decayed else 0.0 for i in range(len(s["sizes"]))],
                          state_bits=case["bits"], copies=_views(s["copy"], s) if case["copy"] else None)
            opt.m.copy_(s.pop("m"))
            opt.v.copy_(s.pop("v"))
            opt.steps.copy_(s.pop("steps"))
            if case["bits"] == 8:
                opt.scale.copy_(s.pop("scale"))
            s["opt"] = opt
    return s


# ------------------------------------------------------------- the library's calls
def _run_own(s):
    from paper_2003_06513_amd import binding as B
    case = s["case"]
    if case["kind"] == "gn_fwd":
        B.group_norm_fwd(s["x"], case["groups"], s["gamma"], s["beta"], s["out"], eps=_EPS, act=case["act"],
                         mean=s["mean"], rstd=s["rstd"])
        return {"y": s["out"], "mean": s["mean"], "rstd": s["rstd"]}
    if case["kind"] == "gn_bwd":
        B.group_norm_bwd(s["x"], s["dy"], case["groups"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["out"],
                         s["dgamma"], s["dbeta"], act=case["act"])
        return {"dx": s["out"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if case["kind"] == "clip":
        B.grad_norm(s["list"], s["norm"], max_norm=_MAX_NORM)
        return {"norm": s["norm"]}
    opt = s["opt"]
    out = {}
    if case["clip"]:
        out["norm"] = opt.grad_norm(_MAX_NORM)
        opt.step(factor=opt.factor)
    else:
        opt.step()
    out["p"], out["steps"] = s["p"], opt.steps
    out["m"], out["v"] = opt.moments()
    if case["copy"]:
        out["copy"] = s["copy"]
    return out


# ------------------------------------------------------------- the plain forms
def _act(u, act):
    return u.clamp(min=0) if act == "relu" else u * torch.sigmoid(u) if act == "silu" else u


def _dact(u, act):
    if act == "relu":
        return (u > 0).to(u.dtype)
    if act == "silu":
        t = torch.sigmoid(u)
        return t * (1 + u * (1 - t))
    return torch.ones_like(u)


def _by_group(s):
    """x, and gamma and beta to go with it, as [n, groups, c / groups, h, w]."""
    g = s["case"]["groups"]
    return (s["x"].float().unflatten(1, (g, -1)), s["gamma"].view(1, g, -1, 1, 1), s["beta"].view(1, g, -1, 1, 1))


def _plain_gn_fwd(s):
    x, gamma, beta = _by_group(s)
    mean = x.mean((2, 3, 4), keepdim=True)
    d = x - mean
    rstd = (d.square().mean((2, 3, 4), keepdim=True) + _EPS).rsqrt()
    y = _act(d * rstd * gamma + beta, s["case"]["act"])
    return {"y": y.flatten(1, 2).to(s["x"].dtype), "mean": mean.flatten(1), "rstd": rstd.flatten(1)}


def _plain_gn_bwd(s):
    x, gamma, beta = _by_group(s)
    mean, rstd = s["mean"][:, :, None, None, None], s["rstd"][:, :, None, None, None]
    xh = (x - mean) * rstd
    du = s["dy"].float().unflatten(1, (s["case"]["groups"], -1)) * _dact(xh * gamma + beta, s["case"]["act"])
    e = du * gamma
    s1 = e.mean((2, 3, 4), keepdim=True)
    s2 = (e * xh).mean((2, 3, 4), keepdim=True)
    dx = rstd * (e - s1 - xh * s2)
    return {"dx": dx.flatten(1, 2).to(s["x"].dtype), "dgamma": (du * xh).sum((0, 3, 4)).flatten(),
            "dbeta": du.sum((0, 3, 4)).flatten()}


def _plain_norm(g):
    """[norm, factor]; the squares are summed in 64 bits."""
    norm = g.double().square().sum().sqrt()
    return torch.stack((norm, (_MAX_NORM / norm).clamp(max=1.0))).float()


def _decoded(s):
    """The moments that 8-bit codes and the peaks of their blocks stand for, in 64 bits."""
    peak = s["scale"].double()
    m, v = s["m"].view(-1, 256).double(), s["v"].view(-1, 256).double()
    return (m * m.abs() / 127 ** 2 * peak[:, :1]).view(-1), ((v / 255) ** 4 * peak[:, 1:]).view(-1)


def _encode(x, peak, top, power):
    """How many of the borders (k - 1/2) ** power, k = 1..top, lie at or below x * top ** power / peak: in 64 bits,
    as a value next to a border decides."""
    borders = (torch.arange(1, top + 1, device=x.device, dtype=torch.float64) - 0.5) ** power
    inv = torch.where(peak > 0, top ** power / peak.double(), 0.0)
    return torch.bucketize(x * inv, borders, out_int32=True, right=True)


def _plain_adamw(s):
    case = s["case"]
    wide = torch.float64 if case["bits"] == 8 else torch.float32
    g = s["g"].to(wide)
    out = {}
    if case["clip"]:
        out["norm"] = _plain_norm(s["g"])
        g = g * out["norm"][1]
    m, v = _decoded(s) if case["bits"] == 8 else (s["m"], s["v"])
    b1, b2 = float(np.float32(_B1)), float(np.float32(_B2))
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    t = (s["steps"] + 1).double()
    rate, root = _LR / (1 - b1 ** t), (1 - b2 ** t).rsqrt()
    if wide is torch.float32:
        rate, root = rate.float(), root.float()
    p, cut = s["p"], s["decayed"]
    p[:cut].mul_(1 - _LR * _WD)
    p.sub_(m / (v.sqrt() * root + _ADAM_EPS) * rate)
    s["steps"] += 1
    if case["copy"]:
        s["copy"].copy_(p)
        out["copy"] = s["copy"]
    if case["bits"] == 8:
        m, v = m.view(-1, 256), v.view(-1, 256)
        peak = torch.stack((m.abs().amax(1), v.amax(1)), 1).float()     # held in 32 bits
        s["scale"].copy_(peak)
        s["m"].view(-1, 256).copy_(_encode(m.abs(), peak[:, :1], 127, 2) * m.sign())
        # a moment that is not zero never becomes zero
        s["v"].view(-1, 256).copy_(torch.maximum(_encode(v, peak[:, 1:], 255, 4), (v > 0).int()))
        out["m"], out["v"] = (d.float() for d in _decoded(s))
    else:
        out["m"], out["v"] = s["m"].copy_(m), s["v"].copy_(v)
    out["p"], out["steps"] = p, s["steps"]
    return out


def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    if kind == "clip":
        return {"norm": _plain_norm(s["g"])}
    return {"gn_fwd": _plain_gn_fwd, "gn_bwd": _plain_gn_bwd, "adamw": _plain_adamw}[kind](s)


def work(case):
    if case["kind"] in ("gn_fwd", "gn_bwd"):
        numel = case["n"] * case["c"] * case["h"] * case["w"]
        bwd = case["kind"] == "gn_bwd"
        return {"bytes": (3 if bwd else 2) * _ELT[case["dtype"]] * numel + 8 * case["n"] * case["groups"]
                + (16 if bwd else 8) * case["c"], "flops": (24 if bwd else 12) * numel}
    decayed, others = _sizes(case)
    numel = sum(decayed) + sum(others)
    if case["kind"] == "clip":
        return {"bytes": _ELT[case["grad"]] * numel + 8, "flops": 2 * numel}
    # parameter read and written, gradient read, moments read and written (8 bits: and written as the values they
    # stand for), the copy written
    moments = 16 if case["bits"] == 32 else 4 + 16 / 256 + 8
    return {"bytes": int((8 + _ELT[case["grad"]] + moments + (2 if case["copy"] else 0)) * numel),
            "flops": (16 if case["bits"] == 32 else 40) * numel}


# ------------------------------------------------------------- 64-bit reference
def _exact_gn(s):
    case = s["case"]
    n, c, h, w, k = case["n"], case["c"], case["h"], case["w"], case["groups"]
    flat = lambda t: t.double().contiguous().reshape(n, k, -1)      # noqa: E731
    per = lambda t: t.double().repeat_interleave(h * w).reshape(1, k, -1)    # noqa: E731
    x, gamma, beta = flat(s["x"]), per(s["gamma"]), per(s["beta"])
    if case["kind"] == "gn_fwd":
        var, mean = torch.var_mean(x, dim=2, correction=0)
        rstd = 1 / torch.sqrt(var + _EPS)
        u = (x - mean[..., None]) * rstd[..., None] * gamma + beta
        y = {"none": u, "relu": torch.relu(u), "silu": u / (1 + torch.exp(-u))}[case["act"]]
        return {"y": y.reshape(n, c, h, w), "mean": mean, "rstd": rstd}
    rstd = s["rstd"].double()[..., None]
    xh = (x - s["mean"].double()[..., None]) * rstd
    u = xh * gamma + beta
    e = torch.exp(-u)
    slope = {"none": torch.ones_like(u), "relu": (u > 0).double(), "silu": (1 + e + u * e) / (1 + e) ** 2}[case["act"]]
    du = flat(s["dy"]) * slope
    lead = du * gamma
    dx = (lead - lead.mean(2, keepdim=True) - xh * (lead * xh).mean(2, keepdim=True)) * rstd
    by_channel = lambda t: t.reshape(n, c, h * w).sum((0, 2))       # noqa: E731
    return {"dx": dx.reshape(n, c, h, w), "dgamma": by_channel(du * xh), "dbeta": by_channel(du)}


def _exact_adamw(s):
    case = s["case"]
    g, p = s["g"].double(), s["p"].double()
    out = {}
    if case["clip"]:
        norm = torch.linalg.vector_norm(g)
        factor = torch.where(norm > _MAX_NORM, _MAX_NORM / norm, 1.0)
        out["norm"] = torch.stack((norm, factor))
        g = g * factor.float()          # the step takes the factor that the norm's call wrote, in 32 bits
    m, v = s["m"].double(), s["v"].double()
    if case["bits"] == 8:
        peak = s["scale"].double().repeat_interleave(256, dim=0)
        m, v = torch.sign(m) * (m / 127) ** 2 * peak[:, 0], (v / 255) ** 4 * peak[:, 1]
        del peak
    b1, b2 = float(np.float32(_B1)), float(np.float32(_B2))
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g ** 2
    t = _STEPS + 1
    decay = torch.zeros_like(p)
    decay[:s["decayed"]] = _LR * _WD
    p = p - decay * p - _LR * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + _ADAM_EPS)
    if case["bits"] == 8:
        mb, vb = m.reshape(-1, 256), v.reshape(-1, 256)
        # the peaks are held in 32 bits, and the codes are taken against what is held
        am, av = (z.max(1, keepdim=True).values.float().double() for z in (mb.abs(), vb))
        cm = torch.floor(torch.sqrt(mb.abs() / am.clamp(min=1e-300)) * 127 + 0.5)
        cv = torch.floor(torch.sqrt(torch.sqrt(vb / av.clamp(min=1e-300))) * 255 + 0.5)
        cv = torch.where((vb > 0) & (cv == 0), 1.0, cv)
        m, v = (torch.sign(mb) * (cm / 127) ** 2 * am).reshape(-1), ((cv / 255) ** 4 * av).reshape(-1)
    out.update(p=p, m=m, v=v, steps=None)
    if case["copy"]:
        out["copy"] = p
    return out


def exact(case, seed):
    if case["kind"] in ("gn_fwd", "gn_bwd"):
        return _exact_gn(_gn_inputs(case, seed))
    s = _tensor_inputs(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(s)
    norm = torch.linalg.vector_norm(s["g"].double())
    return {"norm": torch.stack((norm, torch.where(norm > _MAX_NORM, _MAX_NORM / norm, 1.0)))}
