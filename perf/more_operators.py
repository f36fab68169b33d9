"""Operators of a sequence or image model's training step beside the convolution, and what they have to give.

A case is one call:

  gnorm_forward    group norm with an activation of x, channels last [batch][sites][channels] or first
                   [batch][channels][sites]: y and each group's (mean, 1 / deviation)
  gnorm_backward   its gradients: of x, and of weight and bias summed over batch and sites
  recur_forward    a gated linear recurrence h_t = a_t h_(t-1) + b_t over the middle axis of
                   [outer][length][inner], with an initial state and steps at which the state is dropped:
                   h of every step and the last state
  recur_backward   its gradients: of gates, values and initial state
  muon_step        one step over many matrices: momentum, orthogonalised by five Newton-Schulz products, and
                   the parameters' update
  orthogonalize    the products alone: of many matrices, each with its singular values brought near 1

``listed()`` holds sizes of the time-series network and of the ResNet-shaped stacks (maps of 512 samples and of
56 x 56 points, their parameter lists) and generic ones beside them; ``draw()`` samples the ranges they stand
for: 1 to 256 samples of 4 to 16384 sites and 1 to 1024 channels, sequences of 1 to 131072 steps and 1 to 4096
channels or of single channels side by side, 1 to 24 matrices with sides of 1 to 2048, three types.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)  # of s, s^3 and s^5, for every singular value s
STEPS = 5
ALIGN = 64  # a matrix's values start at a multiple of this many in the momentum's layout
LR, MOMENTUM, DECAY, EPS, SEED = 0.02, 0.95, 0.01, 1e-7, 7


# ---- cases ----------------------------------------------------------------------
def _gnorm(op, batch, sites, channels, groups, dtype, act="silu", last=True, gap=0):
    """gap: unused values between the samples of x."""
    return {"op": op, "batch": batch, "sites": sites, "channels": channels, "groups": groups, "dtype": dtype,
            "act": act, "last": last, "gap": gap}


def _recur(op, outer, length, inner, dtype, gate="sigmoid", resets=0, halves=False):
    """gate: a = sigmoid(gate) and b = (1 - a) x, or a = exp(gate) and b = x.  resets: sequences that lie one
    after another (0: no step drops the state).  halves: gates and values are the halves of one tensor."""
    return {"op": op, "outer": outer, "length": length, "inner": inner, "dtype": dtype, "gate": gate,
            "resets": resets, "halves": halves}


def _muon(op, net, param="f32", grad="f32", matrices=0, most=0, mix=0):
    """net: a list of matrices by name, or "drawn": `matrices` with sides of 1 to `most` by the number `mix`."""
    return {"op": op, "net": net, "param": param, "grad": grad, "matrices": matrices, "most": most, "mix": mix}


def listed():
    return [
        # a small map of a few samples: latency
        dict(_gnorm("gnorm_forward", 2, 64, 32, 8, "f32"), name="gnorm_last_2x64x32_forward"),
        # the large-image layer's maps with their channels side by side, in reduced precision
        dict(_gnorm("gnorm_forward", 128, 3136, 64, 32, "bf16"), name="gnorm_last_128x3136x64_forward"),
        # gradients at a wide layer
        dict(_gnorm("gnorm_backward", 32, 3136, 256, 32, "bf16"), name="gnorm_last_32x3136x256_backward"),
        # gradients at the time-series network's widest map
        dict(_gnorm("gnorm_backward", 64, 512, 256, 16, "f32", last=False), name="gnorm_first_64x256x512_backward"),
        # one token for each of many requests: latency
        dict(_recur("recur_forward", 256, 1, 1024, "bf16"), name="recur_256x1x1024_forward"),
        # prompts of a model of that width
        dict(_recur("recur_forward", 8, 4096, 2048, "bf16", halves=True), name="recur_8x4096x2048_forward"),
        # one long run of packed sequences in few channels
        dict(_recur("recur_forward", 1, 65537, 256, "f32", gate="exp", resets=37), name="recur_1x65537x256_forward"),
        # a training step's gradients
        dict(_recur("recur_backward", 8, 4096, 1024, "bf16", halves=True), name="recur_8x4096x1024_backward"),
        # the maps of 64 series of 128 channels, samples side by side
        dict(_recur("recur_backward", 8192, 1250, 1, "f32"), name="recur_8192x1250_backward"),
        # the time-series network's filters and classifier: latency
        dict(_muon("muon_step", "fcn"), name="muon_fcn"),
        # an 18-layer residual network's, gradients in reduced precision
        dict(_muon("muon_step", "resnet", grad="bf16"), name="muon_resnet"),
        # matrices of a model of some hundred million parameters
        dict(_muon("orthogonalize", "wide", param="bf16", grad="bf16"), name="orthogonalize_wide"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    """About what a pass's floor takes, in seconds."""
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 5e14


def draw(rng):
    op = rng.choice(["gnorm_forward", "gnorm_backward", "recur_forward", "recur_backward", "muon_step",
                     "orthogonalize"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op.startswith("gnorm"):
        groups, each = _log_int(rng, 1, 64), _log_int(rng, 1, 64)
        # (where a ReLU's argument is within rounding of 0 its gradient has no value to compare)
        act = rng.choice(["silu", "none"] + ["relu"] * (op == "gnorm_forward"))
        case = _gnorm(op, _log_int(rng, 1, 256), _log_int(rng, 4, 16384), groups * min(each, 1024 // groups), groups,
                      dtype, act, rng.random() < 0.6, rng.choice([0, 0, 0, 1, 8, 40]))
        shrink = ("sites", "batch")
    elif op.startswith("recur"):
        if rng.random() < 0.3:
            outer, inner = _log_int(rng, 1, 16384), 1
        else:
            outer, inner = _log_int(rng, 1, 64), _log_int(rng, 1, 4096)
        length = _log_int(rng, 1, 131072)
        resets = 0 if rng.random() < 0.6 else _log_int(rng, 1, min(length, 4096))
        case = _recur(op, outer, length, inner, dtype, rng.choice(["sigmoid", "exp"]), resets, rng.random() < 0.4)
        shrink = ("length", "outer", "inner")
    else:
        param = rng.choice(["f32", "bf16"]) if op == "muon_step" else "bf16"
        case = _muon(op, "drawn", param, dtype, _log_int(rng, 1, 24), _log_int(rng, 4, 2048), rng.randint(1, 1 << 20))
        shrink = ("matrices", "most")
    most = max(_cost(x) for x in listed() if x["op"].split("_")[0][:4] == op[:4])
    while _cost(case) > most:
        k = next((k for k in shrink if case[k] > 64), max(shrink, key=lambda k: case[k]))
        case[k] = max(1, case[k] * 3 // 4)
        if "resets" in case:
            case["resets"] = min(case["resets"], case["length"])
    return case


def _shapes(case):
    """(rows, columns) of the matrices, in the order of the network's layers."""
    if case["net"] == "fcn":  # 1 -> 128 -> 256 -> 128 channels, 8, 5 and 3 taps, 50 classes
        return [(128, 8), (256, 128 * 5), (128, 256 * 3), (128, 50)]
    if case["net"] == "resnet":  # four stages of two blocks of two 3 x 3 layers
        got, ci = [(64, 27)], 64
        for co in (64, 128, 256, 512):
            for layer in range(4):
                got.append((co, (ci if layer == 0 else co) * 9))
                if layer == 0 and ci != co:
                    got.append((co, ci))
            ci = co
        return got + [(512, 10)]
    if case["net"] == "wide":  # ten blocks of width 1024 with a four times wider inner layer
        d = 1024
        return [(d, d), (d, d), (d, d), (d, d), (4 * d, d), (d, 4 * d)] * 10
    rng = random.Random(case["mix"])
    return [(_log_int(rng, 1, case["most"]), _log_int(rng, 1, case["most"])) for _ in range(case["matrices"])]


def _layout(case):
    """Where each matrix starts in the momentum's layout, and its length."""
    starts, at = [], 0
    for r, c in _shapes(case):
        starts.append(at)
        at += -(-r * c // ALIGN) * ALIGN
    return starts, at


def work(case):
    """Inputs in and outputs out once; operations of the formulas (of a symmetric product, half)."""
    if case["op"].startswith("gnorm"):
        n, wide = case["batch"] * case["sites"] * case["channels"], TYPES[case["dtype"]].itemsize
        rest = 8 * case["batch"] * case["groups"]
        if case["op"] == "gnorm_forward":
            return {"bytes": 2 * n * wide + 8 * case["channels"] + rest, "flops": 12 * n}
        return {"bytes": 3 * n * wide + 16 * case["channels"] + rest, "flops": 25 * n}
    if case["op"].startswith("recur"):
        n, wide = case["outer"] * case["length"] * case["inner"], TYPES[case["dtype"]].itemsize
        rest = 8 * case["outer"] * case["inner"] + (case["outer"] * case["length"] if case["resets"] else 0)
        if case["op"] == "recur_forward":
            return {"bytes": 3 * n * wide + rest, "flops": 8 * n}
        return {"bytes": 5 * n * wide + rest, "flops": 20 * n}
    flops = values = 0
    for r, c in _shapes(case):
        m, n = min(r, c), max(r, c)
        values += m * n
        flops += STEPS * (m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n)
    param, grad = TYPES[case["param"]].itemsize, TYPES[case["grad"]].itemsize
    return {"bytes": values * (param + grad if case["op"] == "orthogonalize" else 2 * param + grad + 8), "flops": flops}


# ---- inputs ---------------------------------------------------------------------
class _State:
    """A program's inputs, plan, workspace and output buffers."""


def _random(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, device="cuda", generator=g, dtype=dtype)

    return g, normal


def _prepare_gnorm(s, case, seed):
    _, normal = _random(seed)
    batch, sites, channels, groups = case["batch"], case["sites"], case["channels"], case["groups"]
    dtype = TYPES[case["dtype"]]
    s.last, s.act, s.eps, s.groups = case["last"], case["act"], 1e-5, groups
    s.shape = (batch, sites, channels) if s.last else (batch, channels, sites)
    per = (1, 1, channels) if s.last else (1, channels, 1)
    flat = sites * channels
    s.x = torch.empty(batch, flat + case["gap"], dtype=dtype, device="cuda")[:, :flat]
    # channels with means and deviations of their own
    x = normal(*s.shape, dtype=dtype) * (0.5 + normal(*per).abs()).to(dtype) + normal(*per).to(dtype)
    s.x.copy_(x.view(batch, flat))
    del x
    s.weight, s.bias = 1.0 + 0.2 * normal(channels), 0.3 * normal(channels)
    if case["op"] == "gnorm_forward":
        s.y = torch.empty(batch, flat, dtype=dtype, device="cuda")
        s.stats = torch.empty(2, batch, groups, device="cuda")
    else:
        s.dy = normal(batch, flat, dtype=dtype)
        s.stats = torch.stack(_group_stats(s, _grouped(s, s.x.float()))).reshape(2, batch, groups)
        s.dx = torch.empty(batch, flat + case["gap"], dtype=dtype, device="cuda")[:, :flat]
        s.dweight, s.dbias = torch.empty_like(s.weight), torch.empty_like(s.bias)
    if own:
        from paper_1911_09287_amd import bltrain
        s.plan = bltrain.GroupNormPlan(batch, sites, channels, groups, channels_last=s.last, act=s.act, dtype=dtype,
                                       eps=s.eps, x_stride=flat + case["gap"])
        s.ws = s.plan.workspace("cuda")


def _prepare_recur(s, case, seed):
    g, normal = _random(seed)
    outer, length, inner, dtype = case["outer"], case["length"], case["inner"], TYPES[case["dtype"]]
    s.kind, shape = case["gate"], (outer, length, inner)

    def pair():
        """Gates and values: two tensors, or the halves of one."""
        if not case["halves"]:
            return torch.empty(shape, dtype=dtype, device="cuda"), torch.empty(shape, dtype=dtype, device="cuda")
        if inner == 1:  # rows side by side
            both = torch.empty(outer, 2 * length, dtype=dtype, device="cuda")
            return both[:, :length].unsqueeze(2), both[:, length:].unsqueeze(2)
        both = torch.empty(outer, length, 2 * inner, dtype=dtype, device="cuda")
        return both[..., :inner], both[..., inner:]

    s.gate, s.x = pair()
    s.gate.copy_(normal(*shape, dtype=dtype))
    if s.kind == "sigmoid":
        s.gate.add_(1.5 + normal(1, 1, inner))  # channels that forget sooner and later
    else:  # decays over about 1 to 300 steps, other ones at every step
        s.gate.copy_(-torch.exp(s.gate.float() * 0.5 - 3.0 + normal(1, 1, inner)).clamp(3e-3, 20.0))
    s.x.copy_(normal(*shape, dtype=dtype))
    s.h0 = normal(outer, inner)
    s.resets = None
    if case["resets"]:
        s.resets = torch.zeros(outer, length, dtype=torch.uint8, device="cuda")
        at = torch.randint(0, length, (outer, case["resets"]), device="cuda", generator=g)
        s.resets.scatter_(1, at, 1)
    if case["op"] == "recur_forward":
        s.y, s.last = torch.empty(shape, dtype=dtype, device="cuda"), torch.empty_like(s.h0)
    else:
        s.dy, s.dlast = normal(*shape, dtype=dtype), normal(outer, inner)
        s.dgate, s.dx = pair()
        s.dh0 = torch.empty_like(s.h0)
    if own:
        from paper_1911_09287_amd import bltrain
        per_outer = s.gate.stride(0) if outer > 1 else 0
        s.plan = bltrain.RecurrencePlan(outer, length, inner, gate=s.kind, dtype=dtype,
                                        in_strides=(per_outer, s.gate.stride(1)) if case["halves"] else (0, 0))
        s.ws = s.plan.workspace("cuda")
        s.states = None
        if case["op"] == "recur_backward":  # what the forward call left for it
            s.states = s.plan.states("cuda")
            s.plan.forward(s.gate, s.x, torch.empty(shape, dtype=dtype, device="cuda"), s.ws, h0=s.h0,
                           resets=s.resets, states=s.states)


def _prepare_muon(s, case, seed):
    _, normal = _random(seed)
    shapes, (starts, total) = _shapes(case), _layout(case)
    s.shapes, s.starts, s.step = shapes, starts, 10
    # parameters, gradients and momentum lie in one buffer each, as a program that sums
    # gradients over GPUs in one piece keeps them
    grad = torch.zeros(total, device="cuda")
    for at, (r, c) in zip(starts, shapes):  # a few directions that most of the gradient lies in, and noise
        few = min(8, r, c)
        strong = torch.mm(normal(r, few) * torch.linspace(1.0, 0.2, few, device="cuda"), normal(few, c))
        torch.add(0.3 * normal(r, c), strong, out=grad[at:at + r * c].view(r, c))
    s.g = (1e-3 * grad).to(TYPES[case["grad"]])
    if case["op"] == "muon_step":
        inside = torch.zeros(total, dtype=torch.bool, device="cuda")
        for at, (r, c) in zip(starts, shapes):
            inside[at:at + r * c] = True
        s.p = (0.05 * normal(total)).mul_(inside).to(TYPES[case["param"]])
        s.m = 8e-3 * grad + (1e-3 * normal(total)).mul_(inside)
    else:
        s.p = torch.zeros(total, dtype=TYPES[case["param"]], device="cuda")  # the result
    if own:
        from paper_1911_09287_amd import bltrain
        s.plan = bltrain.MuonPlan(shapes, param_dtype=s.p.dtype, grad_dtype=s.g.dtype)
        s.tensors = s.plan.bind([s.p[at:at + r * c].view(r, c) for at, (r, c) in zip(starts, shapes)],
                                [s.g[at:at + r * c].view(r, c) for at, (r, c) in zip(starts, shapes)])
        s.ws = s.plan.workspace("cuda")
        if case["op"] == "muon_step":
            s.state = s.plan.state("cuda")
            s.plan.momentum(s.state).copy_(s.m)


def prepare(case, seed):
    s = _State()
    s.op = case["op"]
    {"gnor": _prepare_gnorm, "recu": _prepare_recur, "muon": _prepare_muon, "orth": _prepare_muon}[s.op[:4]](s, case, seed)
    return s


# ---- the plain forms ------------------------------------------------------------
def _grouped(s, x):
    """[batch][...][group][...] values with the two axes that a group spans."""
    batch, a, b = s.shape
    if s.last:
        return x.reshape(batch, a, s.groups, b // s.groups)
    return x.reshape(batch, s.groups, a // s.groups, b)


def _axes(s):
    return (1, 3) if s.last else (2, 3)


def _per_channel(s, w):
    return w.view(1, 1, s.groups, -1) if s.last else w.view(1, s.groups, -1, 1)


def _group_stats(s, x):
    mean = x.mean(_axes(s), keepdim=True)
    return mean, ((x - mean).square().mean(_axes(s), keepdim=True) + s.eps).rsqrt()


def _activation(act, z):
    return z if act == "none" else z.clamp(min=0.0) if act == "relu" else z / (1.0 + (-z).exp())


def plain_gnorm_forward(s):
    x = _grouped(s, s.x.float())
    mean, rstd = _group_stats(s, x)
    y = _activation(s.act, (x - mean) * rstd * _per_channel(s, s.weight) + _per_channel(s, s.bias))
    return {"y": y.to(s.x.dtype).view(s.shape), "mean": mean.flatten(1), "rstd": rstd.flatten(1)}


def plain_gnorm_backward(s):
    x, dy, w = _grouped(s, s.x.float()), _grouped(s, s.dy.float()), _per_channel(s, s.weight)
    mean, rstd = s.stats[:, :, None, :, None] if s.last else s.stats[:, :, :, None, None]
    hat = (x - mean) * rstd
    if s.act == "silu":
        z = hat * w + _per_channel(s, s.bias)
        q = 1.0 / (1.0 + (-z).exp())
        dy = dy * (q * (1.0 + z * (1.0 - q)))
    u = dy * w
    axes = _axes(s)
    dx = rstd * (u - u.mean(axes, keepdim=True) - hat * (u * hat).mean(axes, keepdim=True))
    over = (0, 1) if s.last else (0, 3)
    return {"dx": dx.to(s.x.dtype).view(s.shape), "dweight": (dy * hat).sum(over).flatten(),
            "dbias": dy.sum(over).flatten()}


def _scan(a, b):
    """h_t = a_t h_(t-1) + b_t along the middle axis, in steps of doubled reach."""
    reach = 1
    while reach < a.shape[1]:
        b = torch.cat([b[:, :reach], a[:, reach:] * b[:, :-reach] + b[:, reach:]], 1)
        a = torch.cat([a[:, :reach], a[:, reach:] * a[:, :-reach]], 1)
        reach *= 2
    return b


def _coefficients(s):
    """a, 1 - a and b of every step, and a where the state stays (0 where it is dropped)."""
    gate, x = s.gate.float(), s.x.float()
    if s.kind == "sigmoid":
        a, rest = 1.0 / (1.0 + (-gate).exp()), 1.0 / (1.0 + gate.exp())
        b = rest * x
    else:
        a, rest, b = gate.exp(), None, x
    return a, rest, b, a if s.resets is None else a.masked_fill(s.resets.unsqueeze(2) != 0, 0.0)


def _states(s, kept, b):
    first = b[:, :1] + kept[:, :1] * s.h0.unsqueeze(1)
    return _scan(kept, torch.cat([first, b[:, 1:]], 1))


def plain_recur_forward(s):
    _, _, b, kept = _coefficients(s)
    h = _states(s, kept, b)
    return {"y": h.to(s.x.dtype), "last": h[:, -1]}


def plain_recur_backward(s):
    a, rest, b, kept = _coefficients(s)
    h = _states(s, kept, b)
    before = torch.cat([s.h0.unsqueeze(1), h[:, :-1]], 1)
    if s.resets is not None:
        before = before.masked_fill(s.resets.unsqueeze(2) != 0, 0.0)
    del h
    # dh_t = dy_t + a_(t+1) dh_(t+1), from the last step to the first
    later = torch.cat([kept[:, 1:], torch.ones_like(kept[:, :1])], 1).flip(1)
    dy = s.dy.float().flip(1)
    dh = _scan(later, torch.cat([dy[:, :1] + s.dlast.unsqueeze(1), dy[:, 1:]], 1)).flip(1)
    if s.kind == "sigmoid":
        dgate, dx = dh * (before - s.x.float()) * a * rest, dh * rest
    else:
        dgate, dx = dh * before * a, dh
    return {"dgate": dgate.to(s.x.dtype), "dx": dx.to(s.x.dtype), "dh0": kept[:, 0] * dh[:, 0]}


def _orthogonal(u):
    """u with singular values near 1, by Newton-Schulz products."""
    x = u.t() if u.shape[0] > u.shape[1] else u
    x = x / (x.square().sum().sqrt() + EPS)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        gram = torch.mm(x, x.t())
        x = a * x + torch.mm(b * gram + c * torch.mm(gram, gram), x)
    return x.t() if u.shape[0] > u.shape[1] else x


def plain_orthogonalize(s):
    for at, (r, c) in zip(s.starts, s.shapes):
        s.p[at:at + r * c].view(r, c).copy_(_orthogonal(s.g[at:at + r * c].view(r, c).float()))
    return {"out": s.p}


def _signed(word):
    return word - (1 << 32) if word >= 1 << 31 else word


def _round_by_chance(p, step):
    """p with its low 16 bits rounded away by hashed bits of each value's place."""
    key = (SEED * 0x6A09E667 + step * 0xBB67AE85) & 0xFFFFFFFF
    x = torch.arange(p.numel(), dtype=torch.int32, device=p.device) * _signed(0x9E3779B9) + _signed(key)
    x = (x ^ ((x >> 15) & 0x1FFFF)) * _signed(0xBB67AE85)
    x = (x ^ ((x >> 16) & 0xFFFF)) * _signed(0x6A09E667)
    return ((p.view(torch.int32) + ((x >> 16) & 0xFFFF)) & -65536).view(torch.float32)


def plain_muon_step(s):
    g = s.g.float()
    s.m = MOMENTUM * s.m + g
    u = g + MOMENTUM * s.m
    p = s.p.float() * (1.0 - LR * DECAY)
    for at, (r, c) in zip(s.starts, s.shapes):
        scale = LR * math.sqrt(max(1.0, r / c))
        p[at:at + r * c].view(r, c).sub_(scale * _orthogonal(u[at:at + r * c].view(r, c)))
    s.p.copy_(p if s.p.dtype == torch.float32 else _round_by_chance(p, s.step))
    return {"p": s.p, "m": s.m}


# ---- one pass -------------------------------------------------------------------
def _own_gnorm_forward(s):
    s.plan.forward(s.x, s.weight, s.bias, s.y, s.stats, s.ws)
    return {"y": s.y.view(s.shape), "mean": s.stats[0], "rstd": s.stats[1]}


def _own_gnorm_backward(s):
    s.plan.backward(s.dy, s.x, s.weight, s.bias, s.stats, s.dx, s.dweight, s.dbias, s.ws)
    return {"dx": s.dx.unflatten(1, s.shape[1:]), "dweight": s.dweight, "dbias": s.dbias}


def _own_recur_forward(s):
    s.plan.forward(s.gate, s.x, s.y, s.ws, h0=s.h0, last=s.last, resets=s.resets)
    return {"y": s.y, "last": s.last}


def _own_recur_backward(s):
    s.plan.backward(s.gate, s.x, s.dy, s.states, s.dgate, s.dx, s.ws, dlast=s.dlast, dh0=s.dh0, resets=s.resets)
    return {"dgate": s.dgate, "dx": s.dx, "dh0": s.dh0}


def _own_orthogonalize(s):
    s.plan.orthogonalize(s.tensors, s.ws, eps=EPS)
    return {"out": s.p}


def _own_muon_step(s):
    s.plan.step(s.tensors, s.state, s.ws, lr=LR, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY, eps=EPS,
                step=s.step, seed=SEED)
    return {"p": s.p, "m": s.plan.momentum(s.state)}


def run(s):
    got = globals()[("_own_" if own else "plain_") + s.op](s)
    if s.op == "muon_step":
        s.step += 1
    return got


# ---- the same in 64 bits, written from the definitions ---------------------------
def _exact_gnorm(case, s):
    batch, groups, channels = case["batch"], case["groups"], case["channels"]
    to_first = (lambda t: t.view(s.shape).transpose(1, 2)) if s.last else (lambda t: t.view(s.shape))

    def back(t):  # [batch][channels][sites] as the case lays it out
        return t.transpose(1, 2) if s.last else t

    def spread(t):  # [batch][groups] at each channel
        return t.repeat_interleave(channels // groups, 1)[:, :, None]

    x = to_first(s.x.double().contiguous())
    w, b = s.weight.double()[None, :, None], s.bias.double()[None, :, None]
    rows = x.reshape(batch, groups, -1)
    size = rows.shape[2]
    mean = rows.sum(2) / size
    rstd = 1.0 / ((rows - mean[:, :, None]).pow(2).sum(2) / size + s.eps).sqrt()
    hat = (x - spread(mean)) * spread(rstd)
    z = hat * w + b
    q = torch.sigmoid(z)
    if case["op"] == "gnorm_forward":
        y = z * q if s.act == "silu" else torch.relu(z) if s.act == "relu" else z
        return {"y": back(y), "mean": mean, "rstd": rstd}
    dz = to_first(s.dy.double())
    if s.act == "silu":  # (z q)' = q + z q (1 - q)
        dz = dz * (q + z * q * (1.0 - q))
    u = dz * w

    def group_sum(t):
        return spread(t.reshape(batch, groups, -1).sum(2))

    # y = hat w + b;  d hat_i / d x_j = rstd (delta_ij - 1 / size - hat_i hat_j / size)
    dx = spread(rstd) * (u - (group_sum(u) + hat * group_sum(u * hat)) / size)
    return {"dx": back(dx), "dweight": (dz * hat).sum(2).sum(0), "dbias": dz.sum(2).sum(0)}


def _exact_recur(case, s):
    gate, x = s.gate.double(), s.x.double()
    a = torch.sigmoid(gate) if s.kind == "sigmoid" else gate.exp()
    rest = torch.sigmoid(-gate) if s.kind == "sigmoid" else torch.ones_like(a)
    kept = a if s.resets is None else a * (s.resets == 0)[:, :, None]
    b, h, held = rest * x, s.h0.double(), torch.empty_like(a)
    for t in range(case["length"]):
        h = torch.addcmul(b[:, t], kept[:, t], h)
        held[:, t] = h
    if case["op"] == "recur_forward":
        return {"y": held, "last": h}
    before = torch.cat([s.h0.double()[:, None], held[:, :-1]], 1)
    if s.resets is not None:
        before = before * (s.resets == 0)[:, :, None]
    dh, carried, dy = torch.empty_like(a), s.dlast.double(), s.dy.double()
    for t in reversed(range(case["length"])):
        carried = carried + dy[:, t]
        dh[:, t] = carried
        carried = carried * kept[:, t]
    if s.kind == "sigmoid":
        return {"dgate": dh * (before - x) * a * (1.0 - a), "dx": dh * rest, "dh0": carried}
    return {"dgate": dh * before * a, "dx": dh, "dh0": carried}


def _exact_orthogonal(u):
    x = u / (torch.linalg.vector_norm(u) + EPS)
    a, b, c = COEFFICIENTS
    tall = u.shape[0] > u.shape[1]
    for _ in range(STEPS):  # x (a + b x^T x + c (x^T x)^2), from the shorter side
        gram = x.t() @ x if tall else x @ x.t()
        p = (c * gram @ gram + b * gram).contiguous()
        p.diagonal().add_(a)
        x = x @ p if tall else p @ x
    return x


def _exact_muon(case, s):
    if case["op"] == "orthogonalize":
        out = torch.zeros(s.p.numel(), dtype=torch.float64, device="cuda")
        for at, (r, c) in zip(s.starts, s.shapes):
            out[at:at + r * c] = _exact_orthogonal(s.g[at:at + r * c].double().view(r, c)).reshape(-1)
        return {"out": out}
    m = s.m.double() * MOMENTUM + s.g.double()
    u, p = s.g.double() + MOMENTUM * m, s.p.double()
    p = p - LR * DECAY * p
    for at, (r, c) in zip(s.starts, s.shapes):
        p[at:at + r * c] -= LR * math.sqrt(max(1.0, r / c)) * _exact_orthogonal(u[at:at + r * c].view(r, c)).reshape(-1)
    # parameters of 16 bits are rounded by chance: their value before that
    return {"p": p, "m": m}


def exact(case, seed):
    s = prepare(case, seed)
    return {"gnor": _exact_gnorm, "recu": _exact_recur, "muon": _exact_muon, "orth": _exact_muon}[s.op[:4]](case, s)
