"""The operators around the convolution in a training step or an answer, and what they have to give.

A case is one call:

  norm_forward      layer norm of x [outer][size][inner] over its middle axis: y and (mean, 1 / deviation)
  norm_backward     its gradients: of x, and of weight and bias summed over outer and inner
  logprob_forward   of rows of logits: each row's given class's log probability, the row's entropy and
                    its `top` likeliest classes with theirs
  logprob_backward  the gradient of the logits from those of log probability and entropy
  adamw             one AdamW step over many tensors, moments in 32 bits or in 8

``listed()`` holds sizes of the time-series network and of the ResNet- and DenseNet-shaped stacks
(maps of 512 samples, 4 x 4 and 56 x 56 points, their parameter lists) and generic ones beside them;
``draw()`` samples the ranges they stand for: rows of 1 to 262144 values, batches of 1 to 65536 rows, channel
counts of 1 to 1024 on maps of 2 to 4096 points, 2 to 262144 classes, 1 to 400 tensors of one value to
millions, three types.

Moments of 8 bits, as ``plain_adamw`` computes them: blocks of 128 values of a tensor share a power of two S,
the largest that does not exceed the block's largest magnitude (at least 2^-96).  The first moment is held as
a sign, 4 bits of exponent and 3 of fraction of |m| / S, the second as 5 bits of exponent and 3 of fraction of
v / S; both are rounded down or up with a chance that makes the held value right on average, by 16 bits of a
hash of the value's place, the step and a seed.  A positive second moment is never held as zero, and what is
not finite is held as NaN.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ALIGN = 1024  # a tensor's values start at a multiple of this many in the moments' layout
BLOCK = 128   # values that share a power of two

LR, BETA1, BETA2, EPS, DECAY, SEED = 2e-3, 0.9, 0.999, 1e-8, 0.05, 20


# ---- cases ----------------------------------------------------------------------
def _norm(op, outer, size, inner, dtype, gap=0):
    """gap > 0: x and dx are slices of tensors whose outer stride is that many values longer."""
    return {"op": op, "outer": outer, "size": size, "inner": inner, "dtype": dtype, "gap": gap}


def _logprob(op, rows, classes, dtype, top=0, masked=False, entropy=False, gap=0):
    """masked: about a third of the classes of each row at minus infinity, and one row wholly."""
    return {"op": op, "rows": rows, "classes": classes, "dtype": dtype, "top": top, "masked": masked,
            "entropy": entropy, "gap": gap}


def _adamw(net, bits, param="f32", grad="f32", tensors=0, most=0, mix=0):
    """net: a parameter list by name, or "drawn": `tensors` sizes of 1 to `most` values by the number `mix`."""
    return {"op": "adamw", "net": net, "bits": bits, "param": param, "grad": grad, "tensors": tensors,
            "most": most, "mix": mix}


def listed():
    return [
        # pooled features of a few series before the classifier: latency
        dict(_norm("norm_forward", 4, 128, 1, "f32"), name="norm_pooled_4x128_forward"),
        # over the channels at every sample of the time-series network's widest map
        dict(_norm("norm_forward", 64, 256, 512, "f32"), name="norm_channels_64x256x512_forward"),
        # the same layer's gradients
        dict(_norm("norm_backward", 64, 256, 512, "f32"), name="norm_channels_64x256x512_backward"),
        # whole images of the large-image layer, 64 channels of 56 x 56 points each
        dict(_norm("norm_forward", 32, 200704, 1, "f32"), name="norm_images_32x200704_forward"),
        # tokens with their features side by side, in reduced precision
        dict(_norm("norm_backward", 16384, 2048, 1, "bf16"), name="norm_tokens_16384x2048_backward"),
        # one answer of a large vocabulary of odd size, with its eight likeliest tokens
        dict(_logprob("logprob_forward", 1, 131071, "bf16", top=8), name="logprob_1x131071_top8"),
        # a batch of answers, some tokens ruled out
        dict(_logprob("logprob_forward", 513, 50021, "f32", top=20, masked=True), name="logprob_513x50021_top20"),
        # the loss of a series classifier (50 classes, batch 50): latency
        dict(_logprob("logprob_backward", 50, 50, "f32", entropy=True), name="logprob_50x50_backward"),
        # the loss of a language model's step
        dict(_logprob("logprob_backward", 4096, 65536, "bf16"), name="logprob_4096x65536_backward"),
        # the time-series network's parameters: latency
        dict(_adamw("fcn", 32), name="adamw_fcn_32"),
        # an 18-layer residual network's, gradients in reduced precision
        dict(_adamw("resnet", 32, grad="bf16"), name="adamw_resnet_32"),
        # a model of some hundred million, moments in 8 bits
        dict(_adamw("wide", 8, grad="bf16"), name="adamw_wide_8"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    return work(case)["bytes"]


def draw(rng):
    op = rng.choice(["norm_forward", "norm_backward", "logprob_forward", "logprob_backward", "adamw", "adamw"])
    dtype = rng.choice(["f32", "f32", "bf16", "f16"])
    gap = rng.choice([0, 0, 0, 1, 8, 40])
    if op.startswith("norm"):
        if rng.random() < 0.5:
            case = _norm(op, _log_int(rng, 1, 65536), _log_int(rng, 1, 262144), 1, dtype, gap)
        else:
            case = _norm(op, _log_int(rng, 1, 256), _log_int(rng, 1, 1024), _log_int(rng, 2, 4096), dtype, gap)
        shrink = ("outer", "size", "inner")
    elif op.startswith("logprob"):
        classes = _log_int(rng, 2, 262144)
        top = 0 if op == "logprob_backward" or rng.random() < 0.3 else _log_int(rng, 1, min(64, classes))
        case = _logprob(op, _log_int(rng, 1, 16384), classes, dtype, top, rng.random() < 0.4,
                        op == "logprob_backward" and rng.random() < 0.5, gap)
        shrink = ("rows", "classes")
    else:
        case = _adamw("drawn", rng.choice([32, 8]), rng.choice(["f32", "f32", "bf16"]),
                      rng.choice(["f32", "bf16", "f16"]), _log_int(rng, 1, 400), _log_int(rng, 16, 1 << 22),
                      rng.randint(1, 1 << 20))
        shrink = ("most",)
    most = max(_cost(x) for x in listed())
    while _cost(case) > most:
        k = next(k for k in shrink if case[k] > 64 or k == shrink[-1])
        case[k] = max(1, case[k] * 3 // 4)
    return case


def _sizes(case):
    """[(values, decayed)] of the tensors, in the order of the network's layers."""
    def conv(ci, co, taps):
        return [(ci * co * taps, True), (co, False), (co, False)]  # filters, then the norm's weight and bias

    if case["net"] == "fcn":  # 1 -> 128 -> 256 -> 128 channels, 8, 5 and 3 taps, 50 classes
        return conv(1, 128, 8) + conv(128, 256, 5) + conv(256, 128, 3) + [(128 * 50, True), (50, False)]
    if case["net"] == "resnet":  # four stages of two blocks of two 3 x 3 layers
        got, ci = conv(3, 64, 9), 64
        for co in (64, 128, 256, 512):
            for layer in range(4):
                got += conv(ci if layer == 0 else co, co, 9)
                if layer == 0 and ci != co:
                    got += conv(ci, co, 1)
            ci = co
        return got + [(512 * 10, True), (10, False)]
    if case["net"] == "wide":  # ten blocks of width 1024 with a four times wider inner layer
        got, d = [], 1024
        for _ in range(10):
            got += [(d, False), (d, False), (4 * d * d, True), (4 * d, False), (d, False), (d, False),
                    (4 * d * d, True), (4 * d, False), (4 * d * d, True), (d, False)]
        return got
    rng = random.Random(case["mix"])
    sizes = [_log_int(rng, 1, case["most"]) for _ in range(case["tensors"])]
    return [(n, rng.random() < 0.6) for n in sizes]


def _layout(case):
    """Where each tensor starts in the moments' layout, and its length."""
    starts, at = [], 0
    for n, _ in _sizes(case):
        starts.append(at)
        at += -(-n // ALIGN) * ALIGN
    return starts, at


def work(case):
    """Inputs in and outputs out once; elementary operations per value of the formulas."""
    if case["op"].startswith("norm"):
        n, sites = case["outer"] * case["size"] * case["inner"], case["outer"] * case["inner"]
        wide = TYPES[case["dtype"]].itemsize
        if case["op"] == "norm_forward":
            return {"bytes": 2 * n * wide + 8 * case["size"] + 8 * sites, "flops": 7 * n}
        return {"bytes": 3 * n * wide + 12 * case["size"] + 8 * sites, "flops": 14 * n}
    if case["op"].startswith("logprob"):
        n, wide = case["rows"] * case["classes"], TYPES[case["dtype"]].itemsize
        if case["op"] == "logprob_forward":
            return {"bytes": n * wide + case["rows"] * (16 + 12 * case["top"]), "flops": 6 * n}
        return {"bytes": 2 * n * wide + case["rows"] * 28, "flops": 5 * n}
    n = sum(k for k, _ in _sizes(case))
    params = 2 * TYPES[case["param"]].itemsize + TYPES[case["grad"]].itemsize
    # moments read and written; those of 8 bits are read again and given back in two bytes each
    moments = 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 4
    return {"bytes": n * (params + moments), "flops": (15 if case["bits"] == 32 else 60) * n}


# ---- inputs ---------------------------------------------------------------------
class _State:
    """A program's inputs, plan, workspace and output buffers."""


def _random(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, device="cuda", generator=g, dtype=dtype)

    return g, normal


def _with_gap(rows, length, gap, dtype):
    """[rows][length] values whose rows lie `gap` values further apart."""
    return torch.empty(rows, length + gap, dtype=dtype, device="cuda")[:, :length]


def _prepare_norm(s, case, seed):
    _, normal = _random(seed)
    outer, size, inner, dtype = case["outer"], case["size"], case["inner"], TYPES[case["dtype"]]
    s.shape, s.eps = (outer, size, inner), 1e-5
    flat = size * inner
    s.x = _with_gap(outer, flat, case["gap"], dtype)
    x = normal(outer, size, inner, dtype=dtype)
    x = x.mul_(1.5).add_(normal(1, size, 1).to(dtype))  # channels with means of their own
    s.x.copy_(x.view(outer, flat))
    del x
    s.weight = 1.0 + 0.2 * normal(size)
    s.bias = 0.3 * normal(size)
    if case["op"] == "norm_forward":
        s.y = torch.empty(outer, flat, dtype=dtype, device="cuda")
        s.stats = torch.empty(2, outer, inner, device="cuda")
    else:
        s.dy = normal(outer, flat, dtype=dtype)
        s.stats = torch.stack(_norm_stats(s.x.reshape(s.shape).float(), s.eps)).squeeze(2).contiguous()
        s.dx = _with_gap(outer, flat, case["gap"], dtype)
        s.dweight, s.dbias = torch.empty_like(s.weight), torch.empty_like(s.bias)
    if own:
        from paper_1911_09287_amd import bltrain
        s.plan = bltrain.NormPlan(outer, size, inner, dtype=dtype, eps=s.eps, x_stride=flat + case["gap"])
        s.ws = s.plan.workspace("cuda")


def _prepare_logprob(s, case, seed):
    g, normal = _random(seed)
    rows, classes, dtype = case["rows"], case["classes"], TYPES[case["dtype"]]
    s.top, s.with_entropy = case["top"], case["entropy"]
    s.logits = _with_gap(rows, classes, case["gap"], dtype)
    s.logits.copy_(normal(rows, classes, dtype=dtype).mul_(3.0))
    if case["masked"]:
        out = torch.rand(rows, classes, device="cuda", generator=g) < 1.0 / 3.0
        out[seed % rows] = True
        s.logits.masked_fill_(out, -math.inf)
        del out
    s.targets = torch.randint(0, classes, (rows,), device="cuda", generator=g)
    s.targets[torch.rand(rows, device="cuda", generator=g) < 0.05] = -1  # places that hold no token
    if case["op"] == "logprob_forward":
        s.logp = torch.empty(rows, device="cuda")
        s.stats = torch.empty(3, rows, device="cuda")
        s.top_logp = torch.empty(rows, s.top, device="cuda")
        s.top_index = torch.empty(rows, s.top, dtype=torch.int64, device="cuda")
    else:
        s.stats = torch.cat([torch.stack(_row_stats(part.float())[:3]) for part in s.logits.split(1024)], 1)
        s.g_logp = normal(rows) / rows
        s.g_entropy = 0.01 * normal(rows) / rows if s.with_entropy else None
        s.dlogits = torch.empty(rows, classes, dtype=dtype, device="cuda")
    if own:
        from paper_1911_09287_amd import bltrain
        s.plan = bltrain.LogProbPlan(rows, classes, top=s.top, dtype=dtype, stride=classes + case["gap"])
        s.ws = s.plan.workspace("cuda")


def _prepare_adamw(s, case, seed):
    g, normal = _random(seed)
    sizes = _sizes(case)
    starts, total = _layout(case)
    s.bits, s.step = case["bits"], 10
    s.inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    s.decayed = torch.zeros(total, dtype=torch.bool, device="cuda")
    for at, (n, decay) in zip(starts, sizes):
        s.inside[at:at + n] = True
        s.decayed[at:at + n] = decay
    # parameters and gradients lie in one buffer each, as a program that sums
    # gradients over GPUs in one piece keeps them
    s.p = (0.05 * normal(total)).mul_(s.inside).to(TYPES[case["param"]])
    s.g = (1e-3 * normal(total)).mul_(s.inside).to(TYPES[case["grad"]])
    s.m = (3e-4 * normal(total)).mul_(s.inside)
    s.v = (1e-6 * normal(total).square()).mul_(s.inside)
    if s.bits == 8:
        dither = torch.full((total,), 1 << 15, dtype=torch.int32, device="cuda")
        s.m, s.v = _held_m(s.m, dither), _held_v(s.v, dither)
    s.grad_scale = torch.full((1,), 0.75, device="cuda")  # a clipped norm's factor
    if own:
        from paper_1911_09287_amd import bltrain
        s.plan = bltrain.AdamWPlan([n for n, _ in sizes], param_dtype=s.p.dtype, grad_dtype=s.g.dtype, bits=s.bits,
                                   decay=[d for _, d in sizes])
        s.tensors = s.plan.bind([s.p[at:at + n] for at, (n, _) in zip(starts, sizes)],
                                [s.g[at:at + n] for at, (n, _) in zip(starts, sizes)])
        s.state = s.plan.state("cuda")
        s.plan.load_moments(s.state, s.m, s.v)


def prepare(case, seed):
    s = _State()
    s.op = case["op"]
    {"norm": _prepare_norm, "logprob": _prepare_logprob, "adamw": _prepare_adamw}[s.op.split("_")[0]](s, case, seed)
    return s


# ---- the plain forms ------------------------------------------------------------
def _norm_stats(x, eps):
    mean = x.mean(1, keepdim=True)
    return mean, ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()


def plain_norm_forward(s):
    x = s.x.reshape(s.shape).float()
    mean, rstd = _norm_stats(x, s.eps)
    y = (x - mean) * rstd * s.weight.view(1, -1, 1) + s.bias.view(1, -1, 1)
    return {"y": y.to(s.x.dtype), "mean": mean, "rstd": rstd}


def plain_norm_backward(s):
    x, dy = s.x.reshape(s.shape).float(), s.dy.view(s.shape).float()
    mean, rstd = s.stats.unsqueeze(2)
    hat, g = (x - mean) * rstd, dy * s.weight.view(1, -1, 1)
    dx = rstd * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
    return {"dx": dx.to(s.x.dtype), "dweight": (dy * hat).sum((0, 2)), "dbias": dy.sum((0, 2))}


def _row_stats(z):
    """Per row: the maximum, the log of the sum of exp(z - maximum), the entropy; and z - maximum."""
    top = z.amax(1)
    d = z - top.masked_fill(top == -math.inf, 0.0).unsqueeze(1)
    e = d.exp()
    total = e.sum(1)
    entropy = total.log() - (e * d).masked_fill(e == 0, 0.0).sum(1) / total
    return top, total.log(), entropy.masked_fill(top == -math.inf, 0.0), d


def _in_row(targets, classes):
    return (targets >= 0) & (targets < classes)


def plain_logprob_forward(s):
    z = s.logits.float()
    top, log_sum, entropy, d = _row_stats(z)
    empty = (top == -math.inf).unsqueeze(1)
    there = _in_row(s.targets, z.shape[1])
    at = torch.where(there, s.targets, 0).unsqueeze(1)
    logp = (d.gather(1, at) - log_sum.unsqueeze(1)).masked_fill(empty, -math.inf).squeeze(1)
    got = {"logp": torch.where(there, logp, 0.0), "entropy": entropy}
    if s.top:
        # one whole number for a value and its place, so that equal values go by the lower place
        bits = (z + 0.0).view(torch.int32)
        order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).masked_fill(z.isnan(), 0x7FFFFFFF)
        last = z.shape[1] - 1
        keys = (order.to(torch.int64) << 32) | (last - torch.arange(last + 1, device=z.device))
        index = last - (keys.topk(s.top, 1).values & 0xFFFFFFFF)
        got["top_logp"] = (d.gather(1, index) - log_sum.unsqueeze(1)).masked_fill(empty, -math.inf)
        got["top_index"] = index
    return got


def plain_logprob_backward(s):
    z = s.logits.float()
    top, log_sum, entropy = s.stats.unsqueeze(2)
    there = _in_row(s.targets, z.shape[1])
    logq = z - top.masked_fill(top == -math.inf, 0.0) - log_sum
    q = logq.exp().masked_fill(top == -math.inf, 0.0)
    g = torch.where(there, s.g_logp, 0.0).unsqueeze(1)
    dz = -g * q
    if s.with_entropy:
        dz = dz - s.g_entropy.unsqueeze(1) * (q * (logq + entropy)).masked_fill(q == 0, 0.0)
    dz.scatter_add_(1, torch.where(there, s.targets, 0).unsqueeze(1), g.masked_fill(top == -math.inf, 0.0))
    return {"dlogits": dz.to(s.logits.dtype)}


def _signed(word):
    return word - (1 << 32) if word >= 1 << 31 else word


def _dither(total, step, device):
    """32 hashed bits for each value's place, as int32 words."""
    key = (SEED * 0x6A09E667 + step * 0xBB67AE85) & 0xFFFFFFFF
    x = torch.arange(total, dtype=torch.int32, device=device) * _signed(0x9E3779B9) + _signed(key)
    x = (x ^ ((x >> 15) & 0x1FFFF)) * _signed(0xBB67AE85)
    return x ^ ((x >> 16) & 0xFFFF)


def _scale(a):
    """The power of two that each block of magnitudes shares, at each of its values."""
    largest = a.masked_fill(~a.isfinite(), 0.0).view(-1, BLOCK).amax(1, keepdim=True)
    power = (largest.view(torch.int32) & 0x7F800000).view(torch.float32).clamp(min=2.0 ** -96)
    return power.expand(-1, BLOCK).reshape(-1)


def _code(a, scale, down, dither16):
    """Exponent and fraction bits of a / scale, rounded by 16 bits of dither."""
    t = (a / scale * 2.0 ** -down).view(torch.int32)
    return (t + (dither16 << 4)) >> 20


def _value(code, scale, down):
    return (code << 20).view(torch.float32) * 2.0 ** down * scale


def _held_m(m, dither16):
    """m as its 8 bits hold it (exact in bfloat16)."""
    a = m.abs()
    scale = _scale(a)
    held = _value(_code(a.masked_fill(~a.isfinite(), 0.0), scale, 113, dither16), scale, 113)
    return torch.copysign(held, m).masked_fill(~a.isfinite(), math.nan).bfloat16()


def _held_v(v, dither16):
    scale = _scale(v)
    code = _code(v.masked_fill(~v.isfinite(), 0.0), scale, 97, dither16)
    held = _value(torch.maximum(code, (v > 0).to(torch.int32)), scale, 97)
    return held.masked_fill(~v.isfinite(), math.nan).bfloat16()


def plain_adamw(s):
    rest1, rest2 = 1.0 - BETA1 ** s.step, 1.0 - BETA2 ** s.step
    g = s.g.float() * s.grad_scale
    m = s.m.float() * BETA1 + g * (1.0 - BETA1)
    v = s.v.float() * BETA2 + g * g * (1.0 - BETA2)
    p = s.p.float()
    p = torch.where(s.decayed, p * (1.0 - LR * DECAY), p)
    p = p - m * (LR / rest1) / (v.sqrt() * (1.0 / math.sqrt(rest2)) + EPS)
    if s.bits == 8 or s.p.dtype != torch.float32:
        dither = _dither(p.numel(), s.step, p.device)
    if s.bits == 8:
        m, v = _held_m(m, dither & 0xFFFF), _held_v(v, (dither >> 16) & 0xFFFF)
    if s.p.dtype != torch.float32:
        up = ((dither * _signed(0x6A09E667)) >> 16) & 0xFFFF
        p = ((p.view(torch.int32) + up) & -65536).view(torch.float32)
    s.m, s.v = m, v
    s.p.copy_(p)
    return {"p": s.p, "m": s.m, "v": s.v}


# ---- one pass -------------------------------------------------------------------
def _own_norm_forward(s):
    s.plan.forward(s.x, s.weight, s.bias, s.y, s.stats, s.ws)
    mean, rstd = s.stats.unsqueeze(2)
    return {"y": s.y.view(s.shape), "mean": mean, "rstd": rstd}


def _own_norm_backward(s):
    s.plan.backward(s.dy, s.x, s.weight, s.stats, s.dx, s.dweight, s.dbias, s.ws)
    return {"dx": s.dx.unflatten(1, s.shape[1:]), "dweight": s.dweight, "dbias": s.dbias}


def _own_logprob_forward(s):
    s.plan.forward(s.logits, s.targets, s.logp, s.stats, s.top_logp, s.top_index, s.ws)
    got = {"logp": s.logp, "entropy": s.stats[2]}
    return dict(got, top_logp=s.top_logp, top_index=s.top_index) if s.top else got


def _own_logprob_backward(s):
    s.plan.backward(s.logits, s.targets, s.stats, s.g_logp, s.g_entropy, s.dlogits)
    return {"dlogits": s.dlogits}


def _own_adamw(s):
    s.plan.step(s.tensors, s.state, lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY,
                step=s.step, grad_scale=s.grad_scale, seed=SEED)
    m, v = s.plan.moments(s.state)  # views of 32-bit moments; 8-bit ones as bfloat16 values
    return {"p": s.p, "m": m, "v": v}


def run(s):
    got = globals()[("_own_" if own else "plain_") + s.op](s)
    if s.op == "adamw":
        s.step += 1
    return got


# ---- the same in 64 bits, written from the definitions ---------------------------
def _exact_norm(case, s):
    outer, size, inner = s.shape
    x = s.x.reshape(s.shape).double()
    w, b = s.weight.double()[None, :, None], s.bias.double()[None, :, None]
    mean = x.sum(1, keepdim=True) / size
    var = (x - mean).pow(2).sum(1, keepdim=True) / size
    rstd = 1.0 / (var + s.eps).sqrt()
    hat = (x - mean) * rstd
    if case["op"] == "norm_forward":
        return {"y": hat * w + b, "mean": mean, "rstd": rstd}
    dy = s.dy.view(s.shape).double()
    # y = hat w + b;  d hat_i / d x_j = rstd (delta_ij - 1 / size - hat_i hat_j / size)
    u = dy * w
    dx = rstd * (u - (u.sum(1, keepdim=True) + hat * (u * hat).sum(1, keepdim=True)) / size)
    return {"dx": dx, "dweight": (dy * hat).sum(2).sum(0), "dbias": dy.sum(2).sum(0)}


def _exact_logprob(case, s):
    got = []
    for at in range(0, case["rows"], 1024):
        z = s.logits[at:at + 1024].double()
        t, rows = s.targets[at:at + 1024], torch.arange(z.shape[0], device=z.device)
        empty, there = (z == -math.inf).all(1), t >= 0
        lse = torch.logsumexp(z, 1)
        logq = z - torch.where(empty, 0.0, lse)[:, None]
        q = torch.where(empty[:, None], 0.0, logq.exp())
        entropy = -torch.special.xlogy(q, q).sum(1)
        if case["op"] == "logprob_forward":
            logp = torch.where(there, logq[rows, t.clamp(min=0)], 0.0)
            part = {"logp": logp, "entropy": entropy}
            if case["top"]:
                top, index = z.sort(stable=True, dim=1, descending=True)
                part["top_logp"] = top[:, :case["top"]] - torch.where(empty, 0.0, lse)[:, None]
                part["top_index"] = index[:, :case["top"]]
        else:
            g = torch.where(there & ~empty, s.g_logp[at:at + 1024].double(), 0.0)
            dz = -g[:, None] * q
            dz[rows, t.clamp(min=0)] += g
            if case["entropy"]:
                dz -= s.g_entropy[at:at + 1024].double()[:, None] * (torch.special.xlogy(q, q) + q * entropy[:, None])
            part = {"dlogits": dz}
        got.append(part)
    return {k: torch.cat([p[k] for p in got]) for k in got[0]}


def _exact_held(a, most, chance):
    """Magnitudes as held: `most` is the exponent code of the block's power of two, chance in [0, 1)."""
    blocks = a.view(-1, BLOCK)
    power = torch.floor(torch.log2(blocks.amax(1, keepdim=True).clamp(min=2.0 ** -96)))
    rel = blocks * torch.exp2(-power)
    exponent = torch.floor(torch.log2(rel.clamp(min=2.0 ** (1 - most))))
    unit = torch.exp2(exponent - 3.0)
    held = torch.floor(rel / unit + chance.view(-1, BLOCK)) * unit
    return held, power, 2.0 ** (-2 - most)


def _exact_adamw(case, s):
    t, total = s.step, s.p.numel()
    g = s.g.double() * s.grad_scale.double()
    m = s.m.double() * BETA1 + (1.0 - BETA1) * g
    v = s.v.double() * BETA2 + (1.0 - BETA2) * g * g
    p = s.p.double() * (1.0 - LR * DECAY * s.decayed.double())
    p = p - LR * (m / (1.0 - BETA1 ** t)) / ((v / (1.0 - BETA2 ** t)).sqrt() + EPS)
    if case["bits"] == 8:
        mask = 0xFFFFFFFF
        x = (torch.arange(total, device="cuda") * 0x9E3779B9 + SEED * 0x6A09E667 + t * 0xBB67AE85) & mask
        x = ((x ^ (x >> 15)) * 0xBB67AE85) & mask
        x = x ^ (x >> 16)
        held, power, _ = _exact_held(m.abs(), 14, (x & 0xFFFF) / 65536.0)
        m = (held * torch.exp2(power)).view(-1) * m.sign()
        held, power, least = _exact_held(v, 30, (x >> 16) / 65536.0)
        held = torch.where(v.view(-1, BLOCK) > 0, held.clamp(min=least), 0.0)
        v = (held * torch.exp2(power)).view(-1)
    # parameters of 16 bits are rounded by chance: their value before that
    return {"p": p, "m": m, "v": v}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "logprob": _exact_logprob, "adamw": _exact_adamw}[s.op.split("_")[0]](case, s)
