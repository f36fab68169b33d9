"""The operators around the convolution layer against plain implementations in 64 bits (MI355X).

Tolerances come from the arithmetic, before any run.  U = 2^-24 is half an ulp
of fp32, relative.  A tree or blocked sum of n fp32 terms is taken to be off by
at most 16 U times the sum of their magnitudes (log2 n + the lengths of the
serial parts, in the worst case of one sign), statistics and a handful of
elementary operations by a few U more; a result of 16 bits adds half an ulp of
its type.  Outputs are filled with NaN (or -7 for whole numbers) before a call,
so that an element that is not written fails.
"""
import math

import numpy as np
import pytest

from paper_1911_09287_amd import blconv, bltrain

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch as _torch
    if not _torch.cuda.is_available():
        pytest.skip("no GPU")
    blconv.load()
    return _torch


def half_ulp(dtype):
    return {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dtype]


def tdtype(torch, name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def near(got, want, bound, what=""):
    """|got - want| <= bound where want is finite; the same infinities and NaN elsewhere."""
    got, want = got.double().cpu(), want.double().cpu()
    bound = bound if isinstance(bound, float) else bound.double().cpu()
    fine = want.isfinite()
    assert (got.isnan() == want.isnan()).all(), what
    assert (got[~fine & ~want.isnan()] == want[~fine & ~want.isnan()]).all(), what
    over = ((got - want).abs() - bound)
    over = over[fine]
    assert over.numel() == 0 or over.max().item() <= 0, (what, over.max().item(), int((over > 0).sum()), over.numel())


# ---- layer norm -------------------------------------------------------------------
ROWS = [(1, 1, 1), (3, 1, 1), (3, 5, 1), (5, 7, 1), (2, 63, 1), (2, 64, 1), (9, 65, 1), (300, 33, 1), (17, 128, 1),
        (3, 255, 1), (4, 257, 1), (3, 1000, 1), (2, 1025, 1), (7, 2047, 1), (3, 4099, 1), (2, 8192, 1), (3, 16385, 1),
        (2, 33000, 1), (1, 65537, 1), (2, 200704, 1), (1, 262144, 1), (600, 768, 1), (4000, 64, 1), (513, 2050, 1)]
MAPS = [(2, 3, 2), (4, 1, 33), (3, 5, 7), (2, 33, 49), (2, 128, 16), (1, 256, 270), (3, 512, 16), (2, 64, 56 * 56),
        (2, 1024, 9), (1, 1500, 6), (1, 2100, 40), (5, 17, 3), (70, 128, 4), (2, 130, 513), (64, 100, 25),
        (2, 300, 9), (1, 513, 5), (1, 300, 6), (2, 700, 6), (1, 270, 130), (1, 600, 4), (2, 1024, 12), (3, 65, 35),
        (1, 40, 7)]


def norm_reference(x, w, b, dy, eps):
    """y, mean, rstd, dx, dw, db in 64 bits, and the scale of what their errors are made of."""
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    h = (x - mean) * rstd
    wv, bv = w.view(1, -1, 1), b.view(1, -1, 1)
    u = dy * wv
    c1, c2 = u.mean(1, keepdim=True), (u * h).mean(1, keepdim=True)
    return {"y": h * wv + bv, "mean": mean, "rstd": rstd, "dx": rstd * (u - c1 - h * c2),
            "dw": (dy * h).sum((0, 2)), "db": dy.sum((0, 2)), "h": h, "u": u}


def norm_bounds(x, w, b, dy, r, eps, dtype, wdtype):
    # h: the mean is off by 16 U mean|x| and the subtraction by U |x - mean|; rstd by
    # 16 U relative (a sum of squares) and by half the relative change that the mean's
    # error makes in the variance, |d mean| rstd at most
    size = x.shape[1]
    big = x.abs().amax(1, keepdim=True)
    dmean = 16 * U * big
    drel = 24 * U + dmean * r["rstd"]
    dh = dmean * r["rstd"] + r["h"].abs() * drel + 2 * U * r["h"].abs()
    wv, bv = w.abs().view(1, -1, 1), b.abs().view(1, -1, 1)
    t = half_ulp(dtype)
    got = {"mean": dmean + 1e-30, "rstd": r["rstd"] * drel}
    got["y"] = dh * wv + 3 * U * (r["h"].abs() * wv + bv) + t * r["y"].abs() + 2.0 ** -25 * (dtype == "f16")
    # means over the row of u and u h: 16 U of the mean of magnitudes, and h's own error
    au = r["u"].abs()
    d1 = 18 * U * au.mean(1, keepdim=True)
    d2 = 18 * U * (au * r["h"].abs()).mean(1, keepdim=True) + (au * dh).mean(1, keepdim=True)
    c2 = (au * r["h"].abs()).mean(1, keepdim=True)
    parts = au + au.mean(1, keepdim=True) + r["h"].abs() * c2
    got["dx"] = r["rstd"] * (d1 + r["h"].abs() * d2 + dh * c2 + 6 * U * parts) + r["rstd"] * drel * parts \
        + t * r["dx"].abs() + 2.0 ** -25 * (dtype == "f16")
    tw = half_ulp(wdtype)
    got["dw"] = 18 * U * (dy * r["h"]).abs().sum((0, 2)) + (dy.abs() * dh).sum((0, 2)) + tw * r["dw"].abs() + 1e-30
    got["db"] = 18 * U * dy.abs().sum((0, 2)) + tw * r["db"].abs() + 1e-30
    return got


def norm_inputs(torch, shape, dtype, wdtype, seed, offset=0.5):
    g = torch.Generator().manual_seed(seed)
    outer, size, inner = shape
    x = (torch.randn(shape, generator=g) * 1.5 + offset).to(tdtype(torch, dtype))
    dy = torch.randn(shape, generator=g).to(tdtype(torch, dtype))
    w = (1 + 0.3 * torch.randn(size, generator=g)).to(tdtype(torch, wdtype))
    b = (0.3 * torch.randn(size, generator=g)).to(tdtype(torch, wdtype))
    return x, dy, w, b


def run_norm(torch, shape, x, dy, w, b, dtype, wdtype, eps, x_gap=0, y_gap=0, shift=0, weights=True, grads=True):
    """The plan's results, on tensors whose slices lie `gap` elements further apart and start `shift` elements in."""
    outer, size, inner = shape
    flat, dt = size * inner, tdtype(torch, dtype)
    plan = bltrain.NormPlan(outer, size, inner, dtype=dt, wdtype=tdtype(torch, wdtype), eps=eps,
                            x_stride=flat + x_gap, y_stride=flat + y_gap)

    def place(t, gap):
        room = torch.full((outer * (flat + gap) + shift,), float("nan"), dtype=dt, device="cuda")
        view = room[shift:].view(outer, flat + gap)[:, :flat]
        if t is not None:
            view.copy_(t.reshape(outer, flat))
        return view

    xs, ds = place(x, x_gap), place(dy, y_gap)
    y, dx = place(None, y_gap), place(None, x_gap)
    ws = plan.workspace()
    ws.fill_(255)
    wd, bd = (w.cuda(), b.cuda()) if weights else (None, None)
    stats = torch.full(plan.stats_shape(), float("nan"), device="cuda")
    dw = torch.full((size,), float("nan"), dtype=tdtype(torch, wdtype), device="cuda") if grads else None
    db = torch.full((size,), float("nan"), dtype=tdtype(torch, wdtype), device="cuda") if grads else None
    plan.forward(xs, wd, bd, y, stats, ws)
    ws.fill_(255)
    plan.backward(ds, xs, wd, stats, dx, dw, db, ws)
    torch.cuda.synchronize()
    got = {"y": y.reshape(shape), "mean": stats[0].view(outer, 1, inner), "rstd": stats[1].view(outer, 1, inner),
           "dx": dx.reshape(shape)}
    if grads:
        got.update(dw=dw, db=db)
    return got


def check_norm(torch, shape, dtype, wdtype, eps=1e-5, offset=0.5, seed=0, **kw):
    x, dy, w, b = norm_inputs(torch, shape, dtype, wdtype, seed, offset)
    if not kw.get("weights", True):
        w, b = torch.ones_like(w), torch.zeros_like(b)
    got = run_norm(torch, shape, x, dy, w, b, dtype, wdtype, eps, **kw)
    x, dy, w, b = (t.double() for t in (x, dy, w, b))
    r = norm_reference(x, w, b, dy, eps)
    bound = norm_bounds(x, w, b, dy, r, eps, dtype, wdtype)
    for name, t in got.items():
        near(t, r[name], bound[name], (shape, dtype, name))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", ROWS + MAPS, ids=str)
def test_norm_against_64_bits(torch, shape, dtype):
    check_norm(torch, shape, dtype, "f32", seed=sum(shape))


@pytest.mark.parametrize("shape", [(5, 130, 1), (3, 4099, 1), (2, 40000, 1), (3, 20, 18), (2, 130, 33), (4, 64, 64)],
                         ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_norm_strides_offsets_and_weight_types(torch, shape, dtype):
    for k, (xg, yg, shift) in enumerate([(1, 0, 0), (0, 3, 1), (8, 40, 0), (5, 5, 3)]):
        check_norm(torch, shape, dtype, dtype if k % 2 else "f32", x_gap=xg, y_gap=yg, shift=shift, seed=k)
    check_norm(torch, shape, dtype, dtype, weights=False)
    check_norm(torch, shape, dtype, dtype, grads=False)


@pytest.mark.parametrize("shape", [(4, 96, 1), (3, 3000, 1), (2, 70000, 1), (2, 48, 20)], ids=str)
def test_norm_far_from_zero(torch, shape):
    # a mean of 3000 deviations: sums of squares of the values themselves would lose the variance
    check_norm(torch, shape, "f32", "f32", offset=4500.0)


def test_norm_eps_and_constant_rows(torch):
    plan = bltrain.NormPlan(2, 50, eps=0.25)
    x = torch.full((2, 50), 3.0, device="cuda")
    y, stats = torch.empty_like(x), torch.empty(2, 2, 1, device="cuda")
    bias = torch.arange(50.0, device="cuda")
    plan.forward(x, None, bias, y, stats, plan.workspace())
    assert (y == bias).all() and (stats[0] == 3.0).all() and (stats[1] == 2.0).all()


def test_norm_not_finite_stays_in_its_row(torch):
    for shape in [(3, 100, 1), (3, 5000, 1), (3, 70000, 1)]:
        plan = bltrain.NormPlan(*shape)
        x = torch.randn(shape[:2], device="cuda")
        x[1, 7] = float("inf")
        y, stats = torch.empty_like(x), torch.empty(plan.stats_shape(), device="cuda")
        plan.forward(x, None, None, y, stats, plan.workspace())
        assert y[1].isnan().all() and y[0].isfinite().all() and y[2].isfinite().all()
    plan = bltrain.NormPlan(2, 40, 30)
    x = torch.randn(2, 40, 30, device="cuda")
    x[1, 3, 5] = float("nan")
    y, stats = torch.empty_like(x), torch.empty(plan.stats_shape(), device="cuda")
    plan.forward(x, None, None, y, stats, plan.workspace())
    bad = torch.zeros(2, 40, 30, dtype=torch.bool, device="cuda")
    bad[1, :, 5] = True
    assert (y.isnan() == bad).all()


@pytest.mark.parametrize("shape", [(5, 1, 1), (300, 1, 1), (2, 1, 163), (3, 1, 8)], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_one_value_has_no_gradient(torch, shape, dtype):
    # y = bias whatever x is; 1 / deviation is 1 / sqrt(eps) = 316 times any rounding left over
    x, dy, w, b = norm_inputs(torch, shape, dtype, "f32", 1)
    got = run_norm(torch, shape, x, dy, w, b, dtype, "f32", 1e-5)
    assert (got["dx"] == 0).all() and (got["dw"] == 0).all()


def test_norm_either_weight_gradient_alone(torch):
    for shape in [(40, 300, 1), (2, 70000, 1), (3, 40, 50)]:
        x, dy, w, b = (t.cuda() for t in norm_inputs(torch, shape, "f32", "f32", 2))
        plan = bltrain.NormPlan(*shape)
        ws, stats, y = plan.workspace(), torch.empty(plan.stats_shape(), device="cuda"), torch.empty_like(x)
        plan.forward(x, w, b, y, stats, ws)
        both = [torch.empty_like(w) for _ in range(2)]
        plan.backward(dy, x, w, stats, torch.empty_like(x), *both, ws)
        dw, db, dx = torch.empty_like(w), torch.empty_like(w), torch.empty_like(x)
        plan.backward(dy, x, w, stats, dx, dw, None, ws)
        plan.backward(dy, x, w, stats, dx, None, db, ws)
        assert torch.equal(dw, both[0]) and torch.equal(db, both[1])


def test_norm_of_no_rows(torch):
    plan = bltrain.NormPlan(0, 40)
    none = torch.empty(0, 40, device="cuda")
    dw, db = torch.full((40,), 5.0, device="cuda"), torch.full((40,), 5.0, device="cuda")
    stats = torch.empty(2, 0, 1, device="cuda")
    plan.forward(none, None, None, none, stats, plan.workspace())
    plan.backward(none, none, None, stats, none, dw, db, plan.workspace())
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("shape", [(6, 200, 1), (3, 6000, 1), (2, 80000, 1), (4, 40, 36), (2, 1200, 8)], ids=str)
def test_norm_in_place_and_without_stats(torch, shape):
    x, dy, w, b = norm_inputs(torch, shape, "f32", "f32", 3)
    want = run_norm(torch, shape, x, dy, w, b, "f32", "f32", 1e-5)
    plan = bltrain.NormPlan(*shape)
    ws, stats = plan.workspace(), torch.stack([want["mean"], want["rstd"]]).contiguous()
    xs, ds, wd = x.cuda(), dy.cuda(), w.cuda()
    plan.forward(xs, wd, b.cuda(), xs, None, ws)
    assert torch.equal(xs.view(shape), want["y"])
    for into in ("dy", "x"):
        xs, ds = x.cuda(), dy.cuda()
        dw, db = torch.empty(shape[1], device="cuda"), torch.empty(shape[1], device="cuda")
        plan.backward(ds, xs, wd, stats, ds if into == "dy" else xs, dw, db, ws)
        assert torch.equal((ds if into == "dy" else xs).view(shape), want["dx"])
        assert torch.equal(dw, want["dw"]) and torch.equal(db, want["db"])


@pytest.mark.parametrize("shape", [(7, 60, 1), (3, 2500, 1), (3, 12, 25)], ids=str)
def test_norm_gradients_against_differences(torch, shape):
    # the loss <dy, y> in 64 bits of the kernel's own y, along a random direction of x, weight and bias.
    # h = 2^-6: the third derivative's term is h^2 / 6 times O(1) per value, rounding 2^-24 / h per value,
    # both small against 1 % of the norms' product
    x, dy, w, b = (t.cuda() for t in norm_inputs(torch, shape, "f32", "f32", 4))
    plan = bltrain.NormPlan(*shape)
    ws, stats, y = plan.workspace(), torch.empty(plan.stats_shape(), device="cuda"), torch.empty_like(x)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    plan.forward(x, w, b, y, stats, ws)
    plan.backward(dy, x, w, stats, dx, dw, db, ws)
    g = torch.Generator(device="cuda").manual_seed(5)
    for k, (t, grad) in enumerate(((x, dx), (w, dw), (b, db))):
        v = torch.randn(t.shape, device="cuda", generator=g)
        loss, h = [], 2.0 ** -6
        for sign in (1, -1):
            args = [x, w, b]
            args[k] = t + sign * h * v
            plan.forward(*args, y, None, ws)
            loss.append((y.double() * dy.double()).sum().item())
        along = (grad.double() * v.double()).sum().item()
        scale = grad.double().norm().item() * v.double().norm().item()
        assert abs((loss[0] - loss[1]) / (2 * h) - along) <= 0.01 * scale, k


def test_norm_refuses_wrong_tensors(torch):
    plan = bltrain.NormPlan(2, 8)
    x, ws = torch.zeros(2, 8, device="cuda"), plan.workspace()
    stats = torch.zeros(plan.stats_shape(), device="cuda")
    for bad in (x.half(), x[:, :7], x.cpu(), torch.zeros(8, 2, device="cuda").T):
        with pytest.raises(ValueError):
            plan.forward(bad, None, None, x, stats, ws)
        with pytest.raises(ValueError):
            plan.forward(x, None, None, bad, stats, ws)
    with pytest.raises(ValueError):
        plan.forward(x, torch.zeros(7, device="cuda"), None, x, stats, ws)
    with pytest.raises(ValueError):
        plan.forward(x, None, None, x, stats[0], ws)
    wide = bltrain.NormPlan(2, 8, x_stride=10)
    with pytest.raises(ValueError):
        wide.forward(x, None, None, x, stats, wide.workspace())


def test_norm_offsets_past_32_bits(torch):
    # two slices more than 2^32 bytes apart: rows, long rows, channels
    for shape, gap in [((2, 700, 1), 1 << 30), ((2, 40000, 1), 1 << 30), ((2, 24, 10), 1 << 30)]:
        check_norm(torch, shape, "f32", "f32", x_gap=gap, seed=9)
    check_norm(torch, (2, 24, 10), "bf16", "f32", y_gap=(1 << 31) + 6, seed=9)


# ---- log probabilities ------------------------------------------------------------
def logprob_reference(torch, z, targets, top, g=None, ge=None):
    z = z.double()
    rows, classes = z.shape
    m = z.amax(1)
    none = m == -math.inf
    d = z - torch.where(none, 0.0, m)[:, None]
    e = d.exp()
    log_sum = e.sum(1).log()
    logq = d - torch.where(none, 0.0, log_sum)[:, None]
    q = torch.where(none[:, None], 0.0, logq.exp())
    entropy = -torch.where(q == 0, 0.0, q * logq).sum(1)
    there = (targets >= 0) & (targets < classes)
    at = torch.where(there, targets, 0)
    r = {"logp": torch.where(there, logq[torch.arange(rows), at], 0.0), "entropy": entropy, "logq": logq, "q": q,
         "d": d}
    order = torch.where(z.isnan(), math.inf, z + 0.0)  # (tests have no infinity beside a NaN)
    index = order.sort(dim=1, descending=True, stable=True).indices[:, :top]
    r["top_index"] = torch.nn.functional.pad(index, (0, top - index.shape[1]), value=-1)
    r["top_logp"] = torch.nn.functional.pad(logq.gather(1, index), (0, top - index.shape[1]), value=-math.inf)
    if g is not None:
        ga = torch.where(there & ~none, g.double(), 0.0)
        dz = -ga[:, None] * q
        dz[torch.arange(rows), at] += ga
        if ge is not None:
            dz -= ge.double()[:, None] * torch.where(q == 0, 0.0, q * (logq + entropy[:, None]))
        r["dz"] = dz
    return r


def check_logprob(torch, z, targets, top, dtype, gap=0, shift=0, entropy_grad=True, seed=0):
    rows, classes = z.shape
    dt = tdtype(torch, dtype)
    z = z.to(dt)
    gen = torch.Generator().manual_seed(seed)
    g, ge = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)
    plan = bltrain.LogProbPlan(rows, classes, top=top, dtype=dt, stride=classes + gap, grad_stride=classes + 2 * gap)

    def place(step):
        room = torch.full((rows * step + shift,), float("nan"), dtype=dt, device="cuda")
        return room[shift:].view(rows, step)[:, :classes]

    zs, dz = place(classes + gap), place(classes + 2 * gap)
    zs.copy_(z)
    nan = float("nan")
    logp, stats = torch.full((rows,), nan, device="cuda"), torch.full((3, rows), nan, device="cuda")
    top_logp = torch.full((rows, top), nan, device="cuda")
    top_index = torch.full((rows, top), -7, dtype=torch.int64, device="cuda")
    ws = plan.workspace()
    ws.fill_(255)
    t = targets.cuda()
    plan.forward(zs, t, logp, stats, top_logp, top_index, ws)
    plan.backward(zs, t, stats, g.cuda(), ge.cuda() if entropy_grad else None, dz)
    torch.cuda.synchronize()
    r = logprob_reference(torch, z, targets, top, g, ge if entropy_grad else None)
    # z - m is rounded once, exp and the sum are off by 20 U relative, the log by that and U of itself
    log_n = math.log(classes) + 1.0
    dl = 24 * U + 4 * U * log_n
    name = (rows, classes, top, dtype)
    near(logp, r["logp"], dl + 4 * U * r["logp"].abs().nan_to_num(0, 0, 0), name + ("logp",))
    near(stats[2], r["entropy"], 2 * dl + 40 * U * log_n, name + ("entropy",))
    assert torch.equal(top_index.cpu(), r["top_index"]), name
    near(top_logp, r["top_logp"], dl + 4 * U * r["top_logp"].abs().nan_to_num(0, 0, 0), name + ("top",))
    # q off by dl and by U |log q| relative; the entropy's gradient by H's error and the factor's rounding
    lq = r["logq"].abs().clamp(max=200.0).nan_to_num(0)
    dq = r["q"] * (dl + 6 * U * (lq + 1))
    bound = (g.abs()[:, None] * (dq + 2 * U)).double()
    if entropy_grad:
        bound = bound + ge.abs()[:, None].double() * (dq * (lq + log_n) + r["q"] * (3 * dl + 48 * U * (log_n + lq)))
    bound = bound + half_ulp(dtype) * r["dz"].abs() + (2.0 ** -25 if dtype == "f16" else 1e-37)
    near(dz, r["dz"], bound.nan_to_num(0), name + ("dz",))


LOGITS = [(1, 1, 1), (3, 2, 2), (5, 50, 5), (70, 7, 3), (300, 10, 0), (2, 63, 8), (2, 64, 64), (9, 65, 1), (4, 255, 20),
          (4, 1000, 0), (3, 1025, 64), (33, 2049, 8), (3, 4097, 20), (2, 9000, 33), (1, 16385, 8), (2, 50021, 20),
          (1, 131071, 8), (1, 262144, 64), (40, 20000, 2), (700, 513, 4)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,classes,top", LOGITS)
def test_logprob_against_64_bits(torch, rows, classes, top, dtype):
    g = torch.Generator().manual_seed(rows + classes)
    z = 3.0 * torch.randn(rows, classes, generator=g)
    t = torch.randint(-1, classes + 1, (rows,), generator=g)  # -1 and classes: no target
    check_logprob(torch, z, t, top, dtype)
    check_logprob(torch, z, t, top, dtype, gap=1 + classes % 3, shift=1, entropy_grad=False, seed=1)


@pytest.mark.parametrize("classes", [3, 64, 200, 3000, 40000])
def test_logprob_ties_orders_and_extremes(torch, classes):
    g = torch.Generator().manual_seed(classes)
    few = torch.randint(-2, 3, (1, classes), generator=g).float()  # many equal values
    rising = torch.arange(classes).float().view(1, -1) / classes   # every class beats those before it
    rows = [few, rising, rising.flip(1), torch.zeros(1, classes), -few.abs(),
            torch.where(torch.rand(1, classes, generator=g) < 0.5, torch.tensor(0.0), torch.tensor(-0.0)),
            3e4 * few + 1e4, torch.full((1, classes), torch.finfo(torch.float32).min),
            torch.where(few > 0, few, torch.tensor(torch.finfo(torch.float32).min))]
    z = torch.cat(rows)
    t = torch.randint(0, classes, (len(rows),), generator=g)
    for top in (1, 5, 64):
        check_logprob(torch, z, t, top, "f32")
    lowest = torch.cat([few, rising, torch.full((1, classes), torch.finfo(torch.bfloat16).min)])
    check_logprob(torch, lowest, t[:3], 8, "bf16")


@pytest.mark.parametrize("classes", [2, 70, 1500, 33000])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_logprob_masked_rows(torch, classes, dtype):
    g = torch.Generator().manual_seed(classes)
    z = torch.randn(6, classes, generator=g)
    z[0] = -math.inf                                             # nothing left
    z[1, torch.rand(classes, generator=g) < 0.7] = -math.inf
    z[2] = -math.inf
    z[2, classes - 1] = 1.5                                      # one class left: certain
    z[3, : classes // 2] = -math.inf
    z[4] = -math.inf
    z[4, 0] = -2.0
    t = torch.tensor([1, classes // 2, classes - 1, 0, classes - 1, -1])
    for top in (0, 1, 9):
        check_logprob(torch, z, t, top, dtype)


@pytest.mark.parametrize("classes", [5, 300, 20000])
def test_logprob_not_finite(torch, classes):
    z = torch.randn(4, classes)
    z[1, classes // 2] = math.nan
    z[2, classes - 2] = math.inf
    z[2, 0] = -math.inf
    t = torch.tensor([1, 0, 1, 2])
    check_logprob(torch, z, t, 3, "f32")
    check_logprob(torch, z, t, 3, "bf16")


def test_logprob_offsets_past_32_bits(torch):
    for classes, top in [(300, 3), (20000, 3)]:
        z = torch.randn(3, classes)
        check_logprob(torch, z, torch.tensor([1, 2, 3]), top, "f32", gap=1 << 30)


def test_logprob_optional_outputs_and_in_place(torch):
    rows, classes = 9, 777
    z = torch.randn(rows, classes, device="cuda")
    t = torch.randint(0, classes, (rows,), device="cuda")
    plan = bltrain.LogProbPlan(rows, classes)
    ws = plan.workspace()
    logp, stats = torch.empty(rows, device="cuda"), torch.empty(3, rows, device="cuda")
    plan.forward(z, t, logp, stats, None, None, ws)
    alone = torch.empty(rows, device="cuda")
    plan.forward(z, t, alone, None, None, None, ws)
    assert torch.equal(alone, logp)
    again = torch.empty(3, rows, device="cuda")
    plan.forward(z, None, None, again, None, None, ws)
    assert torch.equal(again, stats)
    g, ge = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    dz = torch.empty_like(z)
    plan.backward(z, t, stats, g, ge, dz)
    inplace = z.clone()
    plan.backward(inplace, t, stats, g, ge, inplace)
    assert torch.equal(inplace, dz)
    plan.backward(z, None, stats, g, None, dz)
    assert (dz == 0).all()


def test_logprob_gradient_against_differences(torch):
    # the loss sum g logp + ge entropy in 64 bits of the kernel's outputs, along a random direction;
    # h = 2^-6: h^2 / 6 and 2^-24 / h per row, small against 1 % of the norms' product
    rows, classes, h = 6, 300, 2.0 ** -6
    gen = torch.Generator(device="cuda").manual_seed(1)
    z, v = (torch.randn(rows, classes, device="cuda", generator=gen) for _ in range(2))
    g, ge = (torch.randn(rows, device="cuda", generator=gen) for _ in range(2))
    t = torch.randint(0, classes, (rows,), device="cuda", generator=gen)
    plan = bltrain.LogProbPlan(rows, classes)
    ws, logp, stats = plan.workspace(), torch.empty(rows, device="cuda"), torch.empty(3, rows, device="cuda")
    dz = torch.empty_like(z)
    plan.forward(z, t, logp, stats, None, None, ws)
    plan.backward(z, t, stats, g, ge, dz)
    loss = []
    for sign in (1, -1):
        plan.forward(z + sign * h * v, t, logp, stats, None, None, ws)
        loss.append((g.double() * logp.double() + ge.double() * stats[2].double()).sum().item())
    along = (dz.double() * v.double()).sum().item()
    assert abs((loss[0] - loss[1]) / (2 * h) - along) <= 0.01 * dz.double().norm().item() * v.double().norm().item()


def test_logprob_refuses_wrong_tensors(torch):
    plan = bltrain.LogProbPlan(3, 20, top=2)
    z, t = torch.zeros(3, 20, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    f, k = torch.zeros(3, 2, device="cuda"), torch.zeros(3, 2, dtype=torch.int64, device="cuda")
    logp, stats, ws = torch.zeros(3, device="cuda"), torch.zeros(3, 3, device="cuda"), plan.workspace()
    plan.forward(z, t, logp, stats, f, k, ws)
    for args in ((z.half(), t, logp, stats, f, k), (z, t.int(), logp, stats, f, k), (z, t, logp[:2], stats, f, k),
                 (z, t, logp, stats[:2], f, k), (z, t, logp, stats, f[:, :1], k), (z, t, logp, stats, f, k.int())):
        with pytest.raises(ValueError):
            plan.forward(*args, ws)
    with pytest.raises(bltrain.BlError):
        plan.forward(z, t, logp, stats, None, None, ws)


# ---- AdamW ------------------------------------------------------------------------
def held(a, signed, dither16):
    """The header's 8-bit values of magnitudes a (numpy fp32, blocks of 128), without NaN."""
    down, up = (np.float32(2.0 ** -113), np.float32(2.0 ** 113)) if signed else (np.float32(2.0 ** -97), np.float32(2.0 ** 97))
    b = a.reshape(-1, 128)
    s = np.maximum((b.max(1, keepdims=True).view(np.uint32) & np.uint32(0x7F800000)).view(np.float32),
                   np.float32(2.0 ** -96))
    code = ((b / s * down).view(np.uint32) + (dither16.reshape(-1, 128) << np.uint32(4))) >> np.uint32(20)
    if not signed:
        code = np.where((b > 0) & (code == 0), np.uint32(1), code)
    return ((code << np.uint32(20)).astype(np.uint32).view(np.float32) * up * s).reshape(-1)


def words(total, step, seed):
    key = np.uint32((seed * 0x6A09E667 + step * 0xBB67AE85) & 0xFFFFFFFF)
    x = np.arange(total, dtype=np.uint32) * np.uint32(0x9E3779B9) + key
    x = (x ^ (x >> np.uint32(15))) * np.uint32(0xBB67AE85)
    return x ^ (x >> np.uint32(16))


LISTS = [[1], [5], [1024], [1025, 3], [0, 7, 0, 2000, 1, 128, 129], [4096, 1023, 300000, 64, 65], [77] * 300,
         [1, 5000] * 130 + [0, 0, 9]]


def adamw_setup(torch, sizes, param, grad, bits, seed, shift=0):
    g = torch.Generator().manual_seed(seed)
    decay = [i % 3 != 1 for i in range(len(sizes))]
    plan = bltrain.AdamWPlan(sizes, param_dtype=tdtype(torch, param), grad_dtype=tdtype(torch, grad), bits=bits,
                             decay=decay)

    def fresh(scale, dtype):
        ts = []
        for n in sizes:  # guards of NaN on both sides, `shift` elements off alignment
            room = torch.full((n + 16 + shift,), float("nan"), dtype=tdtype(torch, dtype), device="cuda")
            room[8 + shift:8 + shift + n] = (scale * torch.randn(n, generator=g)).to(tdtype(torch, dtype)).cuda()
            ts.append(room)
        return ts, [r[8 + shift:8 + shift + n] for r, n in zip(ts, sizes)]

    return plan, decay, fresh(0.1, param), fresh(1e-2, grad)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"),
                                        ("bf16", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}x{sum(s)}")
def test_adamw_against_64_bits(torch, sizes, param, grad, bits):
    lr, b1, b2, eps, wd, seed, scale = 3e-3, 0.9, 0.95, 1e-6, 0.1, 11, 0.5
    plan, decay, (rooms, params), (_, grads) = adamw_setup(torch, sizes, param, grad, bits, len(sizes), shift=1)
    tensors, state = plan.bind(params, grads), plan.state()
    gs = torch.full((1,), scale, device="cuda")
    total = plan.total
    m, v = np.zeros(total, np.float32), np.zeros(total, np.float32)
    where = [(at, n) for at, n in zip(plan.starts, sizes)]
    for t in range(1, 4):
        before = [p.double().cpu().numpy() for p in params]
        plan.step(tensors, state, lr=lr, betas=(b1, b2), eps=eps, weight_decay=wd, step=t, grad_scale=gs, seed=seed)
        # the moments in fp32, one rounding an operation: the kernel's are the same, bit for bit
        g = np.zeros(total, np.float32)
        for (at, n), x in zip(where, grads):
            g[at:at + n] = x.float().cpu().numpy() * np.float32(scale)
        m = m * np.float32(b1) + g * np.float32(1 - b1)
        v = v * np.float32(b2) + g * g * np.float32(1 - b2)
        m64, v64 = m.astype(np.float64), v.astype(np.float64)
        if bits == 8:
            w = words(total, t, seed)
            m = np.copysign(held(np.abs(m), True, w & np.uint32(0xFFFF)), m)
            v = held(v, False, w >> np.uint32(16))
        got_m, got_v = plan.moments(state)
        for i, (at, n) in enumerate(where):
            assert (got_m[at:at + n].float().cpu().numpy() == m[at:at + n]).all(), (t, i)
            assert (got_v[at:at + n].float().cpu().numpy() == v[at:at + n]).all(), (t, i)
            up = lr / (1 - b1 ** t) * m64[at:at + n] / (np.sqrt(v64[at:at + n] / (1 - b2 ** t)) + eps)
            want = before[i] * (1 - lr * wd * decay[i]) - up
            # a dozen roundings of the update, three of the parameter; bfloat16 by chance: a whole ulp
            bound = 16 * U * np.abs(up) + 3 * U * np.abs(before[i]) + 1e-30
            if param == "bf16":
                bound += 2.0 ** -7 * np.abs(want)
            off = np.abs(params[i].double().cpu().numpy() - want) - bound
            assert n == 0 or off.max() <= 0, (t, i, off.max())
    for room, n in zip(rooms, sizes):  # nothing beside the tensors is written
        assert room[:9].isnan().all() and room[9 + n:].isnan().all()


def test_adamw_live_scalars_equal_the_hosts(torch):
    for bits in (32, 8):
        got = []
        for live in (False, True):
            plan, _, (_, params), (_, grads) = adamw_setup(torch, [3000, 50, 700], "f32", "f32", bits, 3)
            tensors, state = plan.bind(params, grads), plan.state()
            clock = torch.tensor([0.0, 0.0], dtype=torch.float64, device="cuda")
            for t in range(1, 5):
                clock.copy_(torch.tensor([1e-3 * t, t]))
                plan.step(tensors, state, lr=0.0 if live else 1e-3 * t, step=1 if live else t, weight_decay=0.1, seed=9,
                          live=clock if live else None)
            got.append([p.clone() for p in params] + list(plan.moments(state)))
        # pow of the device and of the host may differ in the last bits of 64
        for a, b in zip(*got):
            near(b, a, 4 * U * a.abs() + 4e-3 * 4 * U)


def test_adamw_not_finite_gradients(torch):
    for bits in (32, 8):
        plan = bltrain.AdamWPlan([300], bits=bits)
        p, g = torch.ones(300, device="cuda"), torch.full((300,), 0.5, device="cuda")
        g[7], g[200] = float("nan"), float("inf")
        state = plan.state()
        tensors = plan.bind([p], [g])
        plan.step(tensors, state, lr=0.1, step=1)
        bad = torch.zeros(300, dtype=torch.bool, device="cuda")
        bad[7] = bad[200] = True
        assert (p.isnan() == bad).all()
        m, v = plan.moments(state)
        if bits == 8:
            assert (m[:300].isnan() == bad).all() and (v[:300].isnan() == bad).all()
        good = m[:300][~bad].float()
        assert ((good - 0.05).abs() <= 0.05 / 8).all()
        g[7], g[200] = 0.5, 0.5
        plan.step(tensors, state, lr=0.1, step=2)
        assert (p.isnan() == bad).all()  # they do not spread


def test_adamw_moments_round_trip(torch):
    for bits in (32, 8):
        plan = bltrain.AdamWPlan([5000, 130], bits=bits)
        g = torch.Generator(device="cuda").manual_seed(2)
        m = torch.randn(plan.total, device="cuda", generator=g) * torch.randn(plan.total, device="cuda", generator=g).exp()
        v = m.square()
        state = plan.state()
        plan.load_moments(state, m, v)
        a = [t.clone() for t in plan.moments(state)]
        # to nearest: half a step of an eighth, or half the smallest step of the block
        if bits == 8:
            for x, y, least in ((m, a[0], 2.0 ** -17), (v, a[1], 2.0 ** -33)):
                block = x.abs().view(-1, 128).amax(1, keepdim=True).expand(-1, 128).reshape(-1)
                near(y, x, x.abs() / 16 + block * least * 2)
        other = plan.state()
        plan.load_moments(other, *a)
        for x, y in zip(a, plan.moments(other)):
            assert torch.equal(x, y)
        if bits == 32:
            copies = plan.moments(state, torch.empty_like(m), torch.empty_like(v))
            assert torch.equal(copies[0], m) and torch.equal(copies[1], v)


def test_adamw_8_bit_second_moment_decays(torch):
    # without gradients v falls by 0.1 % a step, far less than its codes' 6 %; rounding by
    # chance holds it right on average.  Each step's rounding has a relative deviation of
    # at most 1/16; after 1000 steps that of one value is below sqrt(1000 * 0.001) / 8 or so
    # and that of a mean over 65536 values below 0.2 %: 5 % leaves room
    n = 65536
    plan = bltrain.AdamWPlan([n], bits=8)
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    state = plan.state()
    v0 = torch.rand(n, device="cuda") + 0.5
    plan.load_moments(state, torch.zeros(n, device="cuda"), v0)
    start = plan.moments(state)[1].double().mean().item()
    tensors = plan.bind([p], [g])
    for t in range(1, 1001):
        plan.step(tensors, state, lr=0.0, betas=(0.9, 0.999), step=t, seed=4)
    mean = plan.moments(state)[1].double().mean().item()
    assert abs(mean / (start * 0.999 ** 1000) - 1) < 0.05


def test_adamw_8_bit_positive_second_moment_stays_positive(torch):
    plan = bltrain.AdamWPlan([256], bits=8)
    state = plan.state()
    v = torch.full((256,), 1e-20, device="cuda")
    v[0], v[128], v[129] = 1.0, 1.0, 0.0
    full = torch.zeros(plan.total, device="cuda")
    full[:256] = v
    plan.load_moments(state, torch.zeros_like(full), full)
    got = plan.moments(state)[1][:256]
    assert ((got > 0) == (v > 0)).all()


def test_adamw_bfloat16_parameters_move_on_average(torch):
    # steps of 1/64 of an ulp: to nearest the parameters would never move.  4096 values, 256 steps:
    # the mean is off by one part in sqrt(4096 * 256 / 64) ~ 128 of a step's, so within 5 %
    n, steps = 4096, 256
    plan = bltrain.AdamWPlan([n], param_dtype=torch.bfloat16)
    p, g = torch.full((n,), 1.5, dtype=torch.bfloat16, device="cuda"), torch.ones(n, device="cuda")
    tensors, state = plan.bind([p], [g]), plan.state()
    lr = 2.0 ** -7 / 64
    for t in range(1, steps + 1):
        plan.step(tensors, state, lr=lr, eps=0.0, weight_decay=0.0, step=t, seed=1)
    moved = 1.5 - p.double().mean().item()
    assert abs(moved / (lr * steps) - 1) < 0.05


def test_adamw_offsets_past_32_bits(torch):
    n = (1 << 31) + 2500  # elements of one tensor: 2^33 bytes of parameters
    for bits in (32, 8):
        plan = bltrain.AdamWPlan([7, n], bits=bits, grad_dtype=torch.bfloat16)
        p = [torch.ones(7, device="cuda"), torch.ones(n, device="cuda")]
        g = [torch.ones(7, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")]
        g[1][-3:] = 1.0
        g[1][:2] = 1.0
        tensors, state = plan.bind(p, g), plan.state()
        plan.step(tensors, state, lr=0.25, weight_decay=0.0, step=1)
        # the first step moves by lr where there is a gradient
        assert (p[0] - 0.75).abs().max().item() < 1e-6
        moved = p[1] != 1.0
        assert moved.sum().item() == 5 and moved[:2].all() and moved[-3:].all()
        m = plan.moments(state)[0]
        assert m[plan.starts[1] + n - 1].item() > 0.09 and m[plan.starts[1] + n - 4].item() == 0
        del p, g, tensors, state, m, moved
        torch.cuda.empty_cache()


def test_adamw_what_lies_between_tensors_has_no_part(torch):
    # a block's power of two goes by the tensor's own values, whatever the state holds past its end
    plan = bltrain.AdamWPlan([100], bits=8)
    g = torch.full((100,), 1e-3, device="cuda")
    state = plan.state()
    full = torch.zeros(plan.total, device="cuda")
    full[110] = 1e9
    plan.load_moments(state, full, full)
    p = torch.zeros(100, device="cuda")
    tensors = plan.bind([p], [g])
    plan.step(tensors, state, step=1)
    m, v = plan.moments(state)
    assert (m[100:] == 0).all() and (v[100:] == 0).all()
    near(m[:100], torch.full((100,), 1e-4), 1e-4 / 8)


def test_adamw_refuses_wrong_tensors(torch):
    plan = bltrain.AdamWPlan([4, 6])
    p = [torch.zeros(4, device="cuda"), torch.zeros(6, device="cuda")]
    tensors, state = plan.bind(p, p), plan.state()
    with pytest.raises(ValueError):
        plan.bind(p, [p[0].half(), p[1]])
    with pytest.raises(ValueError):
        plan.bind([p[1], p[0]], p)
    with pytest.raises(ValueError):
        plan.bind([p[0], torch.zeros(12, device="cuda")[::2]], p)
    with pytest.raises(ValueError):
        plan.step(tensors, state[:-4])
    with pytest.raises(ValueError):
        plan.step(tensors, state, grad_scale=torch.ones(1))
    with pytest.raises(ValueError):
        bltrain.AdamWPlan([4, 6]).step(tensors, state)
    with pytest.raises(bltrain.BlError):
        plan.step(tensors, state, step=0)


# ---- streams, graphs, repeatability -------------------------------------------------
def everything(torch):
    """A call of each operator on fixed inputs: [(outputs, call)]."""
    jobs = []
    for shape in [(40, 300, 1), (9, 5000, 1), (2, 90000, 1), (6, 48, 50), (3, 1100, 5)]:
        x, dy, w, b = (t.cuda() for t in norm_inputs(torch, shape, "f32", "f32", 6))
        plan = bltrain.NormPlan(*shape)
        ws, stats, y = plan.workspace(), torch.empty(plan.stats_shape(), device="cuda"), torch.empty_like(x)
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)

        def norm(plan=plan, x=x, dy=dy, w=w, b=b, ws=ws, stats=stats, y=y, dx=dx, dw=dw, db=db, **kw):
            plan.forward(x, w, b, y, stats, ws, **kw)
            plan.backward(dy, x, w, stats, dx, dw, db, ws, **kw)
        jobs.append(([y, stats, dx, dw, db], norm))
    for rows, classes, top in [(50, 50, 3), (3, 70000, 20), (200, 3000, 5)]:
        g = torch.Generator(device="cuda").manual_seed(classes)
        z = torch.randn(rows, classes, device="cuda", generator=g)
        t = torch.randint(0, classes, (rows,), device="cuda", generator=g)
        plan = bltrain.LogProbPlan(rows, classes, top=top)
        logp, stats, dz = torch.empty(rows, device="cuda"), torch.empty(3, rows, device="cuda"), torch.empty_like(z)
        tl, ti = torch.empty(rows, top, device="cuda"), torch.empty(rows, top, dtype=torch.int64, device="cuda")
        gl = torch.randn(rows, device="cuda", generator=g)

        def prob(plan=plan, z=z, t=t, logp=logp, stats=stats, dz=dz, tl=tl, ti=ti, gl=gl, ws=plan.workspace(), **kw):
            plan.forward(z, t, logp, stats, tl, ti, ws, **kw)
            plan.backward(z, t, stats, gl, gl, dz, **kw)
        jobs.append(([logp, stats, tl, ti, dz], prob))
    for bits in (32, 8):
        sizes = [70, 3000, 1, 1024] * 40
        plan, _, (_, params), (_, grads) = adamw_setup(torch, sizes, "f32", "f32", bits, 8)
        first = [p.clone() for p in params]
        state = plan.state()
        clock = torch.tensor([1e-3, 1.0], dtype=torch.float64, device="cuda")

        def adam(plan=plan, params=params, first=first, tensors=plan.bind(params, grads), state=state, clock=clock, **kw):
            with torch.cuda.stream(kw.get("stream")):
                state.zero_()
                for p, q in zip(params, first):
                    p.copy_(q)
            plan.step(tensors, state, live=clock, **kw)
        jobs.append((params + [state], adam))
    return jobs


def spoil(outs):
    for t in outs:
        t.fill_(-5 if not t.is_floating_point() and t.dtype.itemsize > 1 else 77)


def test_calls_repeat_bit_for_bit_and_follow_their_stream(torch):
    side = torch.cuda.Stream()
    for outs, call in everything(torch):
        call()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for kw in ({}, {"stream": side}):
            spoil(outs)
            torch.cuda.synchronize()
            call(**kw)
            (kw.get("stream") or torch.cuda.current_stream()).synchronize()
            for a, b in zip(outs, want):
                assert torch.equal(a, b)


def test_graph_replays_equal_the_eager_calls(torch):
    for outs, call in everything(torch):
        call()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for replay in range(4):
            spoil(outs)
            torch.ones(1000, device="cuda").sum().item()  # the program's own eager work in between
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(outs, want):
                assert torch.equal(a, b), replay
