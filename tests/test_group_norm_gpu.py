"""Group norm with an activation against plain implementations in 64 bits (MI355X).

Tolerances come from the arithmetic, before any run, as in test_train_ops_gpu: U = 2^-24
is half an ulp of fp32, a sum of n fp32 terms is off by at most 16 U times the sum of their
magnitudes, a result of 16 bits adds half an ulp of its type.  Outputs are filled with NaN
before a call, so that an element that is not written fails.
"""
import math

import pytest

from paper_1911_09287_amd import bltrain
from test_train_ops_gpu import U, half_ulp, near, tdtype, torch  # noqa: F401  (torch: the fixture)

pytestmark = pytest.mark.gpu


def spread(t, groups, channels, last):
    """[batch][groups] at every channel of [batch][sites][channels] or [batch][channels][sites]."""
    t = t.repeat_interleave(channels // groups, 1)
    return t[:, None, :] if last else t[:, :, None]


def group_mean(t, groups, last):
    batch = t.shape[0]
    t = t.transpose(1, 2) if last else t
    return t.reshape(batch, groups, -1).mean(2)


def reference(t, x, w, b, dy, groups, last, act, eps):
    """y, mean, rstd, dx, dw, db in 64 bits."""
    channels = x.shape[2] if last else x.shape[1]

    def at(v):
        return spread(v, groups, channels, last)
    mean = group_mean(x, groups, last)
    rstd = (group_mean((x - at(mean)).square(), groups, last) + eps).rsqrt()
    h = (x - at(mean)) * at(rstd)
    wv, bv = (v[None, None, :] if last else v[None, :, None] for v in (w, b))
    z = h * wv + bv
    q = t.sigmoid(z)
    y = {None: z, "relu": z.clamp(min=0), "silu": z * q}[act]
    slope = {None: t.ones_like(z), "relu": (z > 0).double(), "silu": q + z * q * (1 - q)}[act]
    dz = dy * slope
    u = dz * wv
    c1, c2 = group_mean(u, groups, last), group_mean(u * h, groups, last)
    over = (0, 1) if last else (0, 2)
    return {"y": y, "mean": mean, "rstd": rstd, "dx": at(rstd) * (u - at(c1) - h * at(c2)), "dw": (dz * h).sum(over),
            "db": dz.sum(over), "h": h, "z": z, "dz": dz, "wv": wv, "bv": bv, "over": over}


def bounds(x, dy, r, groups, last, act, dtype, wdtype):
    channels = x.shape[2] if last else x.shape[1]

    def at(v):
        return spread(v, groups, channels, last)

    def most(v):
        v = v.transpose(1, 2) if last else v
        return v.reshape(v.shape[0], groups, -1).amax(2)
    # as for layer norm: the mean is off by 16 U of the largest value, rstd by 24 U and by
    # what the mean's error makes of it, h by both
    dmean = 16 * U * most(x.abs())
    drel = 24 * U + dmean * r["rstd"]
    dh = at(dmean * r["rstd"]) + r["h"].abs() * at(drel) + 2 * U * r["h"].abs()
    wv, bv = r["wv"].abs(), r["bv"].abs()
    tiny = 2.0 ** -25 if dtype == "f16" else 1e-30
    t = half_ulp(dtype)
    dz_of_z = dh * wv + 3 * U * (r["h"].abs() * wv + bv)  # z's error
    # |act'| <= 1.1; the logistic is off by an ulp of exp (2 U), of a division and a sum
    got = {"mean": dmean + 1e-30, "rstd": r["rstd"] * drel}
    got["y"] = 1.1 * dz_of_z + 8 * U * r["z"].abs() + t * r["y"].abs() + tiny
    # |act''| <= 0.5; where a ReLU's argument may lie on either side of 0 its slope may be either
    ddz = dy.abs() * (0.5 * dz_of_z + 12 * U * (1 + r["z"].abs())) if act == "silu" else dy.abs() * 2 * U
    if act == "relu":
        ddz = ddz + dy.abs() * (r["z"].abs() <= dz_of_z)
    au = (r["dz"].abs() + ddz) * wv
    du = ddz * wv + U * au
    mean = lambda v: group_mean(v, groups, last)  # noqa: E731
    d1 = 20 * U * mean(au) + mean(du)
    d2 = 20 * U * mean(au * r["h"].abs()) + mean(du * r["h"].abs() + au * dh)
    c1, c2 = mean(au), mean(au * r["h"].abs())
    parts = au + at(c1) + r["h"].abs() * at(c2)
    got["dx"] = at(r["rstd"]) * (du + at(d1) + r["h"].abs() * at(d2) + dh * at(c2) + 6 * U * parts) \
        + at(r["rstd"] * drel) * parts + t * r["dx"].abs() + tiny
    tw = half_ulp(wdtype)
    small = 2.0 ** -25 if wdtype == "f16" else 1e-30
    adz = r["dz"].abs() + ddz
    got["dw"] = (18 * U * adz * r["h"].abs() + ddz * r["h"].abs() + adz * dh).sum(r["over"]) + tw * r["dw"].abs() + small
    got["db"] = (18 * U * adz + ddz).sum(r["over"]) + tw * r["db"].abs() + small
    return got


def inputs(t, shape, last, dtype, wdtype, seed, offset=0.5):
    batch, sites, channels, _ = shape
    g = t.Generator().manual_seed(seed)
    size = (batch, sites, channels) if last else (batch, channels, sites)
    x = (t.randn(size, generator=g) * 1.5 + offset).to(tdtype(t, dtype))
    dy = t.randn(size, generator=g).to(tdtype(t, dtype))
    w = (1 + 0.3 * t.randn(channels, generator=g)).to(tdtype(t, wdtype))
    b = (0.3 * t.randn(channels, generator=g)).to(tdtype(t, wdtype))
    return x, dy, w, b


def run(t, shape, last, act, x, dy, w, b, dtype, wdtype, eps, gaps=(0, 0), shift=0, weights=True, grads=True):
    """The plan's results, on tensors whose samples lie `gaps` elements further apart and start `shift` elements in."""
    batch, sites, channels, groups = shape
    flat, dt = sites * channels, tdtype(t, dtype)
    plan = bltrain.GroupNormPlan(batch, sites, channels, groups, channels_last=last, act=act, dtype=dt,
                                 wdtype=tdtype(t, wdtype), eps=eps, x_stride=flat + gaps[0], y_stride=flat + gaps[1])

    def place(v, gap):
        room = t.full((batch * (flat + gap) + shift,), float("nan"), dtype=dt, device="cuda")
        view = room[shift:].view(batch, flat + gap)[:, :flat]
        if v is not None:
            view.copy_(v.reshape(batch, flat))
        return room, view

    (_, xs), (_, ds) = place(x, gaps[0]), place(dy, gaps[1])
    (yr, y), (xr, dx) = place(None, gaps[1]), place(None, gaps[0])
    ws = plan.workspace()
    ws.fill_(255)
    wd, bd = (w.cuda(), b.cuda()) if weights else (None, None)
    stats = t.full(plan.stats_shape(), float("nan"), device="cuda")
    dw, db = (t.full((channels,), float("nan"), dtype=tdtype(t, wdtype), device="cuda") if grads else None
              for _ in range(2))
    plan.forward(xs, wd, bd, y, stats, ws)
    ws.fill_(255)
    plan.backward(ds, xs, wd, bd, stats, dx, dw, db, ws)
    t.cuda.synchronize()
    for room, gap in ((yr, gaps[1]), (xr, gaps[0])):  # nothing but the samples is written
        assert room[:shift].isnan().all() and room[shift:].view(batch, flat + gap)[:, flat:].isnan().all()
    got = {"y": y.reshape(x.shape), "mean": stats[0], "rstd": stats[1], "dx": dx.reshape(x.shape)}
    return dict(got, dw=dw, db=db) if grads else got


def check(t, shape, last, act, dtype, wdtype, seed, eps=1e-5, offset=0.5, **kw):
    x, dy, w, b = inputs(t, shape, last, dtype, wdtype, seed, offset)
    got = run(t, shape, last, act, x, dy, w, b, dtype, wdtype, eps, **kw)
    if not kw.get("weights", True):
        w, b = t.ones_like(w), t.zeros_like(b)
    x, dy, w, b = (v.double() for v in (x, dy, w, b))
    r = reference(t, x, w, b, dy, shape[3], last, act, eps)
    most = bounds(x, dy, r, shape[3], last, act, dtype, wdtype)
    for name, v in got.items():
        near(v, r[name], most[name], f"{name} {shape} {'last' if last else 'first'} {act} {dtype}")


# (batch, sites, channels, groups)
LAST = [(1, 4, 1, 1), (2, 4, 6, 3), (3, 7, 5, 5), (2, 1, 64, 8), (1, 65, 33, 11), (2, 300, 50, 10), (3, 9, 257, 1),
        (1, 20, 2056, 8), (2, 11, 1030, 2), (1, 5000, 8, 2), (40, 128, 64, 32), (1, 40001, 1, 1), (2, 2500, 3, 1),
        (5, 31, 110, 55), (2, 3136, 64, 32), (1, 513, 1024, 4)]
FIRST = [(1, 4, 1, 1), (2, 3, 6, 3), (3, 7, 5, 5), (2, 1, 64, 8), (1, 65, 33, 11), (2, 300, 50, 10), (3, 49, 64, 4),
         (1, 513, 20, 2), (4, 1250, 16, 4), (1, 40001, 2, 1), (2, 20000, 3, 1), (300, 5, 24, 8), (2, 64, 256, 16),
         (1, 255, 9, 3), (2, 257, 9, 9), (1, 2, 1500, 5)]


@pytest.mark.parametrize("act", [None, "relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", LAST)
def test_channels_last(torch, shape, dtype, act):
    check(torch, shape, True, act, dtype, "f32", seed=sum(shape))


@pytest.mark.parametrize("act", [None, "relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", FIRST)
def test_channels_first(torch, shape, dtype, act):
    check(torch, shape, False, act, dtype, "f32", seed=sum(shape))


@pytest.mark.parametrize("last", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_strides_shifts_weights(torch, dtype, last):
    for shape in ((3, 37, 30, 5), (2, 700, 8, 2)):
        check(torch, shape, last, "silu", dtype, dtype, 1, gaps=(5, 0), shift=1)
        check(torch, shape, last, "silu", dtype, "f32", 2, gaps=(0, 7), shift=3)
        check(torch, shape, last, "relu", dtype, "f32", 3, gaps=(8, 40), weights=False)
        check(torch, shape, last, None, dtype, "f32", 4, grads=False)


@pytest.mark.parametrize("last", [True, False])
def test_means_far_from_zero(torch, last):
    # a variance that is 10^-4 of the squared mean
    for shape in ((2, 1000, 12, 3), (1, 30000, 4, 1)):
        check(torch, shape, last, "silu", "f32", "f32", 5, offset=100.0)


@pytest.mark.parametrize("last", [True, False])
def test_groups_of_one_value_have_no_gradient(torch, last):
    shape = (3, 1, 40, 40)
    x, dy, w, b = inputs(torch, shape, last, "f32", "f32", 6)
    got = run(torch, shape, last, "silu", x, dy, w, b, "f32", "f32", 1e-5)
    assert (got["dx"] == 0).all() and (got["dw"] == 0).all()
    z = b.double().expand(3, 40)
    near(got["y"].reshape(3, 40), z * z.sigmoid(), 16 * U * (1 + z.abs()))


@pytest.mark.parametrize("last", [True, False])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_finite_stays_in_its_group(torch, last, bad):
    shape = (3, 50, 12, 4)
    x, dy, w, b = inputs(torch, shape, last, "f32", "f32", 7)
    clean = run(torch, shape, last, "silu", x, dy, w, b, "f32", "f32", 1e-5)
    x[(1, 20, 4) if last else (1, 4, 20)] = bad  # sample 1, group 1
    got = run(torch, shape, last, "silu", x, dy, w, b, "f32", "f32", 1e-5)
    for name in ("y", "dx"):
        a, c = (v.transpose(1, 2) if last else v for v in (got[name], clean[name]))
        hit = torch.zeros(3, 12, dtype=torch.bool)
        hit[1, 3:6] = True
        assert a[hit].isnan().all()
        assert (a[~hit] == c[~hit]).all()


def test_huge_values(torch):
    # squares beyond fp16's range, means beyond it: statistics are held in fp32
    shape = (2, 400, 8, 2)
    x, dy, w, b = inputs(torch, shape, True, "f16", "f32", 8)
    x = (x * 10000).clamp(-60000, 60000)
    got = run(torch, shape, True, "silu", x, dy, w, b, "f16", "f32", 1e-5)
    r = reference(torch, x.double(), w.double(), b.double(), dy.double(), 2, True, "silu", 1e-5)
    most = bounds(x.double(), dy.double(), r, 2, True, "silu", "f16", "f32")
    for name, v in got.items():
        near(v, r[name], most[name], name)


@pytest.mark.parametrize("last", [True, False])
def test_in_place_and_without_statistics(torch, last):
    shape = (3, 100, 24, 4)
    x, dy, w, b = (v.cuda() for v in inputs(torch, shape, last, "bf16", "f32", 9))
    plan = bltrain.GroupNormPlan(*shape, channels_last=last, act="silu", dtype=torch.bfloat16)
    ws, stats = plan.workspace(), torch.empty(plan.stats_shape(), device="cuda")
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    plan.forward(x, w, b, y, stats, ws)
    plan.backward(dy, x, w, b, stats, dx, dw, db, ws)
    again = torch.empty_like(y)
    plan.forward(x, w, b, again, None, ws)
    assert (again == y).all()
    over = dy.clone()
    plan.backward(over, x, w, b, stats, over, None, db, ws)
    assert (over == dx).all()
    over = x.clone()
    plan.backward(dy, over, w, b, stats, over, dw, None, ws)
    assert (over == dx).all()
    over = x.clone()
    plan.forward(over, w, b, over, None, ws)
    assert (over == y).all()


def test_no_samples(torch):
    plan = bltrain.GroupNormPlan(0, 5, 8, 2, act="silu")
    e, w = torch.empty(0, 8, 5, device="cuda"), torch.ones(8, device="cuda")
    stats, dw, db = torch.empty(2, 0, 2, device="cuda"), torch.ones(8, device="cuda"), torch.ones(8, device="cuda")
    plan.forward(e, w, w, e, stats, None)
    plan.backward(e, e, w, w, stats, e, dw, db, None)
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("last", [True, False])
def test_same_bits_each_time_and_in_a_graph(torch, last):
    shape = (4, 600, 48, 8)
    x, dy, w, b = (v.cuda() for v in inputs(torch, shape, last, "f32", "f32", 10))
    plan = bltrain.GroupNormPlan(*shape, channels_last=last, act="silu")
    ws, stats = plan.workspace(), torch.empty(plan.stats_shape(), device="cuda")
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)

    def both():
        plan.forward(x, w, b, y, stats, ws)
        plan.backward(dy, x, w, b, stats, dx, dw, db, ws)
    both()
    want = [v.clone() for v in (y, stats, dx, dw, db)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        for v in (y, stats, dx, dw, db):
            v.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for v, e in zip((y, stats, dx, dw, db), want):
            assert (v == e).all()
        both()


def test_the_reference_against_differences():
    """The formulas' gradients against central differences in 64 bits (the host)."""
    import torch as t
    t.manual_seed(0)
    for last in (True, False):
        for act in (None, "relu", "silu"):
            x = t.randn((2, 5, 6) if last else (2, 6, 5), dtype=t.float64)
            w, b, dy = 1 + 0.3 * t.randn(6, dtype=t.float64), t.randn(6, dtype=t.float64), t.randn_like(x)
            r = reference(t, x, w, b, dy, 3, last, act, 1e-3)
            for name, v in (("dx", x), ("dw", w), ("db", b)):
                way, step = t.randn_like(v), 1e-6
                ends = []
                for s in (step, -step):
                    v.add_(way, alpha=s)
                    ends.append((reference(t, x, w, b, dy, 3, last, act, 1e-3)["y"] * dy).sum())
                    v.add_(way, alpha=-s)
                # (truncation step^2 times a third derivative of some hundreds, rounding 2^-52 / step)
                assert abs((ends[0] - ends[1]) / (2 * step) - (r[name] * way).sum()) < 1e-6, (last, act, name)
    assert math.isfinite(U)
