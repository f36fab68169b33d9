"""The orthogonalised update against plain implementations in 64 bits (MI355X).

Tolerances come from the arithmetic, before any run, in the Frobenius norm.  U = 2^-24.  A
value held in two fp16 parts is off by 2^-22 = 4 U, a product of such values by two of those
and what the third product leaves out (2^-22), their sum by 16 U of the magnitudes: together
32 U |P| |Q|^T, whose norm is at most 32 U |P| |Q|, |.| being Frobenius norms of the 64-bit
reference.  So a product R = P Q, held again, of operands that are off by dP and dQ is off by

  dR = ||P|| dQ + ||Q|| dP + 32 U |P| |Q| + 4 U |R|,   ||.|| the largest singular value.

Steps may be taken one by one or joined, X = Q X with Q = ... B2 B1 and A' = B (A B) in place of
X X^T of the next X.  An error of X itself at a run's start is moved by the run's map of
singular values t -> f(t), odd, by at most the product of max |f'|.  What X holds below 2^-14
of the largest power of two is off by 2^-39: 2^-39 sqrt(m n) each time X is held.
"""
import math

import pytest

from paper_1911_09287_amd import bltrain
from test_train_ops_gpu import U, half_ulp, near, tdtype, torch  # noqa: F401  (torch: the fixture)

pytestmark = pytest.mark.gpu

USUAL = ((3.4445, -4.7750, 2.0315),) * 5


def error_bound(t, x, coefficients, most):
    """Of the result's Frobenius norm where runs end before the bound of their B's product passes `most`."""
    places = 2.0 ** -39 * math.sqrt(x.numel())
    err, top, k = 6 * U * x.norm().item() + places, 1.0, 0
    eye = t.eye(x.shape[0], dtype=x.dtype, device=x.device)
    while k < len(coefficients):
        gram = x @ x.t()
        size_a, top_a = gram.norm().item(), top ** 2
        da = 36 * U * x.norm().item() ** 2
        q, size_q, top_q, dq, slope, start = None, 0.0, 1.0, 0.0, 1.0, top
        while True:
            a, b, c = coefficients[k]
            s = t.linspace(0, top + 0.01, 2001, dtype=t.float64)
            top_b = (a + b * s ** 2 + c * s ** 4).abs().max().item()
            if q is not None and top_q * top_b > most:
                break
            slope *= (a + 3 * b * s ** 2 + 5 * c * s ** 4).abs().max().item()
            top = (s * (a + b * s ** 2 + c * s ** 4)).abs().max().item()
            poly = a * eye + b * gram + c * gram @ gram
            size_b = poly.norm().item()
            db = abs(b) * da + abs(c) * (2 * top_a * da + 32 * U * size_a ** 2) + 4 * U * size_b
            if q is None:
                q, dq = poly, db
            else:
                new = poly @ q
                dq = top_b * dq + top_q * db + 32 * U * size_b * size_q + 4 * U * new.norm().item()
                q = new
            size_q, top_q = q.norm().item(), top_q * top_b
            ab = poly @ gram
            size_ab, top_ab = ab.norm().item(), top_a * top_b
            dab = top_b * da + top_a * db + 32 * U * size_b * size_a + 4 * U * size_ab
            gram = poly @ ab
            size_a, top_a = gram.norm().item(), top ** 2
            da = top_b * dab + top_ab * db + 32 * U * size_b * size_ab + 4 * U * size_a
            k += 1
            if k == len(coefficients):
                break
        following = q @ x
        err = slope * err + start * dq + 32 * U * size_q * x.norm().item() + 4 * U * following.norm().item() + places
        x = following
    return err


def reference(t, u, eps, coefficients=USUAL):
    """X in 64 bits and the bound of the error in the Frobenius norm."""
    tall = u.shape[0] > u.shape[1]
    x = (u.t() if tall else u).double()
    x = x / (x.norm() + eps)
    err = max(error_bound(t, x, coefficients, most) for most in (0.0, 50.0))
    for a, b, c in coefficients:
        gram = x @ x.t()
        x = a * x + (b * gram + c * gram @ gram) @ x
    return (x.t() if tall else x), err


def gradient(t, shape, seed, few=6):
    g = t.Generator().manual_seed(seed)
    r, c = shape
    k = min(few, r, c)
    return 1e-3 * (0.3 * t.randn(r, c, generator=g)
                   + (t.randn(r, k, generator=g) * t.linspace(1, 0.2, k)) @ t.randn(k, c, generator=g))


def within(got, want, bound, what):
    """The error in the Frobenius norm, and that of a single element (which it bounds)."""
    off = (got.double().cpu() - want.cpu()).norm().item()
    assert off <= bound, (what, off, bound, want.norm().item())


SHAPES = [(1, 1), (1, 7), (9, 1), (3, 3), (5, 40), (64, 27), (33, 65), (128, 128), (127, 129), (130, 100), (50, 128),
          (300, 200), (96, 700), (640, 130), (257, 513), (512, 512)]


@pytest.mark.parametrize("grad", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("param", ["f32", "bf16"])
def test_orthogonalize(torch, param, grad):
    # all shapes in one call
    us = [gradient(torch, s, k).to(tdtype(torch, grad)) for k, s in enumerate(SHAPES)]
    plan = bltrain.MuonPlan(SHAPES, param_dtype=tdtype(torch, param), grad_dtype=tdtype(torch, grad))
    outs = [torch.full(s, float("nan"), dtype=tdtype(torch, param), device="cuda") for s in SHAPES]
    ws = plan.workspace()
    ws.fill_(255)
    plan.orthogonalize(plan.bind(outs, [u.cuda() for u in us]), ws, eps=1e-7)
    for s, u, out in zip(SHAPES, us, outs):
        want, err = reference(torch, u, 1e-7)
        within(out, want, err + half_ulp(param) * (want.norm().item() + err), f"{s} {param} {grad}")


SMALL = [s for s in SHAPES if min(s) <= 64] + [(64, 1024), (1000, 63), (17, 16), (16, 64), (31, 33), (1, 1024), (2, 65)]


@pytest.mark.parametrize("grad", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("param", ["f32", "bf16"])
def test_orthogonalize_small(torch, param, grad):
    # none has sides over 64 and 1024: a block takes a matrix
    us = [gradient(torch, s, 100 + k).to(tdtype(torch, grad)) for k, s in enumerate(SMALL)]
    plan = bltrain.MuonPlan(SMALL, param_dtype=tdtype(torch, param), grad_dtype=tdtype(torch, grad))
    outs = [torch.full(s, float("nan"), dtype=tdtype(torch, param), device="cuda") for s in SMALL]
    ws = plan.workspace()
    ws.fill_(255)
    plan.orthogonalize(plan.bind(outs, [u.cuda() for u in us]), ws, eps=1e-7)
    for s, u, out in zip(SMALL, us, outs):
        want, err = reference(torch, u, 1e-7)
        within(out, want, err + half_ulp(param) * (want.norm().item() + err), f"{s} {param} {grad}")


@pytest.mark.parametrize("shape", [(1024, 1030), (2000, 300), (64, 4097), (700, 1)])
def test_orthogonalize_larger(torch, shape):
    u = gradient(torch, shape, 1)
    plan = bltrain.MuonPlan([shape])
    out = torch.full(shape, float("nan"), device="cuda")
    plan.orthogonalize(plan.bind([out], [u.cuda()]), plan.workspace())
    want, err = reference(torch, u.cuda(), 1e-7)
    within(out, want, err + U * want.norm().item(), shape)


def test_singular_values_come_near_one(torch):
    u = gradient(torch, (200, 333), 2, few=200)
    plan = bltrain.MuonPlan([(200, 333)])
    out = torch.empty(200, 333, device="cuda")
    plan.orthogonalize(plan.bind([out], [u.cuda()]), plan.workspace())
    # every singular value goes through the polynomials, off by no more than the matrix is (Weyl)
    s = torch.linalg.svdvals(u.double()) / u.double().norm()
    start = s.clone()
    for a, b, c in USUAL:
        s = s * (a + b * s ** 2 + c * s ** 4)
    _, err = reference(torch, u, 1e-7)
    got = torch.linalg.svdvals(out.double().cpu())
    near(got, s.sort(descending=True).values, err + U * s.norm().item())
    # and the polynomials take 0.01 ... 1 to 0.67 ... 1.21
    there = s[start > 0.01]
    assert len(there) > 100 and 0.66 < there.min() and there.max() < 1.22


def test_more_matrices_than_a_launch_takes(torch):
    shapes = [(3 + k % 5, 4 + k % 7) for k in range(150)] + [(0, 4), (5, 0)]
    us = [gradient(torch, s, k) if min(s) else torch.empty(s) for k, s in enumerate(shapes)]
    plan = bltrain.MuonPlan(shapes)
    outs = [torch.full(s, float("nan"), device="cuda") for s in shapes]
    ws = plan.workspace()
    ws.fill_(255)
    plan.orthogonalize(plan.bind(outs, [u.cuda() for u in us]), ws)
    for s, u, out in zip(shapes, us, outs):
        if min(s):
            want, err = reference(torch, u, 1e-7)
            within(out, want, err + U * want.norm().item(), s)


def test_other_coefficients(torch):
    steps = ((1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (1.5, -0.5, 0.0))
    u = gradient(torch, (90, 150), 3)
    plan = bltrain.MuonPlan([(90, 150)], coefficients=steps)
    out = torch.empty(90, 150, device="cuda")
    plan.orthogonalize(plan.bind([out], [u.cuda()]), plan.workspace())
    want, err = reference(torch, u, 1e-7, steps)
    within(out, want, err + U * want.norm().item(), "three steps")


@pytest.mark.parametrize("size", [1e-30, 1e-6, 1.0, 1e6, 1e30])
def test_sizes_of_gradients(torch, size):
    # squares far beyond fp32's range; norms far below eps give what the definition gives
    u = gradient(torch, (40, 60), 4).double() * 1e3 * size
    u = u.float()
    plan = bltrain.MuonPlan([(40, 60)])
    out = torch.empty(40, 60, device="cuda")
    plan.orthogonalize(plan.bind([out], [u.cuda()]), plan.workspace(), eps=1e-7)
    want, err = reference(torch, u, 1e-7)
    within(out, want, err + U * want.norm().item(), size)


def test_zeros_and_what_is_not_finite(torch):
    shapes = [(20, 30), (30, 20), (140, 150), (7, 7)]
    us = [torch.zeros(20, 30), gradient(torch, (30, 20), 5), gradient(torch, (140, 150), 6), gradient(torch, (7, 7), 7)]
    us[1][3, 4] = float("nan")
    us[2][139, 0] = float("inf")
    plan = bltrain.MuonPlan(shapes)
    outs = [torch.full(s, 5.0, device="cuda") for s in shapes]
    plan.orthogonalize(plan.bind(outs, [u.cuda() for u in us]), plan.workspace())
    assert (outs[0] == 0).all() and outs[1].isnan().all() and outs[2].isnan().all() and outs[3].isfinite().all()


def step_reference(t, p, g, m, shapes, starts, a, decay, scales, gs):
    new_p, new_m, err = [], [], []
    for k, (s, at) in enumerate(zip(shapes, starts)):
        gk = gs * g[k].double()
        mk = a["momentum"] * m[at:at + s[0] * s[1]].double().view(s) + gk
        u = gk + a["momentum"] * mk if a["nesterov"] else mk
        x, e = reference(t, u, a["eps"])
        # u itself is rounded twice: the same error relative to its norm, moved by all steps
        e += 4 * U * 4.0 ** 5
        scale = scales[k] if scales else math.sqrt(max(1.0, s[0] / s[1]))
        keep = 1.0 - a["lr"] * a["weight_decay"] * (decay is None or decay[k])
        new_p.append(p[k].double() * keep - a["lr"] * scale * x)
        new_m.append(mk)
        err.append(a["lr"] * scale * (e + 3 * U * x.norm().item()) + 4 * U * p[k].double().norm().item())
    return new_p, new_m, err


@pytest.mark.parametrize("small", [False, True])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("param,grad", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f16")])
def test_step(torch, param, grad, nesterov, small):
    shapes = [(1, 1), (64, 27), (130, 140), (5, 300), (300, 90), (128, 256)]
    if small:
        shapes = [(1, 1), (64, 27), (63, 64), (5, 300), (300, 9), (32, 256)]
    decay, scales = [True, False, True, True, False, True], None if nesterov else [1.0, 0.5, 2.0, 0.0, 1.5, 0.1]
    a = {"lr": 0.02, "momentum": 0.95, "eps": 1e-7, "weight_decay": 0.1, "nesterov": nesterov}
    plan = bltrain.MuonPlan(shapes, param_dtype=tdtype(torch, param), grad_dtype=tdtype(torch, grad), decay=decay,
                            scales=scales)
    gen = torch.Generator().manual_seed(8)
    p = [(0.05 * torch.randn(s, generator=gen)).to(tdtype(torch, param)) for s in shapes]
    dev = [v.cuda() for v in p]
    state, ws = plan.state(), plan.workspace()
    gs = torch.full((1,), 0.75, device="cuda")
    m = torch.zeros(plan.total)
    for step in (1, 2, 3):
        g = [gradient(torch, s, 10 * step + k).to(tdtype(torch, grad)) for k, s in enumerate(shapes)]
        before = [v.cpu() for v in dev]
        m = plan.momentum(state).cpu()
        ws.fill_(255)
        plan.step(plan.bind(dev, [v.cuda() for v in g]), state, ws, step=step, seed=3, grad_scale=gs, **a)
        want_p, want_m, err = step_reference(torch, before, g, m, shapes, plan.starts, a, decay, scales, 0.75)
        got_m = plan.momentum(state).cpu()
        inside = torch.zeros(plan.total, dtype=torch.bool)
        for k, (s, at) in enumerate(zip(shapes, plan.starts)):
            n = s[0] * s[1]
            inside[at:at + n] = True
            near(got_m[at:at + n].view(s), want_m[k], 3 * U * (want_m[k].abs() + (0.75 * g[k].double()).abs()) + 1e-30)
            # bfloat16 parameters are rounded up or down by chance: a whole ulp
            rounding = 0.0 if param == "f32" else 2.0 ** -7 * (want_p[k].norm().item() + err[k])
            within(dev[k], want_p[k], err[k] + rounding, (s, step, param, grad))
        assert (got_m[~inside] == 0).all()


def test_rounding_of_bfloat16_parameters_is_right_on_average(torch):
    # one product step of a constant 1 x n matrix: every element moves by the same small amount
    n = 1 << 16
    plan = bltrain.MuonPlan([(1, n)], param_dtype=torch.bfloat16)
    p, g = torch.ones(1, n, dtype=torch.bfloat16, device="cuda"), torch.ones(1, n, device="cuda")
    state, ws, tensors = plan.state(), plan.workspace(), None
    tensors = plan.bind([p], [g])
    x, _ = reference(torch, g.cpu(), 1e-7)
    lr = 2.0 ** -10 / x[0, 0].item()  # a move of 2^-10: a quarter of the step of 2^-8 below 1
    plan.step(tensors, state, ws, lr=lr, weight_decay=0.0, step=1, seed=5)
    values, counts = p.float().unique(return_counts=True)
    assert values.tolist() == [1.0 - 2.0 ** -8, 1.0]
    # a binomial share of 1/4 over 65536: six standard deviations are 0.0102
    assert abs(counts[0].item() / n - 0.25) < 0.0102
    again = torch.ones_like(p)
    state.zero_()
    plan.step(plan.bind([again], [g]), state, ws, lr=lr, weight_decay=0.0, step=1, seed=5)
    assert (again == p).all()
    state.zero_()
    again.fill_(1.0)
    plan.step(plan.bind([again], [g]), state, ws, lr=lr, weight_decay=0.0, step=1, seed=6)
    assert (again != p).any()


@pytest.mark.parametrize("shapes", [[(70, 30), (128, 200), (3, 3)], [(70, 30), (3, 3)]])
@pytest.mark.parametrize("param", ["f32", "bf16"])
def test_live_rate_and_step_and_a_graph(torch, param, shapes):
    plan = bltrain.MuonPlan(shapes, param_dtype=tdtype(torch, param))
    gen = torch.Generator().manual_seed(9)
    start = [(0.05 * torch.randn(s, generator=gen)).to(tdtype(torch, param)).cuda() for s in shapes]
    grads = [gradient(torch, s, k).cuda() for k, s in enumerate(shapes)]
    ws = plan.workspace()

    def eager(steps):
        p, state = [v.clone() for v in start], plan.state()
        bound = plan.bind(p, grads)
        for k in range(1, steps + 1):
            plan.step(bound, state, ws, lr=0.01 * k, step=k, seed=2, weight_decay=0.01)
        return p, plan.momentum(state).clone()
    p, state = [v.clone() for v in start], plan.state()
    bound, live = plan.bind(p, grads), torch.zeros(2, dtype=torch.float64, device="cuda")
    live.copy_(torch.tensor([0.01, 1.0], dtype=torch.float64))
    plan.step(bound, state, ws, live=live, seed=2, weight_decay=0.01)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.step(bound, state, ws, live=live, seed=2, weight_decay=0.01)
    for k in range(2, 6):
        live.copy_(torch.tensor([0.01 * k, float(k)], dtype=torch.float64))
        ws.fill_(255)
        graph.replay()
        want_p, want_m = eager(k)
        torch.cuda.synchronize()
        assert (plan.momentum(state) == want_m).all()
        for v, w in zip(p, want_p):
            assert (v == w).all()


def test_in_place_and_with_empty_lists(torch):
    u = gradient(torch, (60, 90), 10).cuda()
    plan = bltrain.MuonPlan([(60, 90)])
    ws, out = plan.workspace(), torch.empty(60, 90, device="cuda")
    plan.orthogonalize(plan.bind([out], [u]), ws)
    plan.orthogonalize(plan.bind([u], [u]), ws)
    assert (u == out).all()
    for shapes in ([], [(0, 5)]):
        plan = bltrain.MuonPlan(shapes)
        empty = [torch.empty(s, device="cuda") for s in shapes]
        plan.orthogonalize(plan.bind(empty, empty), plan.workspace())
        plan.step(plan.bind(empty, empty), plan.state(), plan.workspace())
