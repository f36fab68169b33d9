"""The gated linear recurrence against plain implementations in 64 bits (MI355X).

Tolerances come from the arithmetic, before any run.  U = 2^-24 is half an ulp of fp32,
relative.  h is a sum of b_s times the product of the a behind it; a is off by at most 6 U
relative (an ulp of exp, a sum, a division, a product) and each product rounds once or twice,
so that a term is off by 8 U for every factor, and by 32 U for its sums over steps, lanes,
waves and chunks.  With M_t = a M_(t-1) + |b| the sum of magnitudes, the error e_t = a e_(t-1)
+ 8 U a M_(t-1) + 32 U |b| is a bound in whatever order stretches are joined.  A result of 16
bits adds half an ulp of its type.
"""
import pytest

from paper_1911_09287_amd import bltrain
from test_train_ops_gpu import U, half_ulp, near, tdtype, torch  # noqa: F401  (torch: the fixture)

pytestmark = pytest.mark.gpu


def reference(t, gate, x, h0, dy, dlast, resets, kind):
    """h, dgate, dx, dh0 in 64 bits, step by step, and bounds on their errors without the results' roundings."""
    a = gate.sigmoid() if kind == "sigmoid" else gate.exp()
    rest = (-gate).sigmoid() if kind == "sigmoid" else t.ones_like(a)
    b = rest * x
    length = x.shape[1]
    drop = t.zeros(x.shape[:2], dtype=t.bool) if resets is None else resets.bool()
    h, m, e = h0.clone(), h0.abs(), t.zeros_like(h0)
    hs, before, before_m, before_e, errs = [], [], [], [], []
    for s in range(length):
        d = drop[:, s, None]
        zero = t.zeros_like(h)
        h, m, e = t.where(d, zero, h), t.where(d, zero, m), t.where(d, zero, e)
        before.append(h)
        before_m.append(m)
        before_e.append(e)
        e = a[:, s] * e + 8 * U * a[:, s] * m + 32 * U * b[:, s].abs()
        h, m = t.where(d, b[:, s], a[:, s] * h + b[:, s]), a[:, s] * m + b[:, s].abs()
        e = t.where(d, 32 * U * b[:, s].abs(), e)
        m = t.where(d, b[:, s].abs(), m)
        hs.append(h)
        errs.append(e)
    got = {"y": t.stack(hs, 1) if hs else x.clone(), "last": h}
    most = {"y": t.stack(errs, 1) if errs else x.clone(), "last": e + 1e-30}
    back, size, err = dlast.clone(), dlast.abs(), t.zeros_like(dlast)
    dgate, dx, eg, ex = (t.zeros_like(x) for _ in range(4))
    for s in reversed(range(length)):
        dh, dm, de = back + dy[:, s], size + dy[:, s].abs(), err + 32 * U * dy[:, s].abs() + 2 * U * size
        if kind == "sigmoid":
            slope, diff = a[:, s] * rest[:, s], before[s] - x[:, s]
            dgate[:, s], dx[:, s] = dh * slope * diff, dh * rest[:, s]
            eg[:, s] = slope * (de * diff.abs() + dm * (before_e[s] + 20 * U * (before_m[s] + x[:, s].abs())))
            ex[:, s] = rest[:, s] * (de + 8 * U * dm)
        else:
            dgate[:, s], dx[:, s] = dh * a[:, s] * before[s], dh
            eg[:, s] = a[:, s] * (de * before[s].abs() + dm * (before_e[s] + 8 * U * before_m[s]))
            ex[:, s] = de
        zero, d = t.zeros_like(dh), drop[:, s, None]
        back = t.where(d, zero, a[:, s] * dh)
        size = t.where(d, zero, a[:, s] * dm)
        err = t.where(d, zero, a[:, s] * (de + 8 * U * dm))
    got.update(dgate=dgate, dx=dx, dh0=back)
    most.update(dgate=eg, dx=ex, dh0=err + 1e-30)
    return got, most


def inputs(t, shape, kind, dtype, seed, resets):
    g = t.Generator().manual_seed(seed)
    outer, length, inner = shape
    gate = t.randn(shape, generator=g)
    gate = gate * 1.5 + 1.5 if kind == "sigmoid" else -(0.7 * gate - 2.5).exp()
    drop = None
    if resets:
        drop = t.rand(outer, length, generator=g) < min(0.5, 3.0 / max(length, 1))
        drop[0, :1] = True
    return {"gate": gate.to(tdtype(t, dtype)), "x": t.randn(shape, generator=g).to(tdtype(t, dtype)),
            "h0": t.randn(outer, inner, generator=g), "dy": t.randn(shape, generator=g).to(tdtype(t, dtype)),
            "dlast": t.randn(outer, inner, generator=g), "resets": drop}


def run(t, shape, kind, dtype, v, place=None, strides=((0, 0), (0, 0)), states_of=None):
    """The plan's results.  place(values or None, which): a tensor of the plan's layout, which in "in", "out"."""
    plan = bltrain.RecurrencePlan(*shape, gate=kind, dtype=tdtype(t, dtype), in_strides=strides[0], out_strides=strides[1])

    def dense(values, which):
        if values is not None:
            return values.cuda()
        return t.full(shape, float("nan"), dtype=tdtype(t, dtype), device="cuda")
    place = place or dense
    ws = plan.workspace()
    ws.fill_(255)
    gate, x, dy = place(v["gate"], "in"), place(v["x"], "in"), place(v["dy"], "out")
    y, dgate, dx = place(None, "out"), place(None, "in"), place(None, "in")
    h0, dlast = (None if v[k] is None else v[k].cuda() for k in ("h0", "dlast"))
    resets = None if v["resets"] is None else v["resets"].cuda()
    last, dh0 = (t.full((shape[0], shape[2]), float("nan"), device="cuda") for _ in range(2))
    states = plan.states().fill_(float("nan"))
    plan.forward(gate, x, y, ws, h0=h0, last=last, resets=resets, states=states)
    ws.fill_(255)
    plan.backward(gate, x, dy, states, dgate, dx, ws, dlast=dlast, dh0=dh0, resets=resets)
    t.cuda.synchronize()
    return {"y": y, "last": last, "dgate": dgate, "dx": dx, "dh0": dh0}


def check(t, shape, kind, dtype, seed, resets, **kw):
    v = inputs(t, shape, kind, dtype, seed, resets)
    got = run(t, shape, kind, dtype, v, **kw)
    r, most = reference(t, *(v[k].double() for k in ("gate", "x", "h0", "dy", "dlast")), v["resets"], kind)
    tiny = 2.0 ** -25 if dtype == "f16" else 1e-30
    for name in got:
        bound = most[name]
        if name in ("y", "dgate", "dx"):
            bound = bound + half_ulp(dtype) * (r[name].abs() + bound) + tiny
        near(got[name], r[name], bound, f"{name} {shape} {kind} {dtype} resets {resets}")


SHAPES = [(1, 1, 1), (3, 1, 5), (2, 7, 3), (2, 8, 70), (2, 9, 1), (5, 16, 70), (3, 17, 64), (2, 100, 33), (4, 257, 130),
          (1, 1000, 4), (2, 1029, 2), (3, 300, 1), (2100, 70, 1), (1, 5000, 40), (1, 20000, 1), (1, 9000, 3),
          (2, 2500, 32), (600, 33, 17), (1, 4097, 256), (2, 200, 65), (3, 150, 66), (300, 20, 67)]


@pytest.mark.parametrize("resets", [False, True])
@pytest.mark.parametrize("kind", ["sigmoid", "exp"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_steps(torch, shape, dtype, kind, resets):
    check(torch, shape, kind, dtype, sum(shape), resets)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_halves_of_one_tensor(torch, dtype):
    for shape in ((2, 40, 33), (3, 1500, 16), (2, 300, 3)):
        outer, length, inner = shape

        def place(values, which):
            if which == "out":
                return values.cuda() if values is not None else torch.full(shape, float("nan"), dtype=tdtype(torch, dtype), device="cuda")
            both = torch.full((outer, length, 2 * inner + 1), float("nan"), dtype=tdtype(torch, dtype), device="cuda")
            half = both[..., inner + 1:]
            if values is not None:
                half.copy_(values)
            return half
        check(torch, shape, "sigmoid", dtype, 3, True, place=place,
              strides=((length * (2 * inner + 1), 2 * inner + 1), (0, 0)))


@pytest.mark.parametrize("shape", [(5, 600, 7), (4, 70, 1), (3, 30, 1), (9, 2100, 40)])
def test_steps_outermost(torch, shape):
    # [length][outer][inner], as networks keep it that go through time in the outer loop
    outer, length, inner = shape

    def place(values, which):
        room = torch.full((length, outer, inner), float("nan"), device="cuda")
        view = room.transpose(0, 1)
        if values is not None:
            view.copy_(values)
        return view
    strides = (inner, outer * inner)
    check(torch, shape, "exp", "f32", 4, True, place=place, strides=(strides, strides))


def test_rows_further_apart_and_shifted(torch):
    for shape, dtype in (((6, 333, 1), "f32"), ((6, 333, 1), "bf16"), ((2100, 65, 1), "f16"), ((2, 30000, 1), "bf16")):
        outer, length, _ = shape

        def place(values, which):
            room = torch.full((outer * (length + 3) + 1,), float("nan"), dtype=tdtype(torch, dtype), device="cuda")
            view = room[1:].view(outer, length + 3)[:, :length].unsqueeze(2)
            if values is not None:
                view.copy_(values)
            return view
        check(torch, shape, "sigmoid", dtype, 5, True, place=place, strides=((length + 3, 1), (length + 3, 1)))


@pytest.mark.parametrize("shape", [(2, 300, 20), (2, 300, 1), (2, 300, 3), (1, 6000, 20), (1, 40000, 1)])
@pytest.mark.parametrize("kind", ["sigmoid", "exp"])
def test_what_lies_before_a_reset_or_behind_the_end_does_not_count(torch, shape, kind):
    outer, length, inner = shape
    v = inputs(torch, shape, kind, "f32", 6, False)
    drop = torch.zeros(outer, length, dtype=torch.bool)
    cut, end = length // 3, length - length // 5
    drop[:, cut] = drop[:, end] = True  # (the second one ends the sequence)
    v["resets"] = drop
    v["dy"][:, end:] = 0
    v["dlast"] = None
    clean = run(torch, shape, kind, "f32", v)
    for bad in (float("nan"), float("inf"), -3e38):
        w = {k: None if x is None else x.clone() for k, x in v.items()}
        w["x"][:, cut - 1] = bad  # the state before the reset
        w["h0"][:] = bad
        w["x"][:, end:] = bad
        w["gate"][:, end:] = bad if bad != 3e38 else float("nan")
        got = run(torch, shape, kind, "f32", w)
        assert (got["y"][:, cut:end] == clean["y"][:, cut:end]).all()
        for name in ("dgate", "dx"):
            assert (got[name][:, cut:end] == clean[name][:, cut:end]).all(), (name, bad)


def test_gates_at_the_ends_of_their_range(torch):
    shape = (1, 40, 8)
    v = inputs(torch, shape, "sigmoid", "f32", 7, False)
    for at, g in ((3, 1e4), (5, -1e4), (9, float("inf")), (11, -float("inf")), (13, -3.4e38), (15, 3.4e38)):
        v["gate"][:, at] = g
    got = run(torch, shape, "sigmoid", "f32", v)
    r, most = reference(torch, *(v[k].double() for k in ("gate", "x", "h0", "dy", "dlast")), None, "sigmoid")
    for name in got:
        near(got[name], r[name], most[name] + 1e-30, name)
    v = inputs(torch, shape, "exp", "f32", 7, False)
    v["gate"][:, 5], v["gate"][:, 9], v["gate"][:, 11] = -float("inf"), -3.4e38, 0.0
    got = run(torch, shape, "exp", "f32", v)
    r, most = reference(torch, *(v[k].double() for k in ("gate", "x", "h0", "dy", "dlast")), None, "exp")
    for name in got:
        near(got[name], r[name], most[name] + 1e-30, name)


@pytest.mark.parametrize("kind", ["sigmoid", "exp"])
def test_token_by_token_and_in_parts(torch, kind):
    # the state of one call is the next one's, in its place
    shape = (3, 50, 20)
    v = inputs(torch, shape, kind, "bf16", 8, False)
    r, most = reference(torch, *(v[k].double() for k in ("gate", "x", "h0", "dy", "dlast")), None, kind)
    gate, x = v["gate"].cuda(), v["x"].cuda()
    for cuts in (range(51), (0, 1, 9, 30, 50)):
        state, ys = v["h0"].cuda(), []
        cuts = list(cuts)
        for lo, hi in zip(cuts, cuts[1:]):
            plan = bltrain.RecurrencePlan(3, hi - lo, 20, gate=kind, dtype=torch.bfloat16)
            y = torch.full((3, hi - lo, 20), float("nan"), dtype=torch.bfloat16, device="cuda")
            plan.forward(gate[:, lo:hi].contiguous(), x[:, lo:hi].contiguous(), y, plan.workspace(), h0=state, last=state)
            ys.append(y)
        near(torch.cat(ys, 1), r["y"], most["y"] + half_ulp("bf16") * (r["y"].abs() + most["y"]) + 1e-30)
        near(state, r["last"], most["last"])


# (channels one to three over those of a whole number of blocks among them: no two blocks may share one)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 900, 24), (1, 6000, 24), (3, 700, 1), (2, 900, 33), (2, 900, 65), (40, 300, 66),
                                   (40, 300, 67), (1, 9000, 129), (300, 40, 65), (300, 6, 65)])
def test_in_place(torch, shape, dtype):
    v = inputs(torch, shape, "sigmoid", dtype, 9, True)
    want = run(torch, shape, "sigmoid", dtype, v)
    plan = bltrain.RecurrencePlan(*shape, dtype=tdtype(torch, dtype))
    ws, states = plan.workspace(), plan.states()
    gate, x, dy, resets = (v[k].cuda() for k in ("gate", "x", "dy", "resets"))
    state, y = v["h0"].cuda(), x.clone()
    plan.forward(gate, y, y, ws, h0=state, last=state, resets=resets, states=states)
    assert (y == want["y"]).all() and (state == want["last"]).all()
    back = v["dlast"].cuda()
    g2, x2 = gate.clone(), x.clone()
    plan.backward(g2, x2, dy, states, g2, x2, ws, dlast=back, dh0=back, resets=resets)
    assert (g2 == want["dgate"]).all() and (x2 == want["dx"]).all() and (back == want["dh0"]).all()


def test_nothing_wanted_and_nothing_given(torch):
    shape = (2, 100, 20)
    v = inputs(torch, shape, "exp", "f32", 10, False)
    v["h0"], v["dlast"] = torch.zeros(2, 20), torch.zeros(2, 20)
    want = run(torch, shape, "exp", "f32", v)
    plan = bltrain.RecurrencePlan(*shape, gate="exp")
    ws, states = plan.workspace(), plan.states()
    gate, x, dy = (v[k].cuda() for k in ("gate", "x", "dy"))
    y, dgate, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    plan.forward(gate, x, y, ws)
    assert (y == want["y"]).all()
    plan.forward(gate, x, y, ws, states=states)
    plan.backward(gate, x, dy, states, dgate, dx, ws)
    assert (dgate == want["dgate"]).all() and (dx == want["dx"]).all()


def test_no_steps_and_no_sequences(torch):
    h0, last = torch.randn(3, 5, device="cuda"), torch.full((3, 5), float("nan"), device="cuda")
    e = torch.empty(3, 0, 5, device="cuda")
    plan = bltrain.RecurrencePlan(3, 0, 5)
    plan.forward(e, e, e, None, h0=h0, last=last)
    assert (last == h0).all()
    plan.forward(e, e, e, None, last=last)
    assert (last == 0).all()
    dh0 = torch.full((3, 5), float("nan"), device="cuda")
    plan.backward(e, e, e, plan.states(), e, e, None, dlast=h0, dh0=dh0)
    assert (dh0 == h0).all()
    e = torch.empty(0, 4, 5, device="cuda")
    plan = bltrain.RecurrencePlan(0, 4, 5)
    plan.forward(e, e, e, None)
    plan.backward(e, e, e, plan.states(), e, e, None)


@pytest.mark.parametrize("shape", [(4, 2000, 40), (300, 500, 1), (1, 9000, 64)])
def test_same_bits_each_time_and_in_a_graph(torch, shape):
    v = inputs(torch, shape, "sigmoid", "bf16", 11, True)
    gate, x, dy, h0, dlast, resets = (v[k].cuda() for k in ("gate", "x", "dy", "h0", "dlast", "resets"))
    plan = bltrain.RecurrencePlan(*shape, dtype=torch.bfloat16)
    ws, states = plan.workspace(), plan.states()
    y, dgate, dx, last, dh0 = (torch.empty_like(k) for k in (x, x, x, h0, h0))

    def both():
        plan.forward(gate, x, y, ws, h0=h0, last=last, resets=resets, states=states)
        plan.backward(gate, x, dy, states, dgate, dx, ws, dlast=dlast, dh0=dh0, resets=resets)
    both()
    want = [k.clone() for k in (y, last, dgate, dx, dh0)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        for k in (y, last, dgate, dx, dh0, states):
            k.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for k, e in zip((y, last, dgate, dx, dh0), want):
            assert (k == e).all()
        both()


def test_the_reference_against_differences():
    """The formulas' gradients against central differences in 64 bits (the host)."""
    import torch as t
    t.manual_seed(0)
    for kind in ("sigmoid", "exp"):
        v = inputs(t, (2, 12, 3), kind, "f32", 12, True)
        w = {k: x.double() if k != "resets" else x for k, x in v.items()}
        args = ("gate", "x", "h0", "dy", "dlast")
        r, _ = reference(t, *(w[k] for k in args), w["resets"], kind)
        for name, of in (("dgate", "gate"), ("dx", "x"), ("dh0", "h0")):
            way, step, ends = t.randn_like(w[of]), 1e-6, []
            for s in (step, -step):
                w[of].add_(way, alpha=s)
                h, _ = reference(t, *(w[k] for k in args), w["resets"], kind)
                ends.append((h["y"] * w["dy"]).sum() + (h["last"] * w["dlast"]).sum())
                w[of].add_(way, alpha=-s)
            # (truncation step^2 times a third derivative of some hundreds, rounding 2^-52 / step)
            assert abs((ends[0] - ends[1]) / (2 * step) - (r[name] * way).sum()) < 1e-6, (kind, name)
