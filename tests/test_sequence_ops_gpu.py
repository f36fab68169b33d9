"""Group norm, recurrence and orthogonalised update as programs use them: calls on two streams at a time,
graphs that share a workspace, tensors and workspaces beyond 2^31 elements and 2^32 bytes (MI355X).

What is compared bit for bit are calls that do the same operations in the same order; tolerances are those
of the operators' own tests.
"""
import pytest

from paper_1911_09287_amd import bltrain
from test_group_norm_gpu import bounds as norm_bounds, reference as norm_reference
from test_muon_gpu import USUAL, gradient, reference as muon_reference, within
from test_recurrence_gpu import inputs as steps_inputs, reference as steps_reference
from test_train_ops_gpu import U, half_ulp, near, tdtype, torch  # noqa: F401  (torch: the fixture)

pytestmark = pytest.mark.gpu


def problem(t, kind, seed):
    """call(), which fills `outputs` from tensors and a workspace of its own, and what it fills."""
    g = t.Generator().manual_seed(seed)

    def rand(*shape, dtype=t.float32):
        return t.randn(*shape, generator=g).to(dtype).cuda()
    if kind in ("norm_whole", "norm_parts"):
        shape = (6, 200, 64, 8) if kind == "norm_whole" else (6, 5000, 48, 8)
        plan = bltrain.GroupNormPlan(*shape, channels_last=True, act="silu", dtype=t.bfloat16, wdtype=t.bfloat16)
        x, dy, w, b = (rand(*s, dtype=t.bfloat16) for s in (shape[:3], shape[:3], shape[2:3], shape[2:3]))
        y, dx, dw, db, stats = *(t.empty_like(v) for v in (x, x, w, b)), t.empty(plan.stats_shape(), device="cuda")
        ws = plan.workspace()

        def call():
            plan.forward(x, w, b, y, stats, ws)
            plan.backward(dy, x, w, b, stats, dx, dw, db, ws)
        return call, [y, stats, dx, dw, db], ws
    if kind in ("steps", "steps_chunks"):
        shape = (20, 700, 96) if kind == "steps" else (1, 9000, 64)
        plan = bltrain.RecurrencePlan(*shape)
        gate, x, dy, h0 = rand(*shape), rand(*shape), rand(*shape), rand(shape[0], shape[2])
        y, dgate, dx, last, dh0 = (t.empty_like(v) for v in (x, x, x, h0, h0))
        ws, states = plan.workspace(), plan.states()

        def call():
            plan.forward(gate, x, y, ws, h0=h0, last=last, states=states)
            plan.backward(gate, x, dy, states, dgate, dx, ws, dh0=dh0)
        return call, [y, last, dgate, dx, dh0], ws
    shapes = [(40, 64), (1024, 9)] if kind == "update_small" else [(200, 300), (64, 640), (130, 9)]
    plan = bltrain.MuonPlan(shapes)
    outs, ws = [t.empty(s, device="cuda") for s in shapes], plan.workspace()
    tensors = plan.bind(outs, [rand(*s) for s in shapes])
    return (lambda: plan.orthogonalize(tensors, ws)), outs, ws


KINDS = ["norm_whole", "norm_parts", "steps", "steps_chunks", "update_small", "update"]


def cleared(outputs):
    for v in outputs:
        v.fill_(float("nan"))


def check_bits(outputs, want, what):
    for v, e in zip(outputs, want):
        assert (v == e).all(), what


@pytest.mark.parametrize("kind", KINDS)
def test_two_streams_at_a_time(torch, kind):  # noqa: F811
    problems = [problem(torch, kind, k) for k in range(2)]
    wants = []
    for call, outputs, _ in problems:
        call()
        torch.cuda.synchronize()
        wants.append([v.clone() for v in outputs])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for _, outputs, _ in problems:
            cleared(outputs)
        torch.cuda.synchronize()
        for _ in range(4):
            for stream, (call, _, _) in zip(streams, problems):
                with torch.cuda.stream(stream):
                    call()
        torch.cuda.synchronize()
        for (_, outputs, _), want in zip(problems, wants):
            check_bits(outputs, want, kind)


def test_graphs_that_share_a_workspace(torch):  # noqa: F811
    # one buffer for all plans, whose graphs are replayed one after another, in two orders
    problems = [problem(torch, kind, 5) for kind in KINDS]
    room = torch.empty(max(ws.nbytes if ws is not None else 0 for _, _, ws in problems), dtype=torch.uint8, device="cuda")
    graphs, wants = [], []
    for call, outputs, ws in problems:
        for cell in call.__closure__:  # the plan's own workspace, by a part of the shared one
            if cell.cell_contents is ws and ws is not None:
                cell.cell_contents = room[:ws.nbytes]
        call()
        torch.cuda.synchronize()
        wants.append([v.clone() for v in outputs])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    for order in (1, -1, 1):
        for _, outputs, _ in problems:
            cleared(outputs)
        for graph in graphs[::order]:
            graph.replay()
        torch.cuda.synchronize()
        for (_, outputs, _), want, kind in zip(problems, wants, KINDS):
            check_bits(outputs, want, kind)
        room.fill_(255)
        problems[1][0]()


@pytest.mark.parametrize("last", [True, False])
def test_group_norm_of_more_than_31_bits_of_values(torch, last):  # noqa: F811
    # 160 samples alike: every one's results are the first one's, and the weights' gradients 160 times its own
    batch, sites, channels, groups, act = 160, 1 << 18, 64, 8, "silu"
    size = (sites, channels) if last else (channels, sites)
    g = torch.Generator(device="cuda").manual_seed(3)
    one = (torch.randn(1, *size, generator=g, device="cuda") + 0.5).bfloat16()
    done = torch.randn(1, *size, generator=g, device="cuda").bfloat16()
    w, b = (torch.randn(channels, generator=g, device="cuda") * 0.3 + 1 for _ in range(2))
    x, dy = one.repeat(batch, 1, 1), done.repeat(batch, 1, 1)
    assert x.numel() > 1 << 31
    plan = bltrain.GroupNormPlan(batch, sites, channels, groups, channels_last=last, act=act, dtype=torch.bfloat16,
                                 wdtype=torch.float32)
    y, dx, stats = torch.empty_like(x), torch.empty_like(x), torch.empty(plan.stats_shape(), device="cuda")
    dw, db, ws = torch.empty_like(w), torch.empty_like(b), plan.workspace()
    plan.forward(x, w, b, y, stats, ws)
    plan.backward(dy, x, w, b, stats, dx, dw, db, ws)
    for v in (y, dx):
        for n in range(0, batch, 16):
            assert (v[n:n + 16] == v[:1]).all(), n
    assert (stats == stats[:, :1]).all()
    xd, dyd = one.double(), done.double()
    r = norm_reference(torch, xd, w.double(), b.double(), dyd, groups, last, act, 1e-5)
    most = norm_bounds(xd, dyd, r, groups, last, act, "bf16", "f32")
    for name, got in (("y", y[:1]), ("mean", stats[0, :1]), ("rstd", stats[1, :1]), ("dx", dx[:1])):
        near(got, r[name], most[name], name)
    for name, got in (("dw", dw), ("db", db)):
        near(got, batch * r[name], batch * most[name], name)


def test_recurrence_of_more_than_31_bits_of_values(torch):  # noqa: F811
    # 512 times the same 64 channels in each of 24 sequences alike
    outer, length, inner, times = 24, 4096, 64, 512
    v = steps_inputs(torch, (1, length, inner), "sigmoid", "bf16", 4, True)

    def large(k):
        return v[k].cuda().repeat(outer, *(() if v[k].dim() == 2 else (1,)), times)
    gate, x, dy, h0, dlast = (large(k) for k in ("gate", "x", "dy", "h0", "dlast"))
    resets = v["resets"].cuda().repeat(outer, 1)
    assert x.numel() > 1 << 31 and x.shape == (outer, length, inner * times)
    plan = bltrain.RecurrencePlan(outer, length, inner * times, dtype=torch.bfloat16)
    y, dgate, dx, last, dh0 = (torch.empty_like(k) for k in (x, x, x, h0, h0))
    ws, states = plan.workspace(), plan.states()
    plan.forward(gate, x, y, ws, h0=h0, last=last, resets=resets, states=states)
    plan.backward(gate, x, dy, states, dgate, dx, ws, dlast=dlast, dh0=dh0, resets=resets)
    r, most = steps_reference(torch, *(v[k].double() for k in ("gate", "x", "h0", "dy", "dlast")), v["resets"], "sigmoid")
    for name, got in (("y", y), ("dgate", dgate), ("dx", dx), ("last", last), ("dh0", dh0)):
        first = got[:1, ..., :inner]
        for n in range(outer):
            assert (got[n].view(*got.shape[1:-1], times, inner) == first[0].unsqueeze(-2)).all(), (name, n)
        bound = most[name]
        if name in ("y", "dgate", "dx"):
            bound = bound + half_ulp("bf16") * (r[name].abs() + bound) + 1e-30
        near(first, r[name], bound, name)


@pytest.mark.parametrize("inner", [1, 8])
def test_recurrence_of_strides_beyond_32_bits(torch, inner):  # noqa: F811
    # gates and values of a step in one tensor whose steps (inner = 1: sequences) lie 2^25 elements and more apart
    shape = (2, 70, 8) if inner > 1 else (70, 40, 1)
    far = (1 << 25) + 24
    v = steps_inputs(torch, shape, "exp", "bf16", 6, True)
    strides = (70 * far + 8, far) if inner > 1 else (far, 1)
    room = torch.empty(strides[0] * (shape[0] - 1) + strides[1] * (shape[1] - 1) + 64, dtype=torch.bfloat16, device="cuda")
    other = torch.empty_like(room)

    def part(of, at):
        return torch.as_strided(of, shape, (*strides, 1), at)
    gate, x, y, dy, dgate, dx = (part(of, at) for of, at in ((room, 0), (room, 40), (other, 0), (other, 40),
                                                             (torch.empty_like(room), 0), (torch.empty_like(room), 0)))
    for to, k in ((gate, "gate"), (x, "x"), (dy, "dy")):
        to.copy_(v[k])
    plan = bltrain.RecurrencePlan(*shape, gate="exp", dtype=torch.bfloat16, in_strides=strides, out_strides=strides)
    h0, dlast, resets = (v[k].cuda() for k in ("h0", "dlast", "resets"))
    last, dh0, ws, states = torch.empty_like(h0), torch.empty_like(h0), plan.workspace(), plan.states()
    plan.forward(gate, x, y, ws, h0=h0, last=last, resets=resets, states=states)
    plan.backward(gate, x, dy, states, dgate, dx, ws, dlast=dlast, dh0=dh0, resets=resets)
    r, most = steps_reference(torch, *(v[k].double() for k in ("gate", "x", "h0", "dy", "dlast")), v["resets"], "exp")
    for name, got in (("y", y), ("dgate", dgate), ("dx", dx), ("last", last), ("dh0", dh0)):
        bound = most[name]
        if name in ("y", "dgate", "dx"):
            bound = bound + half_ulp("bf16") * (r[name].abs() + bound) + 1e-30
        near(got, r[name], bound, name)


def test_update_with_a_workspace_of_more_than_32_bits(torch):  # noqa: F811
    # one step of the polynomials; two large matrices alike, and small ones before and behind them
    large, shapes = (8192, 8192), [(300, 512), (8192, 8192), (8192, 8192), (512, 300)]
    g = torch.Generator(device="cuda").manual_seed(7)
    u = torch.randn(*large, generator=g, device="cuda") * 1e-3
    few = gradient(torch, shapes[0], 8).cuda()
    plan = bltrain.MuonPlan(shapes, coefficients=USUAL[:1])
    assert plan.workspace_bytes > 1 << 32
    outs = [torch.full(s, float("nan"), device="cuda") for s in shapes]
    plan.orthogonalize(plan.bind(outs, [few, u, u, few.t().contiguous()]), plan.workspace())
    assert (outs[1] == outs[2]).all()
    want, err = muon_reference(torch, few, 1e-7, USUAL[:1])
    for got in (outs[0], outs[3].t()):
        within(got, want, err + U * want.norm().item(), "small")
    want, err = muon_reference(torch, u, 1e-7, USUAL[:1])
    within(outs[1], want, err + U * want.norm().item(), "large")
