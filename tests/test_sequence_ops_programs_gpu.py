"""Group norm, recurrence and orthogonalised update in programs: what resets and bad values leave alone at every
length, a workspace that captured calls share, and a captured training step with its updates (MI355X).

What is compared bit for bit are calls that do the same operations in the same order on the values that count.
"""
import pytest

from paper_1911_09287_amd import bltrain, gated
from paper_1911_09287_amd.series import waves
from test_recurrence_gpu import inputs, run
from test_train_ops_gpu import torch  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


# (up to eight steps are walked by one thread forward; tiles, waves and chunks of steps)
@pytest.mark.parametrize("shape", [(2, 5, 20), (2, 8, 1), (3, 6, 3), (2, 7, 70), (2, 8, 4096), (2, 9, 20), (2, 300, 20),
                                   (300, 300, 1), (2, 300, 3), (1, 6000, 20)])
@pytest.mark.parametrize("kind", ["sigmoid", "exp"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_bad_crosses_a_reset(torch, shape, kind, dtype):  # noqa: F811
    # bad states, values, gates and gradients before a reset, and behind the reset that ends the sequence
    outer, length, inner = shape
    v = inputs(torch, shape, kind, dtype, 41, False)
    cut, end = length // 3, length - 1 - length // 10
    assert 0 < cut < end < length
    drop = torch.zeros(outer, length, dtype=torch.bool)
    drop[:, cut] = drop[:, end] = True
    v["resets"] = drop
    clean = run(torch, shape, kind, dtype, v)
    for state, gate in ((NAN, NAN), (INF, INF), (-INF, -INF), (NAN, -3e38)):
        w = {k: x.clone() for k, x in v.items()}
        w["h0"][:] = state
        w["dlast"][:] = state
        for k, bad in (("x", state), ("dy", state), ("gate", gate)):
            w[k][:, :cut] = bad
            w[k][:, end:] = bad
        got = run(torch, shape, kind, dtype, w)
        for name in ("y", "dgate", "dx"):
            assert (got[name][:, cut:end] == clean[name][:, cut:end]).all(), (name, state, gate)


@pytest.mark.parametrize("shape", [(3, 7, 20), (3, 300, 20), (3, 300, 1), (3, 300, 3), (1, 6000, 70), (2, 700, 33)])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_what_is_not_finite_stays_in_its_channel_and_behind_its_step(torch, shape, bad):  # noqa: F811
    outer, length, inner = shape
    v = inputs(torch, shape, "sigmoid", "f32", 42, False)
    o, t, i = outer - 1, length // 2, inner // 2
    clean = run(torch, shape, "sigmoid", "f32", v)
    w = {k: None if x is None else x.clone() for k, x in v.items()}
    w["x"][o, t, i] = bad
    w["dy"][o, t, i] = bad
    got = run(torch, shape, "sigmoid", "f32", w)
    there = torch.ones(shape, dtype=torch.bool)
    there[o, :, i] = False
    for name in ("y", "dgate", "dx"):
        assert (got[name].cpu()[there] == clean[name].cpu()[there]).all(), name
    y, dx = got["y"][o, :, i], got["dx"][o, :, i]
    assert (y[:t] == clean["y"][o, :t, i]).all() and not y[t:].isfinite().any()
    assert (dx[t + 1:] == clean["dx"][o, t + 1:, i]).all() and not dx[:t + 1].isfinite().any()


def calls_of(t):
    """(bytes of workspace, call(ws), what it fills) of each operator, in one launch and in several."""
    g = t.Generator().manual_seed(43)

    def rand(*shape):
        return t.randn(*shape, generator=g).cuda()
    for shape in ((6, 200, 64, 8), (6, 5000, 48, 8), (3000, 2, 64, 8)):
        def norm(shape=shape):
            plan = bltrain.GroupNormPlan(*shape, channels_last=True, act="silu")
            x, dy, w, b = rand(*shape[:3]), rand(*shape[:3]), rand(shape[2]), rand(shape[2])
            out = [t.empty_like(v) for v in (x, x, w, b)] + [t.empty(plan.stats_shape(), device="cuda")]

            def call(ws):
                plan.forward(x, w, b, out[0], out[4], ws)
                plan.backward(dy, x, w, b, out[4], out[1], out[2], out[3], ws)
            return plan.workspace_bytes, call, out
        yield norm()
    for shape in ((20, 700, 96), (1, 9000, 64)):
        def steps(shape=shape):
            plan = bltrain.RecurrencePlan(*shape)
            gate, x, dy, h0 = rand(*shape), rand(*shape), rand(*shape), rand(shape[0], shape[2])
            out, states = [t.empty_like(v) for v in (x, x, x, h0, h0)], plan.states()

            def call(ws):
                plan.forward(gate, x, out[0], ws, h0=h0, last=out[3], states=states)
                plan.backward(gate, x, dy, states, out[1], out[2], ws, dh0=out[4])
            return plan.workspace_bytes, call, out
        yield steps()
    for shapes in ([(40, 64), (1024, 9)], [(200, 300), (64, 640), (130, 9)]):
        def update(shapes=shapes):
            plan = bltrain.MuonPlan(shapes)
            out = [t.empty(s, device="cuda") for s in shapes]
            tensors = plan.bind(out, [rand(*s) for s in shapes])
            return plan.workspace_bytes, lambda ws: plan.orthogonalize(tensors, ws), out
        yield update()


def test_captured_calls_share_one_workspace(torch):  # noqa: F811
    calls = list(calls_of(torch))
    room = torch.empty(max(n for n, _, _ in calls), dtype=torch.uint8, device="cuda")
    assert sum(n > 0 for n, _, _ in calls) >= 5
    wants, graphs = [], []
    for n, call, out in calls:
        call(torch.empty(n, dtype=torch.uint8, device="cuda"))  # (in a workspace of its own)
        torch.cuda.synchronize()
        wants.append([v.clone() for v in out])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(room)
        graphs.append(graph)
    for order in (1, -1, 1):
        for _, _, out in calls:
            for v in out:
                v.fill_(NAN)
        room.fill_(255)
        for graph in graphs[::order]:
            graph.replay()
        torch.cuda.synchronize()
        for k, ((_, _, out), want) in enumerate(zip(calls, wants)):
            for v, e in zip(out, want):
                assert (v == e).all(), k
        calls[1][1](room)  # (an eager call between the replays)


def test_a_captured_training_step_updates_as_the_eager_one(torch):  # noqa: F811
    net, eager = (gated.GatedNet(8, 64, 4, channels=32, rate=0.5, seed=44) for _ in range(2))
    series, labels = waves(8, 64, 4, 45)
    for n in (net, eager):  # (an eager pass first: it makes the convolution's tables)
        n.backward(n.forward(series), labels)
    live_m, live_v = (torch.zeros(2, dtype=torch.float64, device="cuda") for _ in range(2))

    def updates(n, live):
        a, b = ({"live": live_m}, {"live": live_v}) if live else ({"lr": lr, "step": step}, {"lr": 0.1 * lr, "step": step})
        n.muon.step(n.muon_tensors, n.muon_state, n.muon_ws, seed=1, **a)
        n.adam.step(n.adam_tensors, n.adam_state, seed=1, **b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.backward(net.forward(series), labels)
        updates(net, True)
    for step in (1, 2, 3):
        lr = 0.02 / step
        live_m.copy_(torch.tensor([lr, step], dtype=torch.float64))
        live_v.copy_(torch.tensor([0.1 * lr, step], dtype=torch.float64))
        for p in net.dmatrices + net.dvectors + net.matrices + net.vectors:
            assert p.isfinite().all()
        for p in net.dmatrices + net.dvectors:
            p.fill_(NAN)
        graph.replay()
        # the same gradients: ten operators of some 100 roundings of 2^-24 each in the worst order (torch's products
        # may take another order of sums where they are captured)
        eager.backward(eager.forward(series), labels)
        torch.cuda.synchronize()
        for p, q in zip(net.dmatrices + net.dvectors, eager.dmatrices + eager.dvectors):
            assert (p - q).norm() <= 1e-4 * q.norm() + 1e-7
        # and of these the same updates, to the last bit
        for p, q in zip(net.dmatrices + net.dvectors, eager.dmatrices + eager.dvectors):
            q.copy_(p)
        updates(eager, False)
        for p, q in zip(net.matrices + net.vectors, eager.matrices + eager.vectors):
            assert (p == q).all()
        assert (net.muon_state == eager.muon_state).all() and (net.adam_state == eager.adam_state).all()
