"""Group norm, recurrence and orthogonalised update: which GPU and stream the binding's calls go to, and
what it refuses, on the host (CPU only, no GPU calls)."""
import os

import pytest
import torch

from paper_1911_09287_amd import blconv, bltrain
from test_train_ops_limits import placed, two_gpus  # noqa: F401  (two_gpus: the fixture)

pytestmark = pytest.mark.skipif(not os.path.exists(blconv.LIB_PATH), reason="libblconv.so not built")


def calls_of_every_kind(use):
    """(name, call, its tensors) of each of the binding's calls; the tensors lie on GPU 1."""
    def on(*shape, dtype=torch.float32):
        return placed(torch.zeros(*shape, dtype=dtype), 1)

    def room(plan):
        return on(plan.workspace_bytes, dtype=torch.uint8)
    norm = use(bltrain.GroupNormPlan(2, 40000, 6, 3, channels_last=True))
    x, w, stats = lambda: on(2, 40000, 6), lambda: on(6), lambda: on(*norm.stats_shape())
    yield "bl_group_norm_forward", norm.forward, [x(), w(), w(), x(), stats(), room(norm)]
    yield "bl_group_norm_backward", norm.backward, [x(), x(), w(), w(), stats(), x(), w(), w(), room(norm)]
    rec = use(bltrain.RecurrencePlan(1, 9000, 64))
    v, state = lambda: on(1, 9000, 64), lambda: on(1, 64)
    resets, states = lambda: on(1, 9000, dtype=torch.uint8), lambda: on(rec.states_elements)
    assert rec.workspace_bytes
    yield ("bl_recurrence_forward",
           lambda g, x, y, ws, h0, last, r, s: rec.forward(g, x, y, ws, h0=h0, last=last, resets=r, states=s),
           [v(), v(), v(), room(rec), state(), state(), resets(), states()])
    yield ("bl_recurrence_backward",
           lambda g, x, dy, s, dg, dx, ws, dl, dh, r: rec.backward(g, x, dy, s, dg, dx, ws, dlast=dl, dh0=dh, resets=r),
           [v(), v(), v(), states(), v(), v(), room(rec), state(), state(), resets()])
    muon = use(bltrain.MuonPlan([(4, 6), (3, 2)]))
    shapes = [(4, 6), (3, 2), (4, 6), (3, 2)]

    def step(p0, p1, g0, g1, s, ws, scale, live):
        muon.step(muon.bind([p0, p1], [g0, g1]), s, ws, grad_scale=scale, live=live)

    def alone(p0, p1, g0, g1, ws):
        muon.orthogonalize(muon.bind([p0, p1], [g0, g1]), ws)
    yield "bl_muon_step", step, [on(*s) for s in shapes] + [on(muon.state_bytes, dtype=torch.uint8), room(muon), on(1),
                                                          on(2, dtype=torch.float64)]
    yield "bl_muon_orthogonalize", alone, [on(*s) for s in shapes] + [room(muon)]


def test_calls_go_to_the_gpu_of_their_tensors(two_gpus):  # noqa: F811
    use, calls = two_gpus
    for name, call, tensors in calls_of_every_kind(use):
        calls.clear()
        call(*tensors)
        assert calls == [(name, 1, 1001)]


def test_calls_refuse_tensors_of_several_gpus_and_of_none(two_gpus):  # noqa: F811
    use, calls = two_gpus
    for name, call, tensors in calls_of_every_kind(use):
        for t in tensors:
            for gpu in (0, -1):
                t.gpu = gpu
                with pytest.raises(ValueError):
                    call(*tensors)
                t.gpu = 1
        call(*tensors)
        assert [c[0] for c in calls] == [name]
        calls.clear()


def test_calls_refuse_a_stream_of_another_gpu(two_gpus):  # noqa: F811
    use, calls = two_gpus
    streams = [type("Stream", (), {"device_index": i, "cuda_stream": 2000 + i})() for i in range(2)]
    rec = use(bltrain.RecurrencePlan(2, 1, 8))
    x, s = placed(torch.zeros(2, 1, 8), 1), placed(torch.zeros(2, 8), 1)
    with pytest.raises(ValueError):
        rec.forward(x, x, x, None, h0=s, last=s, stream=streams[0])
    rec.forward(x, x, x, None, h0=s, last=s, stream=streams[1])
    assert calls == [("bl_recurrence_forward", 1, 2001)]


def test_workspaces_that_are_not_contiguous_are_refused():
    for plan in (bltrain.GroupNormPlan(2, 40000, 6, 3, channels_last=True), bltrain.RecurrencePlan(1, 9000, 64),
                 bltrain.MuonPlan([(4, 6), (100, 200)])):
        n = plan.workspace_bytes
        assert plan._ws(placed(torch.zeros(n, dtype=torch.uint8)), 0)
        for ws in (placed(torch.zeros(1, dtype=torch.uint8)).expand(n), placed(torch.zeros(2 * n, dtype=torch.uint8))[::2],
                   placed(torch.zeros(n - 1, dtype=torch.uint8))):
            with pytest.raises(ValueError):
                plan._ws(ws, 0)


def test_matrices_that_share_memory_are_refused():
    plan = bltrain.MuonPlan([(4, 6), (3, 2), (2, 2)])
    room = placed(torch.zeros(100))
    p, q, r = room[:24].view(4, 6), room[24:30].view(3, 2), room[30:34].view(2, 2)
    g = [placed(torch.zeros(4, 6)), placed(torch.zeros(3, 2)), placed(torch.zeros(2, 2))]
    plan.bind([p, q, r], g)
    plan.bind([p, q, r], [p, q, r])  # (each in the place of its own gradient)
    plan.bind([p, q, r], [g[0], room[40:46].view(3, 2), room[40:44].view(2, 2)])  # (gradients are read alone)
    for params in ([p, room[23:29].view(3, 2), r], [p, p[:1].flatten()[:6].view(3, 2), r], [p, q, q.flatten()[:4].view(2, 2)],
                   [p, q, room[20:24].view(2, 2)]):
        with pytest.raises(ValueError, match="share"):
            plan.bind(params, g)
    for grads in ([room[6:30].view(4, 6), g[1], g[2]], [g[0], p.flatten()[:6].view(3, 2), g[2]],
                  [g[0], g[1], room[22:26].view(2, 2)], [room[29:53].view(4, 6), g[1], g[2]]):
        with pytest.raises(ValueError, match="share"):
            plan.bind([p, q, r], grads)
    # and those of empty matrices may be none
    plan = bltrain.MuonPlan([(4, 6), (0, 2)])
    plan.bind([p, None], [g[0], None])
