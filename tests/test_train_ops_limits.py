"""The operators around the convolution layer at the ends of their ranges, on the host (CPU
only, no GPU calls): what the bindings and the plans have to refuse."""
import os

import pytest
import torch

from paper_1911_09287_amd import blconv, bltrain

pytestmark = pytest.mark.skipif(not os.path.exists(blconv.LIB_PATH), reason="libblconv.so not built")


class Placed(torch.Tensor):
    """A tensor of the host that says it lies on a GPU, for checks that come before any launch."""

    is_cuda, gpu = True, 0

    def get_device(self):
        return self.gpu


def placed(t, gpu=0):
    t = t.as_subclass(Placed)
    t.gpu = gpu
    return t


def test_workspaces_that_are_not_contiguous_are_refused():
    # an expanded tensor has as many bytes as it says, and its storage one
    norm, prob = bltrain.NormPlan(2, 100000), bltrain.LogProbPlan(2, 100000)
    conv = blconv.Plan(1, 2, 1, 2, (16,), 3, (1, 1), 0.0)
    x, stats = placed(torch.zeros(2, 100000)), placed(torch.zeros(2, 2, 1))
    w = placed(torch.zeros(100000))
    for plan, on in ((norm, (0,)), (prob, (0,)), (conv, ())):
        assert plan._ws(placed(torch.zeros(plan.workspace_bytes, dtype=torch.uint8)), *on)
        for ws in (placed(torch.zeros(1, dtype=torch.uint8)).expand(plan.workspace_bytes),
                   placed(torch.zeros(2 * plan.workspace_bytes, dtype=torch.uint8))[::2]):
            with pytest.raises(ValueError):
                plan._ws(ws, *on)
    ws = placed(torch.zeros(1, dtype=torch.uint8)).expand(norm.workspace_bytes)
    with pytest.raises(ValueError):
        norm.forward(x, None, None, x, stats, ws)
    with pytest.raises(ValueError):
        norm.backward(x, x, None, stats, x, w, w, ws)
    ws = placed(torch.zeros(1, dtype=torch.uint8)).expand(prob.workspace_bytes)
    with pytest.raises(ValueError):
        prob.forward(x, None, None, None, None, None, ws)


@pytest.fixture
def two_gpus(monkeypatch):
    """A host that seems to have two GPUs, 0 current, and a library that notes which one is current, and the
    stream, when it is called: the list of those notes."""
    current, calls = [0], []

    class Device:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            self.before, current[0] = current[0], self.device

        def __exit__(self, *a):
            current[0] = self.before

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1000 + device)
    monkeypatch.setattr(torch.cuda, "device", Device)

    class Library:
        def __init__(self, lib):
            self.lib = lib

        def __getattr__(self, name):
            if name.endswith("_destroy"):
                return getattr(self.lib, name)

            def call(*args):
                calls.append((name, current[0], args[-1]))
                return 0
            return call

    def use(plan):
        plan._lib = Library(plan._lib)
        return plan
    yield use, calls
    assert current == [0]


def calls_of_every_kind(use):
    """(name, call, its tensors) of each of the binding's calls; the tensors lie on GPU 1."""
    def on(*shape, dtype=torch.float32):
        return placed(torch.zeros(*shape, dtype=dtype), 1)

    def room(plan):
        return on(plan.workspace_bytes, dtype=torch.uint8)
    norm, prob = use(bltrain.NormPlan(2, 100000)), use(bltrain.LogProbPlan(2, 100000, top=1))
    rows, w, stats = lambda: on(2, 100000), lambda: on(100000), lambda: on(2, 2, 1)
    one = lambda dtype=torch.float32: on(2, 1, dtype=dtype)  # noqa: E731
    adam = use(bltrain.AdamWPlan([4, 2], bits=8))
    state = lambda: on(adam.state_bytes, dtype=torch.uint8)  # noqa: E731
    yield "bl_norm_forward", norm.forward, [rows(), w(), w(), rows(), stats(), room(norm)]
    yield "bl_norm_backward", norm.backward, [rows(), rows(), w(), stats(), rows(), w(), w(), room(norm)]
    yield "bl_logprob_forward", prob.forward, [rows(), one(torch.int64), one(), on(3, 2), one(), one(torch.int64),
                                               room(prob)]
    yield "bl_logprob_backward", prob.backward, [rows(), one(torch.int64), on(3, 2), one(), one(), rows()]

    def step(p0, p1, g0, g1, s, scale, live):
        adam.step(adam.bind([p0, p1], [g0, g1]), s, grad_scale=scale, live=live)
    yield "bl_adamw_step", step, [on(4), on(2), on(4), on(2), state(), on(1), on(2, dtype=torch.float64)]
    half = torch.bfloat16
    yield "bl_adamw_get_moments", adam.moments, [state(), on(adam.total, dtype=half), on(adam.total, dtype=half)]
    yield "bl_adamw_set_moments", adam.load_moments, [state(), on(adam.total), on(adam.total)]


def test_calls_go_to_the_gpu_of_their_tensors(two_gpus):
    # launches go to the current GPU: that of the tensors has to be current during the call, and its stream given
    use, calls = two_gpus
    for name, call, tensors in calls_of_every_kind(use):
        calls.clear()
        call(*tensors)
        assert calls == [(name, 1, 1001)]


def test_calls_refuse_tensors_of_several_gpus_and_of_none(two_gpus):
    use, calls = two_gpus
    for name, call, tensors in calls_of_every_kind(use):
        for i, t in enumerate(tensors):
            for gpu in (0, -1):
                t.gpu = gpu
                with pytest.raises(ValueError):
                    call(*tensors)
                t.gpu = 1
        call(*tensors)
        assert [c[0] for c in calls] == [name]
        calls.clear()


def test_calls_refuse_a_stream_of_another_gpu(two_gpus):
    use, calls = two_gpus
    streams = [type("Stream", (), {"device_index": i, "cuda_stream": 2000 + i})() for i in range(2)]
    norm = use(bltrain.NormPlan(2, 8))
    x, ws = placed(torch.zeros(2, 8), 1), placed(torch.zeros(norm.workspace_bytes, dtype=torch.uint8), 1)
    with pytest.raises(ValueError):
        norm.forward(x, None, None, x, None, ws, stream=streams[0])
    norm.forward(x, None, None, x, None, ws, stream=streams[1])
    assert calls == [("bl_norm_forward", 1, 2001)]


def test_adamw_tensors_as_large_as_a_launch():
    # a block takes 1024 elements, and 2^24 blocks of 256 threads are more than a launch may have
    most = (1 << 34) - 1024
    assert bltrain.AdamWPlan([most]).starts == [0]
    assert bltrain.AdamWPlan([most, 5, most]).starts == [0, most, most + 1024]
    for sizes in ([most + 1], [(1 << 34) - 1], [5, most + 1], [(1 << 63) - 1]):
        with pytest.raises(bltrain.BlError) as e:
            bltrain.AdamWPlan(sizes)
        assert e.value.code == 2  # BL_ERR_UNSUPPORTED


def test_norm_rows_whose_weight_gradients_fit_a_launch():
    # the last sum has a thread for each of 2 size columns, 64 a block
    assert bltrain.NormPlan(0, (1 << 31) - 32).workspace_bytes == 0
    assert bltrain.NormPlan(1, (1 << 31) - 32).workspace_bytes > 0
    for outer, size in ((0, (1 << 31) - 31), (1, (1 << 31) - 1)):
        with pytest.raises(bltrain.BlError) as e:
            bltrain.NormPlan(outer, size)
        assert e.value.code == 2  # BL_ERR_UNSUPPORTED


def test_adamw_takes_none_for_empty_tensors(two_gpus):
    use, calls = two_gpus
    adam = use(bltrain.AdamWPlan([0, 4, 0]))
    p, g = (placed(torch.zeros(4), 1) for _ in range(2))
    tensors = adam.bind([None, p, None], [None, g, None])
    adam.step(tensors, placed(torch.zeros(adam.state_bytes, dtype=torch.uint8), 1))
    assert calls == [("bl_adamw_step", 1, 1001)]
    none = use(bltrain.AdamWPlan([0]))
    none.step(none.bind([None], [None]), placed(torch.zeros(0, dtype=torch.uint8), 1))
