"""Host side of group norm, the gated recurrence and the orthogonalised update (CPU only,
no GPU calls): plans and their refusals, null arguments, and the binding's checks of tensors."""
import ctypes
import os

import pytest
import torch

from paper_1911_09287_amd import blconv, bltrain
from test_train_ops_limits import placed

pytestmark = pytest.mark.skipif(not os.path.exists(blconv.LIB_PATH), reason="libblconv.so not built")

INVALID, UNSUPPORTED = 1, 2
BIG = (1 << 63) - 1


def _code(call, *args, **kw):
    with pytest.raises(bltrain.BlError) as e:
        call(*args, **kw)
    return e.value.code


@pytest.mark.parametrize("args,kw,code", [
    ((-1, 4, 8, 2), {}, INVALID), ((2, 0, 8, 2), {}, INVALID), ((2, 4, 0, 1), {}, INVALID), ((2, 4, 8, 0), {}, INVALID),
    ((2, 4, 8, 3), {}, INVALID), ((2, 4, 8, 2), {"eps": -1e-5}, INVALID), ((2, 4, 8, 2), {"eps": float("nan")}, INVALID),
    ((2, 4, 8, 2), {"x_stride": 31}, INVALID), ((2, 4, 8, 2), {"y_stride": -32}, INVALID),
    ((2, 4, 8, 2), {"wdtype": torch.bfloat16}, INVALID),
    ((1, 1 << 16, 1 << 15, 2), {}, UNSUPPORTED), ((1 << 20, 1, 1 << 11, 2), {}, UNSUPPORTED),
    ((1 << 31, 1, 1, 1), {}, UNSUPPORTED), ((1, BIG, 1, 1), {}, UNSUPPORTED), ((1, 1, BIG, 1), {}, UNSUPPORTED),
    ((1 << 25, 1, 1, 1), {"channels_last": True}, UNSUPPORTED), ((1, 1, 1 << 30, 1), {}, UNSUPPORTED),
    ((1, 1, 1 << 30, 1 << 20), {"channels_last": True}, UNSUPPORTED), ((0, 1, 1 << 30, 1 << 20), {}, UNSUPPORTED), ((2, 4, 8, 2), {"x_stride": 1 << 61}, UNSUPPORTED),
])
def test_group_norm_plan_refusals(args, kw, code):
    assert _code(bltrain.GroupNormPlan, *args, **kw) == code


@pytest.mark.parametrize("args,kw,code", [
    ((-1, 4), {}, INVALID), ((2, -1), {}, INVALID), ((2, 4, 0), {}, INVALID),
    ((2, 4, 8), {"in_strides": (0, 7)}, INVALID), ((2, 4, 8), {"in_strides": (31, 8)}, INVALID),
    ((2, 4, 8), {"out_strides": (0, 7)}, INVALID), ((2, 4, 8), {"out_strides": (-32, 8)}, INVALID),
    ((2, 4, 8), {"in_strides": (8, 15)}, INVALID), ((2, 4, 8), {"in_strides": (7, 16)}, INVALID),
    ((1 << 31, 4), {}, UNSUPPORTED), ((2, 1 << 31), {}, UNSUPPORTED), ((1 << 16, 4, 1 << 15), {}, UNSUPPORTED),
    ((2, 4, BIG), {}, UNSUPPORTED), ((2, 1 << 20, 8), {"in_strides": (0, 1 << 50)}, UNSUPPORTED),
    ((1 << 20, 4, 8), {"in_strides": (1 << 50, 8)}, UNSUPPORTED), ((1 << 27, 4), {}, UNSUPPORTED),
])
def test_recurrence_plan_refusals(args, kw, code):
    assert _code(bltrain.RecurrencePlan, *args, **kw) == code


def test_recurrence_plans_of_interleaved_layouts():
    bltrain.RecurrencePlan(5, 9, 8, in_strides=(8, 40), out_strides=(8, 41))  # steps outermost
    bltrain.RecurrencePlan(5, 9, 8, in_strides=(200, 16))                      # halves of one tensor
    bltrain.RecurrencePlan(1, 9, 8, in_strides=(0, 8))
    bltrain.RecurrencePlan(3, 1, 8, in_strides=(8, 0))


@pytest.mark.parametrize("shapes,kw,code", [
    ([(4, -1)], {}, INVALID), ([(-4, 1)], {}, INVALID), ([(4, 4)], {"param_dtype": torch.float16}, INVALID),
    ([(4, 4)], {"scales": [float("inf")]}, INVALID), ([(4, 4)], {"coefficients": []}, INVALID),
    ([(4, 4)], {"coefficients": [(1.5, -0.5, 0.0)] * 17}, INVALID),
    ([(4, 4)], {"coefficients": [(float("nan"), 0.0, 0.0)]}, INVALID),
    ([(4, 4)], {"coefficients": [(1.8, 0.0, 0.0)]}, INVALID),       # 1 becomes 1.8
    ([(4, 4)], {"coefficients": [(1.5, 0.0, 0.0)] * 2}, INVALID),   # and 2.25 in the second step
    ([(4, 4)], {"coefficients": [(6.0, -8.0, 3.0)]}, INVALID),      # 0.6 becomes 2.1
    ([(65537, 4)], {}, UNSUPPORTED), ([(4, 65537)], {}, UNSUPPORTED), ([(65536, 32768)], {}, UNSUPPORTED),
    ([(BIG, BIG)], {}, UNSUPPORTED),
])
def test_muon_plan_refusals(shapes, kw, code):
    assert _code(bltrain.MuonPlan, shapes, **kw) == code


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_recurrence_plans_of_any_number_of_channels(dtype):
    # among them numbers that leave one channel over whatever lanes a block takes (4 lcm(1 ... 16) + 1)
    for inner in list(range(1, 300)) + [2882881, 2882882, 2882883]:
        bltrain.RecurrencePlan(1, 50, inner, dtype=dtype)


def test_muon_layout():
    plan = bltrain.MuonPlan([(3, 5), (0, 7), (8, 8), (1, 1)])
    assert plan.starts == [0, 64, 64, 128] and plan.total == 192 and plan.state_bytes == 768


def test_plans_refuse_other_types_and_names():
    for make in (lambda: bltrain.GroupNormPlan(2, 4, 8, 2, dtype=torch.float64),
                 lambda: bltrain.GroupNormPlan(2, 4, 8, 2, act="tanh"),
                 lambda: bltrain.RecurrencePlan(2, 4, dtype=torch.int32), lambda: bltrain.RecurrencePlan(2, 4, gate="relu"),
                 lambda: bltrain.MuonPlan([(4, 4)], grad_dtype=torch.float64),
                 lambda: bltrain.MuonPlan([(4, 4)], decay=[True, False]), lambda: bltrain.MuonPlan([(4, 4)], scales=[]),
                 lambda: bltrain.MuonPlan([(4, 4)], coefficients=[(1.0, 2.0)])):
        with pytest.raises(ValueError):
            make()


def test_calls_refuse_null_and_misaligned_arguments():
    lib = bltrain.load()
    some, odd = ctypes.c_void_p(16), ctypes.c_void_p(24)  # never reached: each call is refused on the host
    norm = bltrain.GroupNormPlan(2, 4, 8, 2)
    assert norm.workspace_bytes
    assert lib.bl_group_norm_plan_create(None, None) == INVALID
    assert lib.bl_group_norm_forward(None, *[some] * 7) == INVALID
    for k in (0, 3):  # x, y
        args = [some] * 6
        args[k] = None
        assert lib.bl_group_norm_forward(norm._h, *args, None) == INVALID
    for k in (0, 1, 4, 5):  # dy, x, stats, dx
        args = [some] * 9
        args[k] = None
        assert lib.bl_group_norm_backward(norm._h, *args, None) == INVALID
    for ws in (None, odd):
        assert lib.bl_group_norm_forward(norm._h, some, some, some, some, some, ws, None) == INVALID
        assert lib.bl_group_norm_backward(norm._h, *[some] * 8, ws, None) == INVALID
    recur = bltrain.RecurrencePlan(1, 100000, 8)
    assert recur.workspace_bytes
    for k in (0, 1, 4):  # gate, x, y
        args = [some] * 8
        args[k] = None
        assert lib.bl_recurrence_forward(recur._h, *args, None) == INVALID
    for k in (0, 1, 3, 4, 6, 7):  # gate, x, states, dy, dgate, dx
        args = [some] * 10
        args[k] = None
        assert lib.bl_recurrence_backward(recur._h, *args, None) == INVALID
    for ws in (None, odd):
        assert lib.bl_recurrence_forward(recur._h, *[some] * 7, ws, None) == INVALID
        assert lib.bl_recurrence_backward(recur._h, *[some] * 9, ws, None) == INVALID
    muon = bltrain.MuonPlan([(4, 4)])
    ptrs, empty = (ctypes.c_void_p * 1)(16), (ctypes.c_void_p * 1)(None)

    def step(p=ptrs, g=ptrs, state=some, ws=some, **kw):
        a = bltrain.MuonArgs(0.02, 0.95, 1e-7, 0.0, 1, 1, 0, None, None)
        for name, v in kw.items():
            setattr(a, name, v)
        return lib.bl_muon_step(muon._h, p, g, state, ws, ctypes.byref(a), None)
    for kw in ({"p": empty}, {"g": None}, {"g": empty}, {"state": None}, {"state": odd}, {"ws": None}, {"ws": odd},
               {"momentum": 1.0}, {"momentum": -0.1}, {"eps": 0.0}, {"eps": float("nan")}, {"lr": -1.0},
               {"lr": float("inf")}, {"weight_decay": -1.0}, {"step": 0}):
        assert step(**kw) == INVALID, kw
    for args in ((None, ptrs, some, 1e-7), (ptrs, empty, some, 1e-7), (ptrs, ptrs, None, 1e-7), (ptrs, ptrs, odd, 1e-7),
                 (ptrs, ptrs, some, 0.0)):
        assert lib.bl_muon_orthogonalize(muon._h, *args, None) == INVALID


def test_binding_refuses_tensors_that_do_not_fit():
    def on(*shape, dtype=torch.float32):
        return placed(torch.zeros(*shape, dtype=dtype))
    norm = bltrain.GroupNormPlan(2, 4, 8, 2)
    x, w, stats, ws = on(2, 8, 4), on(8), on(2, 2, 2), on(norm.workspace_bytes, dtype=torch.uint8)
    bad = [(torch.zeros(2, 8, 4), w, w, x, stats, ws), (x, on(7), w, x, stats, ws), (x, w, w, on(2, 8, 5), stats, ws),
           (x, w, w, x, on(2, 2, 3), ws), (x, w, w, x, stats, on(3, dtype=torch.uint8)),
           (on(2, 4, 8).transpose(1, 2), w, w, x, stats, ws), (x.double(), w, w, x, stats, ws)]
    for args in bad:
        with pytest.raises(ValueError):
            norm.forward(*args)
    with pytest.raises(ValueError):
        norm.backward(x, x, w, w, stats, x, on(9), w, ws)
    recur = bltrain.RecurrencePlan(2, 6, 4, in_strides=(48, 8))
    both, y, h = on(2, 6, 8), on(2, 6, 4), on(2, 4)
    good = dict(gate=both[..., :4], x=both[..., 4:], y=y, ws=None, h0=h, last=h, resets=on(2, 6, dtype=torch.bool),
                states=on(recur.states_elements))
    for name, v in (("gate", y), ("x", torch.zeros(2, 6, 4)), ("y", both[..., :4]), ("y", on(2, 4, 6)[..., :4]),
                    ("h0", on(2, 5)), ("last", h.double()), ("resets", on(2, 5, dtype=torch.uint8)),
                    ("resets", on(2, 6)), ("states", on(recur.states_elements + 1)), ("gate", both.half()[..., :4])):
        with pytest.raises(ValueError):
            recur.forward(**dict(good, **{name: v}))
    muon = bltrain.MuonPlan([(4, 6), (3, 3)])
    p = [on(4, 6), on(3, 3)]
    for params, grads in ((p[:1], p), (p, p[:1]), ([on(4, 5), p[1]], p), ([on(6, 4).t(), p[1]], p),
                          ([torch.zeros(4, 6), p[1]], p), (p, [on(4, 6).half(), p[1]])):
        with pytest.raises(ValueError):
            muon.bind(params, grads)
    other = bltrain.MuonPlan([(4, 6), (3, 3)])
    with pytest.raises(ValueError):
        other.orthogonalize(muon.bind(p, p), on(other.workspace_bytes, dtype=torch.uint8))
    with pytest.raises(ValueError):
        muon.step(muon.bind(p, p), on(5, dtype=torch.uint8), on(muon.workspace_bytes, dtype=torch.uint8))
    elsewhere = placed(torch.zeros(muon.state_bytes, dtype=torch.uint8), 1)
    with pytest.raises(ValueError):
        muon.step(muon.bind(p, p), elsewhere, on(muon.workspace_bytes, dtype=torch.uint8))
