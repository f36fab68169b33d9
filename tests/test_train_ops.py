"""Host side of the operators around the convolution layer (CPU only, no GPU calls):
declared and exported calls, plans and their refusals, the moments' layout, the
binding's checks of tensors, and the dither's hash as the header gives it."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_1911_09287_amd import blconv, bltrain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.skipif(not os.path.exists(blconv.LIB_PATH), reason="libblconv.so not built")

INVALID, UNSUPPORTED = 1, 2


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "bltrain.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(bl_[a-z_]+)\s*\(", header))
    lib = bltrain.load()
    for name in declared:
        assert hasattr(lib, name), name
    assert declared == set(bltrain.EXPORTED)


def _code(call, *args, **kw):
    with pytest.raises(bltrain.BlError) as e:
        call(*args, **kw)
    return e.value.code


@pytest.mark.parametrize("args,kw,code", [
    ((-1, 4), {}, INVALID), ((2, 0), {}, INVALID), ((2, 4, 0), {}, INVALID),
    ((2, 4), {"eps": -1e-5}, INVALID), ((2, 4), {"eps": float("nan")}, INVALID),
    ((2, 4), {"eps": float("inf")}, INVALID), ((2, 4), {"x_stride": 3}, INVALID), ((2, 4), {"y_stride": 3}, INVALID),
    ((2, 4), {"x_stride": -8}, INVALID), ((2, 4), {"wdtype": torch.bfloat16}, INVALID),
    ((2, 4), {"dtype": torch.float16, "wdtype": torch.bfloat16}, INVALID),
    ((1, 1 << 31), {}, UNSUPPORTED), ((1, 1 << 16, 1 << 15), {}, UNSUPPORTED), ((1 << 31, 1), {}, UNSUPPORTED),
    ((1 << 20, 1, 1 << 11), {}, UNSUPPORTED), ((1, (1 << 63) - 1, (1 << 63) - 1), {}, UNSUPPORTED),
])
def test_norm_plan_refusals(args, kw, code):
    assert _code(bltrain.NormPlan, *args, **kw) == code


@pytest.mark.parametrize("args,kw,code", [
    ((-1, 4), {}, INVALID), ((2, 0), {}, INVALID), ((2, 4, -1), {}, INVALID), ((2, 4), {"stride": 3}, INVALID),
    ((2, 4), {"grad_stride": 2}, INVALID), ((2, 4, 65), {}, UNSUPPORTED), ((2, 1 << 31), {}, UNSUPPORTED),
    ((1 << 31, 4), {}, UNSUPPORTED),
])
def test_logprob_plan_refusals(args, kw, code):
    assert _code(bltrain.LogProbPlan, *args, **kw) == code


@pytest.mark.parametrize("sizes,kw,code", [
    ([4, -1], {}, INVALID), ([4], {"bits": 16}, INVALID), ([4], {"param_dtype": torch.float16}, INVALID),
    ([1 << 40], {}, UNSUPPORTED), ([(1 << 40) - 1] * 3, {}, UNSUPPORTED),
])
def test_adamw_plan_refusals(sizes, kw, code):
    assert _code(bltrain.AdamWPlan, sizes, **kw) == code


def test_plans_refuse_other_types():
    with pytest.raises(ValueError):
        bltrain.NormPlan(2, 4, dtype=torch.float64)
    with pytest.raises(ValueError):
        bltrain.LogProbPlan(2, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        bltrain.AdamWPlan([4], grad_dtype=torch.float64)
    with pytest.raises(ValueError):
        bltrain.AdamWPlan([4, 5], decay=[True])


def test_calls_refuse_null_arguments():
    lib = bltrain.load()
    norm, prob, adam = bltrain.NormPlan(2, 4), bltrain.LogProbPlan(2, 4, top=1), bltrain.AdamWPlan([4])
    some = ctypes.c_void_p(16)  # never reached: each call is refused on the host
    none = [None] * 12
    assert lib.bl_norm_plan_create(None, None) == INVALID
    assert lib.bl_norm_forward(None, *none[:7]) == INVALID
    assert lib.bl_norm_forward(norm._h, None, None, None, some, None, None, None) == INVALID
    assert lib.bl_norm_forward(norm._h, some, None, None, None, None, None, None) == INVALID
    assert lib.bl_norm_backward(norm._h, some, some, None, None, some, None, None, some, None) == INVALID
    assert lib.bl_logprob_forward(prob._h, some, None, some, some, None, some, some, None) == INVALID
    assert lib.bl_logprob_forward(prob._h, None, None, some, some, some, some, some, None) == INVALID
    assert lib.bl_logprob_backward(prob._h, some, None, None, some, None, some, None) == INVALID
    args = bltrain.AdamWArgs(1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0, None, None)
    ptrs = (ctypes.c_void_p * 1)(16)
    empty = (ctypes.c_void_p * 1)(None)
    assert lib.bl_adamw_step(adam._h, ptrs, ptrs, None, ctypes.byref(args), None) == INVALID
    assert lib.bl_adamw_step(adam._h, empty, ptrs, some, ctypes.byref(args), None) == INVALID
    assert lib.bl_adamw_step(adam._h, ptrs, None, some, ctypes.byref(args), None) == INVALID
    for name, value in (("step", 0), ("beta1", 1.0), ("beta2", -0.1), ("eps", -1.0), ("lr", float("nan")),
                        ("weight_decay", float("inf"))):
        bad = bltrain.AdamWArgs(1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0, None, None)
        setattr(bad, name, value)
        assert lib.bl_adamw_step(adam._h, ptrs, ptrs, some, ctypes.byref(bad), None) == INVALID, name


def test_calls_refuse_misaligned_workspaces_and_states():
    lib = bltrain.load()
    some, odd = ctypes.c_void_p(16), ctypes.c_void_p(24)
    norm, prob, adam = bltrain.NormPlan(2, 100000), bltrain.LogProbPlan(2, 100000, top=1), bltrain.AdamWPlan([4])
    assert norm.workspace_bytes and prob.workspace_bytes
    for ws in (None, odd):
        assert lib.bl_norm_forward(norm._h, some, None, None, some, None, ws, None) == INVALID
        assert lib.bl_norm_backward(norm._h, some, some, None, some, some, None, None, ws, None) == INVALID
        assert lib.bl_logprob_forward(prob._h, some, None, some, some, some, some, ws, None) == INVALID
    args = bltrain.AdamWArgs(1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0, None, None)
    ptrs = (ctypes.c_void_p * 1)(16)
    assert lib.bl_adamw_step(adam._h, ptrs, ptrs, odd, ctypes.byref(args), None) == INVALID
    assert lib.bl_adamw_get_moments(adam._h, odd, some, some, None) == INVALID
    assert lib.bl_adamw_set_moments(adam._h, odd, some, some, None) == INVALID


def test_binding_refuses_tensors_off_the_gpu_and_wrong_lists():
    plan = bltrain.NormPlan(2, 4)
    x = torch.zeros(2, 4)
    with pytest.raises(ValueError):
        plan.forward(x, None, None, x, None, None)
    adam = bltrain.AdamWPlan([4, 2])
    with pytest.raises(ValueError):
        adam.bind([x], [x])
    with pytest.raises(ValueError):
        adam.bind([x[0], x[0, :2]], [x[0], x[0, :2]])


def test_calls_without_work_need_no_gpu():
    lib = bltrain.load()
    prob, adam = bltrain.LogProbPlan(0, 4), bltrain.AdamWPlan([0, 0])
    assert lib.bl_logprob_forward(prob._h, *[None] * 8) == 0
    assert lib.bl_logprob_backward(prob._h, *[None] * 7) == 0
    args = bltrain.AdamWArgs(1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0, None, None)
    assert lib.bl_adamw_step(adam._h, None, None, None, ctypes.byref(args), None) == 0
    assert adam.state_bytes == 0 and bltrain.AdamWPlan([]).total == 0
    norm = bltrain.NormPlan(0, 4)
    assert lib.bl_norm_forward(norm._h, *[None] * 7) == 0
    assert lib.bl_norm_backward(norm._h, *[None] * 9) == 0


def test_adamw_state_layout():
    sizes = [5, 0, 1024, 1025, 1, 3000]
    for bits, wide in ((32, 4), (8, 1)):
        plan = bltrain.AdamWPlan(sizes, bits=bits)
        starts, at = [], 0
        for n in sizes:
            starts.append(at)
            at += -(-n // 1024) * 1024
        assert plan.starts == starts and plan.total == at
        off = [ctypes.c_size_t() for _ in range(4)]
        assert plan._lib.bl_adamw_state_layout(plan._h, *[ctypes.byref(o) for o in off]) == 0
        scales = at // 128 * 4 if bits == 8 else 0
        assert [o.value for o in off] == [0, at * wide, 2 * at * wide, 2 * at * wide + scales]
        assert plan.state_bytes == 2 * at * wide + 2 * scales


def test_dither_is_even_and_uncorrelated():
    # the header's hash: 2^20 places, two steps.  Counts of 64 bins of 2^14 values
    # are binomial with deviation 127; means of 16 bits over 2^20 values deviate
    # by 2^16 / sqrt(12) / 2^10 = 18.5; correlations by 2^-10.  Bounds: six deviations.
    n = 1 << 20

    def words(step, seed=20):
        key = np.uint32((seed * 0x6A09E667 + step * 0xBB67AE85) & 0xFFFFFFFF)
        x = np.arange(n, dtype=np.uint32) * np.uint32(0x9E3779B9) + key
        x = (x ^ (x >> np.uint32(15))) * np.uint32(0xBB67AE85)
        return x ^ (x >> np.uint32(16))

    a, b = words(1), words(2)
    for x in (a & 0xFFFF, a >> 16, (a * np.uint32(0x6A09E667)) >> 16):
        assert np.abs(np.bincount(x >> 10, minlength=64) - n / 64).max() < 6 * 127
        assert abs(x.mean() - 32767.5) < 6 * 18.5
    centred = [x.astype(np.float64) - 32767.5 for x in (a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16)]
    for i in range(4):
        for j in range(i):
            assert abs(np.corrcoef(centred[i], centred[j])[0, 1]) < 6 / 1024
        assert abs(np.corrcoef(centred[i][1:], centred[i][:-1])[0, 1]) < 6 / 1024
