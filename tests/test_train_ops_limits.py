"""The operators around the convolution layer at the ends of their ranges, on the host (CPU
only, no GPU calls): what the bindings and the plans have to refuse."""
import os

import pytest
import torch

from paper_1911_09287_amd import blconv, bltrain

pytestmark = pytest.mark.skipif(not os.path.exists(blconv.LIB_PATH), reason="libblconv.so not built")


class Placed(torch.Tensor):
    """A tensor of the host that says it lies on GPU 0, for checks that come before any launch."""

    is_cuda = True

    def get_device(self):
        return 0


def placed(t):
    return t.as_subclass(Placed)


def test_workspaces_that_are_not_contiguous_are_refused():
    # an expanded tensor has as many bytes as it says, and its storage one
    norm, prob = bltrain.NormPlan(2, 100000), bltrain.LogProbPlan(2, 100000)
    conv = blconv.Plan(1, 2, 1, 2, (16,), 3, (1, 1), 0.0)
    x, stats = placed(torch.zeros(2, 100000)), placed(torch.zeros(2, 2, 1))
    w = placed(torch.zeros(100000))
    for plan in (norm, prob, conv):
        assert plan._ws(placed(torch.zeros(plan.workspace_bytes, dtype=torch.uint8)))
        for ws in (placed(torch.zeros(1, dtype=torch.uint8)).expand(plan.workspace_bytes),
                   placed(torch.zeros(2 * plan.workspace_bytes, dtype=torch.uint8))[::2]):
            with pytest.raises(ValueError):
                plan._ws(ws)
    ws = placed(torch.zeros(1, dtype=torch.uint8)).expand(norm.workspace_bytes)
    with pytest.raises(ValueError):
        norm.forward(x, None, None, x, stats, ws)
    with pytest.raises(ValueError):
        norm.backward(x, x, None, stats, x, w, w, ws)
    ws = placed(torch.zeros(1, dtype=torch.uint8)).expand(prob.workspace_bytes)
    with pytest.raises(ValueError):
        prob.forward(x, None, None, None, None, None, ws)
