"""Group norm, recurrence and orthogonalised update: roundings that add up over many samples, many steps
or far values (MI355X).  U = 2^-24; each test says where its tolerance comes from.
"""
import pytest

from paper_1911_09287_amd import bltrain
from test_muon_gpu import USUAL, gradient
from test_train_ops_gpu import U, torch  # noqa: F401  (torch: the fixture)

pytestmark = pytest.mark.gpu


def steps_of(t, u, coefficients, runs, dtype):
    """X of u, its steps joined in runs of so many: X = (... B2 B1) X with the next step's A = B (A B), the
    square matrices kept symmetric."""
    def kept(a):
        return a.tril() + a.tril(-1).t()
    x = (u.double() / u.double().norm()).to(dtype)
    at = 0
    for run in runs:
        gram, product = kept(x @ x.t()), None
        for k in range(run):
            a, b, c = coefficients[at]
            poly = kept(b * gram + c * (gram @ gram))
            poly.diagonal().add_(a)
            product = poly if product is None else kept(poly @ product)
            if k + 1 < run:
                gram = kept(poly @ kept(poly @ gram))
            at += 1
        x = product @ x
    return x


# (one block a matrix; one tile on the diagonal; tiles on and off it)
@pytest.mark.parametrize("shape", [(50, 128), (64, 640), (31, 900), (64, 1100), (40, 2000), (100, 1500), (128, 768)])
@pytest.mark.parametrize("runs", [(3,), (3, 2)])
def test_joined_steps_keep_what_fp32_keeps(torch, shape, runs):  # noqa: F811
    # The same steps in fp32 are the measure.  They round every operand and every sum at U of itself; two fp16
    # parts round an operand at 4 U and leave 4 U of a product out, sums in fp32 as they do: no rounding is more
    # than 6 times one of fp32's at the same place, and errors in the Frobenius norm are sums of those squared.
    u = gradient(torch, shape, 21, few=8)
    coefficients = USUAL[:sum(runs)]
    want = steps_of(torch, u, coefficients, (1,) * len(coefficients), torch.float64)
    fp32 = (steps_of(torch, u, coefficients, runs, torch.float32).double() - want).norm().item()
    plan = bltrain.MuonPlan([shape], coefficients=coefficients)
    out = torch.full(shape, float("nan"), device="cuda")
    plan.orthogonalize(plan.bind([out], [u.cuda()]), plan.workspace(), eps=1e-30)
    off = (out.double().cpu() - want).norm().item()
    assert off <= 6 * fp32 + U * want.norm().item(), (shape, off, fp32, want.norm().item())
