"""The operators around the convolution layer at the ends of their ranges (MI355X): logits
of any finite size, subnormal moments, lists of tensors and workspaces as the kernels
need them.  References and bounds are those of test_train_ops_gpu.py."""
import math

import pytest

from test_train_ops_gpu import U, check_logprob, near, torch  # noqa: F401  (torch: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [3, 200, 3000, 40000])
def test_logprob_of_finite_logits_of_any_size(torch, classes, dtype):  # noqa: F811
    g = torch.Generator().manual_seed(classes)
    rows = [torch.full((classes,), x) for x in (-1e10, -1e30, 1e20, 5e9, -1.0e38)]
    for fill in (-1e9, -1e10, -1e30, -9e37):  # half of the classes ruled out by a finite value: whole lanes and pieces
        z = torch.randn(classes, generator=g)
        z[classes // 2:] = fill
        rows.append(z)
        rows.append(z.flip(0))
    spread = torch.randn(classes, generator=g)
    rows += [x * spread for x in (1e8, 1e12, 1e30)]
    for x in (2.0 ** 20 - 2, 2.0 ** 20, 2.0 ** 20 + 2):  # where the kernel changes its form of the exponent
        rows += [x + torch.round(4 * spread) / 8, -x + torch.round(4 * spread) / 8]
    z = torch.stack(rows)
    t = torch.randint(0, classes, (len(rows),), generator=g)
    t[9] = classes - 1  # a class that a finite value rules out, and one that it leaves
    t[10] = classes - 1
    for top in (0, 5):
        check_logprob(torch, z, t, top, dtype, entropy_grad=top == 0)
