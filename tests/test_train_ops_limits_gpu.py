"""The operators around the convolution layer at the ends of their ranges (MI355X): logits
of any finite size, subnormal moments, lists of tensors and workspaces as the kernels
need them.  References and bounds are those of test_train_ops_gpu.py."""
import numpy as np
import pytest

from paper_1911_09287_amd import bltrain
from test_train_ops_gpu import (U, check_logprob, held, near, norm_bounds, norm_reference, run_norm, torch,
                                words)  # noqa: F401  (torch: the fixture)

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


@pytest.mark.parametrize("live", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 1e-50, 1e-42, 1e-20, 1e-12, 1e-8])
def test_adamw_of_subnormal_second_moments(torch, eps, bits, live):  # noqa: F811
    # gradients of 1e-19 to 1e-18: v is subnormal and sqrt(v) is not.  The step is the formula's of the fp32
    # moments, with a dozen roundings of its own and three of the parameter, as at usual sizes
    lr, b1, b2, seed, n = 3e-3, 0.9, 0.999, 5, 3000
    gen = torch.Generator().manual_seed(7)
    g = torch.exp(torch.rand(n, generator=gen) * np.log(10.0)) * 1e-19
    g = g * torch.where(torch.rand(n, generator=gen) < 0.5, -1.0, 1.0)
    if eps:  # (0 / 0 without it)
        g[::7] = 0.0
    p = (0.1 * torch.randn(n, generator=gen)).cuda()
    plan = bltrain.AdamWPlan([n], bits=bits)
    tensors, state = plan.bind([p], [g.cuda()]), plan.state()
    clock = torch.zeros(2, dtype=torch.float64, device="cuda")
    m, v = np.zeros(plan.total, np.float32), np.zeros(plan.total, np.float32)
    gn = np.zeros(plan.total, np.float32)
    gn[:n] = g.numpy()
    for t in range(1, 4):
        before = p.double().cpu().numpy()
        clock.copy_(torch.tensor([lr, t], dtype=torch.float64))
        plan.step(tensors, state, lr=lr, betas=(b1, b2), eps=eps, weight_decay=0.0, step=t, seed=seed,
                  live=clock if live else None)
        m = m * np.float32(b1) + gn * np.float32(1 - b1)
        v = v * np.float32(b2) + gn * gn * np.float32(1 - b2)
        m64, v64 = m[:n].astype(np.float64), v[:n].astype(np.float64)
        assert (v64 < 2.0 ** -126).all() and (v64[gn[:n] != 0] > 0).all()
        if bits == 8:
            w = words(plan.total, t, seed)
            m = np.copysign(held(np.abs(m), True, w & np.uint32(0xFFFF)), m)
            v = held(v, False, w >> np.uint32(16))
        up = lr / (1 - b1 ** t) * m64 / (np.sqrt(v64 / (1 - b2 ** t)) + eps)
        off = np.abs(p.double().cpu().numpy() - (before - up)) - (16 * U * np.abs(up) + 3 * U * np.abs(before) + 1e-30)
        assert off.max() <= 0, (t, off.max())


@pytest.mark.parametrize("shape", [(4, 3, 1), (4, 5, 1), (4, 50, 1), (3, 300, 1), (3, 3000, 1), (2, 40000, 1), (2, 3, 8),
                                   (2, 50, 7), (2, 1100, 3)], ids=str)
def test_norm_gradient_of_equal_values(torch, shape):  # noqa: F811
    # x and dy the same all along a row: h and dx are 0 but for the roundings of two means, times 1 / sqrt(eps).
    # Beside the bounds of other rows, which go by the exact h = 0, h's own error enters squared
    outer, size, inner = shape
    g = torch.Generator().manual_seed(size)
    x, dy = (torch.rand(outer, 1, inner, generator=g).expand(shape).contiguous() for _ in range(2))
    w, b = torch.ones(size), torch.zeros(size)
    got = run_norm(torch, shape, x, dy, w, b, "f32", "f32", 1e-5)
    x, dy, w, b = (t.double() for t in (x, dy, w, b))
    r = norm_reference(x, w, b, dy, 1e-5)
    bound = norm_bounds(x, w, b, dy, r, 1e-5, "f32", "f32")
    dh = 16 * U * x * r["rstd"]
    bound["dx"] = bound["dx"] + 2 * r["rstd"] * dh * dh * dy
    for name in ("y", "mean", "rstd", "dx"):
        near(got[name], r[name], bound[name], (shape, name))
