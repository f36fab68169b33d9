"""Group norm, recurrence and orthogonalised update: roundings that add up over many samples, many steps
or far values (MI355X).  U = 2^-24; each test says where its tolerance comes from.
"""
import pytest

from paper_1911_09287_amd import bltrain
from test_group_norm_gpu import bounds as norm_bounds, inputs as norm_inputs, reference as norm_reference
from test_muon_gpu import USUAL, gradient
from test_recurrence_gpu import inputs as steps_inputs, reference as steps_reference, run as steps_run
from test_train_ops_gpu import U, half_ulp, near, tdtype, torch  # noqa: F401  (torch: the fixture)

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


# (batch, sites, channels, groups): groups that a block keeps, and in the last two shapes parts of them
MANY = [(20000, 1, 64, 8), (20000, 3, 24, 3), (100000, 1, 3, 1), (5000, 2, 1030, 10), (513, 4, 70, 7), (700, 2600, 8, 1),
        (4200, 2600, 8, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("last", [True, False])
@pytest.mark.parametrize("shape", MANY)
def test_weight_gradients_of_many_samples(torch, shape, last, dtype):  # noqa: F811
    # Samples alike: a sum of one value many times, which rounds the same way for long stretches.  The gradients are
    # those of one sample times their number, and so are the bounds of group norm's own tests, which take 16 U for
    # every sum: trees of 16 rows (4), at most 16 of them in a slab's slice, six halvings, and the same over slabs.
    batch, sites, channels, groups = shape
    x, dy, w, b = norm_inputs(torch, (1, sites, channels, groups), last, dtype, "f32", 31)
    dy = (dy * 0.1 + 0.3).to(tdtype(torch, dtype))
    plan = bltrain.GroupNormPlan(batch, sites, channels, groups, channels_last=last, dtype=tdtype(torch, dtype))
    xs, dys, wd, bd = x.cuda().repeat(batch, 1, 1), dy.cuda().repeat(batch, 1, 1), w.cuda(), b.cuda()
    y, stats, dx = torch.empty_like(xs), torch.empty(plan.stats_shape(), device="cuda"), torch.full_like(xs, float("nan"))
    dw, db = (torch.full((channels,), float("nan"), device="cuda") for _ in range(2))
    ws = plan.workspace()
    plan.forward(xs, wd, bd, y, stats, ws)
    ws.fill_(255)
    plan.backward(dys, xs, wd, bd, stats, dx, dw, db, ws)
    x, dy, w, b = (v.double() for v in (x, dy, w, b))
    r = norm_reference(torch, x, w, b, dy, groups, last, None, 1e-5)
    most = norm_bounds(x, dy, r, groups, last, None, dtype, "f32")
    assert (dx == dx[:1]).all()
    near(dx[:1], r["dx"], most["dx"], "dx")
    near(dw, batch * r["dw"], batch * most["dw"], "dw")
    near(db, batch * r["db"], batch * most["db"], "db")


# (parts of samples that many blocks take, long channels side by side, a sample's 512 slices of one block, and
# one sample's 2048 parts)
@pytest.mark.parametrize("shape,last", [((1024, 3136, 256, 32), True), ((64, 50176, 64, 8), False), ((300, 2048, 4, 1), True),
                                        ((1, 1 << 20, 65, 1), True)])
def test_bias_gradients_of_many_sites(torch, shape, last):  # noqa: F811
    # One gradient at every site: a sum of one value, which rounds the same way for long stretches where it is a
    # chain.  16 U for a sum in few levels, as group norm's own tests take it, and U for the value itself.
    batch, sites, channels, groups = shape
    x, _, w, b = norm_inputs(torch, (1, sites, channels, groups), last, "f32", "f32", 32)
    plan = bltrain.GroupNormPlan(batch, sites, channels, groups, channels_last=last)
    xs, wd, bd = x.cuda().repeat(batch, 1, 1), w.cuda(), b.cuda()
    dys = torch.full_like(xs, 0.3)
    stats, dw, db = torch.empty(plan.stats_shape(), device="cuda"), torch.empty_like(wd), torch.empty_like(bd)
    y, ws = torch.empty_like(xs), plan.workspace()
    plan.forward(xs, wd, bd, y, stats, ws)
    plan.backward(dys, xs, wd, bd, stats, y, dw, db, ws)
    want = torch.full((channels,), 0.3).double() * (batch * sites)
    near(db, want, 17 * U * want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("length", [1, 5, 8])
def test_gates_whose_exponential_overflows(torch, length, dtype):  # noqa: F811
    # exp(g) is infinite in fp32 for all but the last two, which 3 e^87 stays below the largest number for, and so
    # is the state from then on
    gates = torch.tensor([float("inf"), 3.3e38, 89.0, 93.5, 100.0, 127.0, 1000.0, 87.0, 86.5])
    n = len(gates)
    gate, x = torch.full((2, length, n), -0.5), torch.ones(2, length, n)
    gate[:, -1] = gates
    h0 = torch.ones(2, n, device="cuda")
    plan = bltrain.RecurrencePlan(2, length, n, gate="exp", dtype=tdtype(torch, dtype))
    y = torch.full((2, length, n), float("nan"), dtype=tdtype(torch, dtype), device="cuda")
    last = torch.full_like(h0, float("nan"))
    plan.forward(gate.to(y.dtype).cuda(), x.to(y.dtype).cuda(), y, plan.workspace(), h0=h0, last=last)
    h = torch.ones(2, n, dtype=torch.float64)
    for t in range(length):
        a = gate[:, t].to(y.dtype).double().exp()
        h = h * a.masked_fill(a >= 2.0 ** 128, float("inf")) + 1.0
    assert (last[:, :7] == float("inf")).all() and (y[:, -1, :7] == float("inf")).all()
    # an exponential of two units, a product and a sum for each step
    near(last[:, 7:], h[:, 7:], 6 * U * length * h[:, 7:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 7, 20), (2, 300, 20), (1, 6000, 24), (300, 300, 1), (3, 300, 1), (2, 300, 3), (1, 9000, 3)])
@pytest.mark.parametrize("how", ["grows", "wanders"])
def test_states_that_grow(torch, how, shape, dtype):  # noqa: F811
    # gates above 0 whose sum stays below 88 over all steps (in bfloat16 with room for its largest values too): by
    # 60 steadily, or a few up and down
    v = steps_inputs(torch, shape, "exp", dtype, 33, False)
    g = torch.Generator().manual_seed(34)
    if how == "grows":
        gate = torch.rand(shape, generator=g) * (120.0 / shape[1])
    else:
        gate = torch.randn(shape, generator=g) * min(1.0, 6.0 / shape[1] ** 0.5)
    v["gate"] = gate.to(tdtype(torch, dtype))
    sums = v["gate"].double().cumsum(1)
    assert (sums.amax(1) - sums.amin(1)).max() < 80
    got = steps_run(torch, shape, "exp", dtype, v)
    r, most = steps_reference(torch, *(v[k].double() for k in ("gate", "x", "h0", "dy", "dlast")), None, "exp")
    for name in got:
        bound = most[name]
        if name in ("y", "dgate", "dx"):
            bound = bound + half_ulp(dtype) * (r[name].abs() + bound) + 1e-30
        near(got[name], r[name], bound, f"{name} {shape} {how}")


@pytest.mark.parametrize("last", [True, False])
def test_silu_far_below_zero(torch, last):  # noqa: F811
    # Groups of one value, whose z is the bias to the last bit: the activation and its slope q (1 + z (1 - q)) alone.
    # q is an exponential of two units (4 U), a sum, a reciprocal of one (2 U) and a product, z q one more: 9 U; the
    # slope has 9 U of both its terms and three roundings of them.  Where z is below -87.3 both are 0.
    z = torch.cat([torch.linspace(-87.2, 30.0, 4001), torch.tensor([-90.0, -1000.0, -3e38, 3e37])])
    n = len(z)
    plan = bltrain.GroupNormPlan(1, 1, n, n, channels_last=last, act="silu")
    x = torch.randn(1, n, generator=torch.Generator().manual_seed(35)).cuda()
    y, dx, stats = torch.full_like(x, float("nan")), torch.full_like(x, float("nan")), torch.empty(2, 1, n, device="cuda")
    w, b, dw, db = torch.ones(n, device="cuda"), z.cuda(), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ws = plan.workspace()
    plan.forward(x, w, b, y, stats, ws)
    plan.backward(torch.ones_like(x), x, w, b, stats, dx, dw, db, ws)
    z = z.double()
    q = z.sigmoid() * (z > -87.3)
    near(y[0], z * q, 10 * U * (z * q).abs())
    near(db, q + z * q * (-z).sigmoid(), 12 * U * (q + (z * q * (-z).sigmoid()).abs()))
    assert (dx == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("eps", [1e-300, 1e-308, 5e-324])
def test_zeros_stay_whatever_eps_is(torch, eps):  # noqa: F811
    # 1 / eps leaves 64 bits; both kernels that lay matrices out, and values beside the smallest there are
    for shapes in ([(5, 7), (7, 5)], [(70, 90), (5, 7), (7, 5)]):
        us = [torch.zeros(s) for s in shapes]
        us[-1] = torch.full(shapes[-1], 2.0 ** -149)
        plan = bltrain.MuonPlan(shapes)
        outs = [torch.full(s, float("nan"), device="cuda") for s in shapes]
        plan.orthogonalize(plan.bind(outs, [u.cuda() for u in us]), plan.workspace(), eps=eps)
        for out in outs[:-1]:
            assert (out == 0).all()
        assert outs[-1].isfinite().all() and (outs[-1] > 0).all()
