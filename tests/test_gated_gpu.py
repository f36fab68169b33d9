"""The gated recurrent classifier: a run of the library's operators together, its gradients against
those of the whole network in 64 bits, and its command (MI355X)."""
import pytest

from paper_1911_09287_amd import gated
from paper_1911_09287_amd.series import same, waves
from test_train_ops_gpu import torch  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def reference(t, net, series, labels):
    """Loss and gradients of the network in 64 bits, by autograd of its definition (on the host)."""
    matrices = [p.double().cpu().requires_grad_() for p in net.matrices]
    vectors = [p.double().cpu().requires_grad_() for p in net.vectors]
    filters, gates, values, classifier = matrices
    w1, b1, w2, b2, gate_bias, class_bias = vectors

    def norm(v, w, b):
        return t.nn.functional.group_norm(v, 8, w, b, 1e-5)
    lo, hi = same(gated.TAPS)
    v = t.nn.functional.conv1d(t.nn.functional.pad(series.double().cpu(), (lo, hi)), filters.unsqueeze(1))
    v = norm(v, w1, b1)
    v = v * v.sigmoid()
    gate, x = gates @ v + gate_bias.view(1, -1, 1), values @ v
    a, h, hs = gate.sigmoid(), t.zeros_like(x[..., 0]), []
    for k in range(x.shape[2]):
        h = a[..., k] * h + (1 - a[..., k]) * x[..., k]
        hs.append(h)
    z = norm(t.stack(hs, 2), w2, b2).mean(2)
    logp = (z @ classifier + class_bias).log_softmax(1)
    loss = -logp.gather(1, labels.cpu().unsqueeze(1)).mean()
    loss.backward()
    return loss.item(), [p.grad for p in matrices], [p.grad for p in vectors]


def test_gradients_of_the_whole_network(torch):
    net = gated.GatedNet(6, 90, 5, channels=48, seed=3)
    series, labels = waves(6, 90, 5, 4)
    logp = net.backward(net.forward(series), labels)
    loss, matrices, vectors = reference(torch, net, series, labels)
    # ten operators of some 100 roundings of 2^-24 each in the worst order; torch's fp32 products among them
    assert abs(-logp.mean().item() - loss) < 1e-4 * (1 + abs(loss))
    for got, want in zip(net.dmatrices + net.dvectors, matrices + vectors):
        off = (got.double().cpu() - want).norm().item()
        assert off <= 1e-3 * want.norm().item() + 1e-7, (tuple(want.shape), off, want.norm().item())


def test_steps_move_all_parameters_and_stay_finite(torch):
    net = gated.GatedNet(8, 64, 4, channels=32, rate=0.5)
    before = [p.clone() for p in net.matrices + net.vectors]
    for step in range(3):
        net.train(*waves(8, 64, 4, step))
    for p, q in zip(net.matrices + net.vectors, before):
        assert p.isfinite().all() and (p != q).any()


def test_a_captured_step_is_the_eager_one(torch):
    nets = [gated.GatedNet(8, 64, 4, channels=32, rate=0.5, seed=5) for _ in range(2)]
    series, labels = waves(8, 64, 4, 7)
    # (an eager pass first: it makes the convolution's tables)
    for net in nets:
        net.backward(net.forward(series), labels)
    net = nets[1]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.backward(net.forward(series), labels)
        net.muon.orthogonalize(net.muon.bind([torch.empty_like(p) for p in net.matrices], net.dmatrices), net.muon_ws)
    for _ in range(3):
        for p in net.dmatrices + net.dvectors:
            p.fill_(float("nan"))
        graph.replay()
        nets[0].backward(nets[0].forward(series), labels)
        torch.cuda.synchronize()
        for p, q in zip(net.dmatrices, nets[0].dmatrices):
            # (torch's products may take another order of sums where they are captured)
            assert (p - q).norm() <= 1e-4 * q.norm()


def test_command(torch, capsys):
    gated.main(["--steps", "2", "--batch", "8", "--length", "64", "--classes", "4"])
    out = capsys.readouterr().out
    assert "step    1" in out and "held out: accuracy" in out
