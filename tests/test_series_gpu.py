"""The series classifier trained from the library's operators (MI355X): its gradients
against torch's own in 64 bits, and a training run that learns."""
import pytest

from paper_1911_09287_amd import blconv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as _torch
    if not _torch.cuda.is_available():
        pytest.skip("no GPU")
    blconv.load()
    return _torch


def test_gradients_against_autograd_in_64_bits(torch):
    # at rate 0 the band-limited layer is the plain correlation
    from paper_1911_09287_amd import series
    net = series.SeriesNet(6, 40, 5, channels=(8, 12, 8), rate=0.0)
    x, labels = series.waves(6, 40, 5, 3)
    logits = net.forward(x)
    logp = net.backward(logits, labels)
    params = [p.double().cpu().requires_grad_() for p in net.params]
    a = x.double().cpu()
    for i, taps in enumerate(series.TAPS):
        a = torch.nn.functional.conv1d(torch.nn.functional.pad(a, series.same(taps)), params[3 * i])
        a = torch.nn.functional.layer_norm(a.transpose(1, 2), (a.shape[1],), params[3 * i + 1], params[3 * i + 2], 1e-5)
        a = a.transpose(1, 2).relu()
    want = (a.mean(2) @ params[-2] + params[-1]).log_softmax(1)[torch.arange(6), labels.cpu()]
    (-want.mean()).backward()
    # the layers' own parity bar is 1e-4 relative; three of them and the norms between
    assert (logp.double().cpu() - want.detach()).abs().max().item() < 1e-4
    for i, (g, p) in enumerate(zip(net.grads, params)):
        err = (g.double().cpu() - p.grad).norm() / p.grad.norm()
        assert err.item() < 1e-3, (i, err.item())


@pytest.mark.parametrize("rate,bits", [(0.0, 32), (0.5, 8)])
def test_training_learns(torch, rate, bits):
    from paper_1911_09287_amd import series
    net = series.SeriesNet(32, 128, 4, channels=(32, 48, 32), rate=rate, bits=bits)
    losses = [net.train(*series.waves(32, 128, 4, step), 3e-3).item() for step in range(60)]
    assert sum(losses[-5:]) < 0.5 * sum(losses[:5])
    x, labels = series.waves(32, 128, 4, 10 ** 6)
    index, logp, entropy = net.answer(x, 2)
    assert (index[:, 0] == labels).float().mean().item() > 0.6
    assert (logp[:, 0] >= logp[:, 1]).all() and (entropy >= 0).all()
