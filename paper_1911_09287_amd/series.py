"""Training a time-series classifier with the library's convolutions, norms, loss and step.

The three-layer fully convolutional network of the time-series workload: band-limited
convolutions (8, 5 and 3 taps), each followed by a layer norm over the channels at
every sample and a ReLU, the mean over time, a linear classifier, the log probability
of the right class and an AdamW step.  Convolutions, norms, log probabilities and the
step are this package's calls; torch adds the ReLU, the mean and the classifier's small
products.

    python -m paper_1911_09287_amd.series --steps 200 --rate 0.5 --bits 8
"""
from __future__ import annotations

import argparse
import math

import torch

from . import blconv, bltrain

TAPS = (8, 5, 3)


def same(taps):
    lo = (taps - 1) // 2
    return lo, taps - 1 - lo


class SeriesNet:
    """The network's parameters, gradients, plans and buffers for batches [batch][1][length]."""

    def __init__(self, batch, length, classes, channels=(128, 256, 128), rate=0.0, bits=32, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.batch, self.length, self.classes = batch, length, classes
        self.convs, self.norms, shapes, decay = [], [], [], []
        c_in = 1
        for c_out, taps in zip(channels, TAPS):
            self.convs.append(blconv.Plan(1, batch, c_in, c_out, (length,), taps, same(taps), rate))
            self.norms.append(bltrain.NormPlan(batch, c_out, length))
            shapes += [(c_out, c_in, taps), (c_out,), (c_out,)]  # filters, the norm's weight and bias
            decay += [True, False, False]
            c_in = c_out
        shapes += [(c_in, classes), (classes,)]
        decay += [True, False]
        self.params = []
        for shape in shapes:
            scale = math.sqrt(2.0 / math.prod(shape[1:])) if len(shape) == 3 else math.sqrt(1.0 / shape[0])
            self.params.append(torch.randn(shape, generator=g, device=device) * scale if len(shape) > 1
                               else torch.zeros(shape, device=device))
        for i in range(len(self.convs)):
            self.params[3 * i + 1].fill_(1.0)
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.loss = bltrain.LogProbPlan(batch, classes)
        self.adam = bltrain.AdamWPlan([p.numel() for p in self.params], bits=bits, decay=decay)
        self.state, self.steps = self.adam.state(device), 0
        self.tensors = self.adam.bind(self.params, self.grads)

        def empty(*shape):
            return torch.empty(*shape, device=device)
        self.conv_ws = [p.workspace(device) for p in self.convs]
        self.norm_ws = [p.workspace(device) for p in self.norms]
        self.loss_ws = self.loss.workspace(device)
        self.maps = [empty(p.y_shape()) for p in self.convs]       # the convolutions' outputs
        self.normed = [torch.empty_like(t) for t in self.maps]
        self.stats = [empty(p.stats_shape()) for p in self.norms]
        self.dmaps = [torch.empty_like(t) for t in self.maps]
        self.dinputs = [empty(p.x_shape()) for p in self.convs]
        self.logp, self.row_stats = empty(batch), empty(3, batch)
        self.g_logp = torch.full((batch,), -1.0 / batch, device=device)  # of the mean negative log probability
        self.dlogits = empty(batch, classes)

    def forward(self, x):
        """Logits [batch][classes]; leaves what backward() needs."""
        a = x
        for i, (conv, norm) in enumerate(zip(self.convs, self.norms)):
            conv.forward(a, self.params[3 * i], self.maps[i], self.conv_ws[i])
            norm.forward(self.maps[i], self.params[3 * i + 1], self.params[3 * i + 2], self.normed[i], self.stats[i],
                         self.norm_ws[i])
            a = self.normed[i].relu_()
        self.features = a.mean(2)
        return torch.addmm(self.params[-1], self.features, self.params[-2])

    def backward(self, logits, labels):
        """The gradients of the mean negative log probability of the labels; returns log probabilities."""
        self.loss.forward(logits, labels, self.logp, self.row_stats, None, None, self.loss_ws)
        self.loss.backward(logits, labels, self.row_stats, self.g_logp, None, self.dlogits)
        torch.mm(self.features.t(), self.dlogits, out=self.grads[-2])
        self.grads[-1].copy_(self.dlogits.sum(0))
        da = (self.dlogits @ self.params[-2].t()).unsqueeze(2).expand_as(self.normed[-1]) / self.length
        for i in reversed(range(len(self.convs))):
            dy = da * (self.normed[i] > 0)
            self.norms[i].backward(dy, self.maps[i], self.params[3 * i + 1], self.stats[i], self.dmaps[i],
                                   self.grads[3 * i + 1], self.grads[3 * i + 2], self.norm_ws[i])
            # the spectra of the layer's input and filters are those that the forward pass left
            self.convs[i].backward(self.dmaps[i], None, None, self.dinputs[i], self.grads[3 * i], self.conv_ws[i],
                                   flags=blconv.BL_REUSE_W | blconv.BL_REUSE_X)
            da = self.dinputs[i]
        return self.logp

    def step(self, lr=1e-3, weight_decay=1e-2):
        self.steps += 1
        self.adam.step(self.tensors, self.state, lr=lr, weight_decay=weight_decay, step=self.steps, seed=1)

    def train(self, x, labels, lr=1e-3):
        """One training step; returns the mean negative log probability before it."""
        logp = self.backward(self.forward(x), labels)
        loss = -logp.mean()
        self.step(lr)
        return loss

    def answer(self, x, top=3):
        """Each series' `top` likeliest classes and their log probabilities, and the entropies."""
        plan = bltrain.LogProbPlan(self.batch, self.classes, top=top)
        logp = torch.empty(self.batch, top, device=x.device)
        index = torch.empty(self.batch, top, dtype=torch.int64, device=x.device)
        stats = torch.empty(3, self.batch, device=x.device)
        plan.forward(self.forward(x), None, None, stats, logp, index, plan.workspace(x.device))
        return index, logp, stats[2]


def waves(batch, length, classes, seed, device="cuda"):
    """Series of a wave whose frequency its class sets, with a phase, a trend and noise: (x, labels)."""
    g = torch.Generator(device=device).manual_seed(seed)
    labels = torch.randint(0, classes, (batch,), generator=g, device=device)
    t = torch.arange(length, device=device) / length
    phase = torch.rand(batch, 1, generator=g, device=device)
    trend = torch.randn(batch, 1, generator=g, device=device)
    x = torch.sin(2.0 * math.pi * ((2.0 + 3.0 * labels.unsqueeze(1)) * t + phase)) + trend * t
    x = x + 0.5 * torch.randn(batch, length, generator=g, device=device)
    return ((x - x.mean(1, keepdim=True)) / x.std(1, keepdim=True)).unsqueeze(1).contiguous(), labels


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--length", type=int, default=512)
    ap.add_argument("--classes", type=int, default=10)
    ap.add_argument("--rate", type=float, default=0.5, help="compression rate of the convolutions")
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32), help="bits of AdamW's moments")
    ap.add_argument("--lr", type=float, default=2e-3)
    a = ap.parse_args(argv)
    net = SeriesNet(a.batch, a.length, a.classes, rate=a.rate, bits=a.bits)
    for step in range(a.steps):
        loss = net.train(*waves(a.batch, a.length, a.classes, step), a.lr)
        if step % 20 == 0 or step == a.steps - 1:
            print(f"step {step:4d}  loss {loss.item():.4f}", flush=True)
    x, labels = waves(a.batch, a.length, a.classes, 10 ** 6)
    index, logp, entropy = net.answer(x, min(3, a.classes))
    print(f"held out: accuracy {(index[:, 0] == labels).float().mean().item():.3f}, "
          f"mean entropy {entropy.mean().item():.3f}")


if __name__ == "__main__":
    main()
