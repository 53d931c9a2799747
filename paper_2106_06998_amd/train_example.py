"""A small image classifier trained the way the parts of this package are meant to be used together: convolutions with
estimated weight gradients (XConv2d), layer normalisation over their channels (XLayerNorm), ReLUs that keep one bit per
element (SignReLU), the convolutions' weights updated by Muon and everything else by plain SGD.

    python -m paper_2106_06998_amd.train_example [--steps 60] [--dtype f32|bf16|f16] [--channels-last]

Synthetic data: noisy copies of ten fixed patterns.  Prints the loss every ten steps, the error rate on held-out data
and the time per step."""
import argparse
import time

import torch

from .layer import SignReLU, XConv2d
from .norm import XLayerNorm
from .optim import Muon

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CLASSES, SIZE = 10, 16


class Block(torch.nn.Module):
    """convolution, normalisation over channels, ReLU"""

    def __init__(self, channels_in, channels, stride, r):
        super().__init__()
        self.conv = XConv2d(channels_in, channels, 3, r=r, stride=stride, padding=1, bias=False)
        self.norm = XLayerNorm(channels, axis=1)
        self.act = SignReLU()

    def forward(self, x):
        return self.act(self.norm(self.conv(x)))


class Net(torch.nn.Module):
    def __init__(self, width=64, r=16):
        super().__init__()
        self.stem = torch.nn.Conv2d(3, width, 3, padding=1, bias=False)
        self.blocks = torch.nn.Sequential(Block(width, width, 1, r), Block(width, 2 * width, 2, r), Block(2 * width, 2 * width, 1, r))
        self.norm = XLayerNorm(2 * width)
        self.head = torch.nn.Linear(2 * width, CLASSES)

    def forward(self, x):
        y = self.blocks(self.stem(x))
        return self.head(self.norm(y.mean(dim=(2, 3))))


def batch(n, patterns, generator, dtype, fmt):
    label = torch.randint(0, CLASSES, (n,), generator=generator, device=patterns.device)
    x = patterns[label] + 0.7 * torch.randn(n, *patterns.shape[1:], generator=generator, device=patterns.device)
    return x.to(dtype).contiguous(memory_format=fmt), label


def train(steps=60, dtype="f32", channels_last=False, batch_size=64, seed=0, device="cuda:0", report=print):
    """Returns the losses of all steps and the error rate on held-out data."""
    torch.manual_seed(seed)
    fmt = torch.channels_last if channels_last else torch.contiguous_format
    gen = torch.Generator(device=device).manual_seed(seed)
    patterns = torch.randn(CLASSES, 3, SIZE, SIZE, generator=gen, device=device)
    net = Net().to(device=device, dtype=TYPES[dtype], memory_format=fmt)
    # matrices of the hidden layers to Muon; the first and the last layer, norms and biases to SGD
    hidden = [b.conv.weight for b in net.blocks]
    others = [p for p in net.parameters() if not any(p is h for h in hidden)]
    optimisers = [Muon(hidden, lr=0.02, momentum=0.9, weight_decay=0.01), torch.optim.SGD(others, lr=0.05, momentum=0.9)]
    losses, start = [], None
    for step in range(steps):
        x, label = batch(batch_size, patterns, gen, TYPES[dtype], fmt)
        loss = torch.nn.functional.cross_entropy(net(x).float(), label)
        for o in optimisers:
            o.zero_grad()
        loss.backward()
        for o in optimisers:
            o.step()
        losses.append(loss.detach())
        if step == 4:
            torch.cuda.synchronize()
            start = time.perf_counter()
        if step % 10 == 0 or step + 1 == steps:
            report("step %3d  loss %.4f" % (step, losses[-1].item()))
    torch.cuda.synchronize()
    if steps > 5:
        report("%.2f ms per step" % ((time.perf_counter() - start) / (steps - 5) * 1e3))
    net.eval()
    with torch.no_grad():
        x, label = batch(512, patterns, gen, TYPES[dtype], fmt)
        wrong = (net(x).argmax(1) != label).float().mean().item()
    report("held-out error rate %.3f" % wrong)
    return [v.item() for v in losses], wrong


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dtype", choices=sorted(TYPES), default="f32")
    ap.add_argument("--channels-last", action="store_true")
    a = ap.parse_args()
    train(a.steps, a.dtype, a.channels_last)


if __name__ == "__main__":
    main()
