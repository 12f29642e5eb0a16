"""Masked retraining of a pattern-pruned conv net on the user's own data (§4.1: the pruned model goes
back with a masking function, and retraining updates its kept weights alone).

A ``Retrainer`` holds the net -- every 3x3 convolution followed by group norm with its activation and,
where the layer says so, a 2x2 max-pool; then the mean over the pixels and a linear classifier -- and
trains it with the framework's operators: ``norm.group_norm`` forward and backward, one gradient norm
over all parameters, one AdamW step that leaves pruned taps alone and writes the rounded weights that the
next forward pass reads.  The dense convolutions and the loss are torch's.  Nothing in a step waits
for the GPU.  ``pack`` hands the retrained weights and their pattern library to the packer, which finds the
same patterns and kernels again, and ``predict`` runs the packed layers.

With ``residual`` a layer that leaves channels and size alone is a residual block: its convolution's output joins the
stream through its norm, a gate a sample and channel (of its own mean over the pixels) and a residual scale, and the
stream's norm with the activation is what the next layer reads (``norm.block_norm``).  Beside the labels a step takes a
teacher's top logits (``distill.pp_top_logits``) -- those of the dense net that the pruned one came from -- and trains on both
(``distill.distill_loss``).

    net = Retrainer(specs, classes=10)                # specs: admm.ConvSpec with the pruned weights
    for x, labels in batches:
        top = pp_top_logits(teacher.logits(x), 10, net.temperature)         # or as stored with the batch; None: labels alone
        loss, norm = net.step(x, labels, top)
    layers = net.pack()

``python -m paper_2003_06513_gb300.retrain`` retrains a small pruned net on synthetic classes; ``--residual`` one with residual
blocks, ``--distill`` beside the dense net, which it trains and prunes first.
"""
from __future__ import annotations

import argparse
import math
from typing import List, Optional, Sequence, Tuple

import numpy as np
import torch
import torch.nn.functional as F

from . import admm, api, distill, norm, optim


class Retrainer:
    """``specs``         the pruned layers (their biases are not used: group norm takes a constant out);
    ``groups``        groups of a norm: their greatest common divisor with the layer's channels;
    ``dtype``         of activations and of the weights that the convolutions read; the weights that
                      AdamW keeps are float32;
    ``max_norm``      the gradients' norm is clipped to it;
    ``state_bits``    of AdamW's moments, 8 or 32;
    ``patterns``      the pattern library that the layers were pruned with, None for the default one: ``pack`` packs
                      with it;
    ``residual``      layers of as many input as output channels, of stride 1 and without a pool, are residual blocks;
    ``temperature, alpha``   of the loss on a teacher's logits, alpha its share beside the labels'."""

    def __init__(self, specs: Sequence[admm.ConvSpec], classes: int, groups: int = 32, act: str = "relu",
                 dtype: torch.dtype = torch.bfloat16, lr: float = 1e-3, weight_decay: float = 0.01,
                 max_norm: float = 1.0, state_bits: int = 8, seed: int = 0, device="cuda",
                 patterns: Optional[Sequence[int]] = None, residual: bool = False, temperature: float = 2.0, alpha: float = 0.5):
        self.residual, self.temperature, self.alpha = residual, temperature, alpha
        self.patterns = None if patterns is None else list(patterns)
        self.specs, self.act, self.dtype, self.max_norm = list(specs), act, dtype, max_norm
        self.weights = [torch.from_numpy(np.ascontiguousarray(s.weight, np.float32)).to(device) for s in self.specs]
        channels = [w.shape[0] for w in self.weights]
        self.groups = [math.gcd(groups, c) for c in channels]
        self.gammas = [torch.ones(c, device=device) for c in channels]
        self.betas = [torch.zeros(c, device=device) for c in channels]
        gen = torch.Generator().manual_seed(seed)
        self.head = (torch.randn(classes, channels[-1], generator=gen) / math.sqrt(channels[-1])).to(device)
        self.head_bias = torch.zeros(classes, device=device)

        n, half = len(self.specs), dtype != torch.float32
        self.params = self.weights + self.gammas + self.betas + [self.head, self.head_bias]
        # of each residual block: the weight of its output's norm, the residual scale, the gate's weight and bias
        self.blocks = {i: len(self.params) + 4 * k for k, i in enumerate(i for i in range(n) if self._is_block(i))}
        for i in self.blocks:
            c = channels[i]
            self.params += [torch.ones(c, device=device), torch.full((c,), 0.5, device=device), torch.zeros(c, device=device),
                            torch.ones(c, device=device)]
        # what the forward pass reads: the rounded weights, and the other parameters themselves
        self.copies = [w.to(dtype) for w in self.weights] if half else []
        self.leaves = (self.copies or self.weights) + self.params[n:]
        rest = len(self.params) - n
        self.optimizer = optim.AdamW(
            self.params, lr=lr, weight_decay=[weight_decay] * n + [0.0] * rest, state_bits=state_bits, seed=seed,
            taps=[optim.taps_of(w) for w in self.weights] + [None] * rest,
            grad_dtypes=[dtype] * n + [torch.float32] * rest, copies=self.copies + [None] * rest if half else None)
        for leaf in self.leaves:
            leaf.requires_grad_(True)

    def _is_block(self, i: int) -> bool:
        w, s = self.specs[i].weight, self.specs[i]
        return self.residual and i > 0 and w.shape[0] == w.shape[1] and s.stride == 1 and not s.pool_after

    def logits(self, x: torch.Tensor) -> torch.Tensor:
        """Class scores (float32) of images [N, C, H, W]."""
        n = len(self.specs)
        x = x.to(self.dtype).contiguous(memory_format=torch.channels_last)
        x = self._features(x, lambda i, t: F.conv2d(t, self.leaves[i], stride=self.specs[i].stride, padding=1), self.leaves)
        return F.linear(x.float().mean((2, 3)), self.leaves[3 * n], self.leaves[3 * n + 1])

    def _features(self, x: torch.Tensor, conv, params) -> torch.Tensor:
        """What the head reads the mean of: the layers' convolutions, conv(i, input), with all that lies between them."""
        n, stream = len(self.specs), None
        for i, spec in enumerate(self.specs):
            x = conv(i, x)
            if not self.residual:
                x = self._normed(i, x)
                continue
            x = x.contiguous(memory_format=torch.channels_last)
            if i in self.blocks:
                post_weight, scale, weight, bias = params[self.blocks[i]:self.blocks[i] + 4]
                gate = torch.sigmoid(x.float().mean((2, 3)) * weight + bias)
                stream, x = norm.block_norm(stream, x, "rms", post_weight, None, scale, gate, "rms", params[n + i], params[2 * n + i], self.act)
            else:
                stream = (F.max_pool2d(x, 2) if spec.pool_after else x).contiguous(memory_format=torch.channels_last)
                _, x = norm.block_norm(stream, None, "none", pre="rms", weight=params[n + i], bias=params[2 * n + i], act=self.act)
        return x

    def _normed(self, i: int, x: torch.Tensor) -> torch.Tensor:
        x = x.contiguous(memory_format=torch.channels_last)
        x = norm.group_norm(x, self.groups[i], self.gammas[i], self.betas[i], act=self.act)
        return F.max_pool2d(x, 2) if self.specs[i].pool_after else x

    def step(self, x: torch.Tensor, labels: Optional[torch.Tensor],
             top: Optional[distill.TopLogits] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """One step on a batch: (loss, norm of the gradients before clipping), on the device.  ``top``: a teacher's top logits for
        it, selected at the net's ``temperature`` (nothing checks that); with them ``labels`` may be None, or hold -100 where there is
        none.  The loss is the mean over all rows with a teacher, and over those that have a label (cross entropy's mean) without."""
        if top is None:
            loss = F.cross_entropy(self.logits(x), labels)
        else:
            loss = distill.distill_loss(self.logits(x), top, labels, self.temperature, self.alpha).mean()
        grads = [g.contiguous() for g in torch.autograd.grad(loss, self.leaves)]
        total, scale = self.optimizer.grad_norm(grads, self.max_norm)
        self.optimizer.step(grads, grad_scale=scale)
        return loss.detach(), total

    def pack(self) -> List[api.Layer]:
        """The retrained layers as the inference library runs them.  ValueError where the packer would prune a kept weight:
        the layer was pruned with another pattern library, or keeps more kernels than its ``keep``."""
        layers = []
        for i, (w, s) in enumerate(zip(self.weights, self.specs)):
            host = w.detach().cpu().numpy()
            layer = api.pp_pack(host, self.patterns, s.keep, 1, s.stride)
            if not np.array_equal(layer.export("dense").reshape(host.shape), host):
                raise ValueError(f"layer {i} is not inside its constraints: `patterns` must be the library it was pruned with, "
                                 "`keep` at least the kernels it has")
            layers.append(layer.bind(w.device))
        return layers

    @torch.no_grad()
    def predict(self, layers: Sequence[api.Layer], x: torch.Tensor) -> torch.Tensor:
        """Class scores with the packed layers, float32 throughout."""
        x = self._features(x.float(), lambda i, t: layers[i].conv(t.contiguous(), torch.zeros_like(self.betas[i]), False), self.params)
        return F.linear(x.mean((2, 3)), self.head, self.head_bias)


def pruned_net(channels: Sequence[int] = (3, 64, 128, 128), keep: float = 0.4, seed: int = 0) -> List[admm.ConvSpec]:
    """A small random net inside the pattern and connectivity constraints; the first layer keeps all kernels."""
    rng = np.random.default_rng(seed)
    specs = []
    for i, (cin, cout) in enumerate(zip(channels, channels[1:])):
        k = 1.0 if i == 0 else keep
        w = (rng.standard_normal((cout, cin, 3, 3)) * math.sqrt(2.0 / (9 * cin))).astype(np.float32)
        specs.append(admm.ConvSpec(admm.project(w, None, k), np.zeros(cout, np.float32), pool_after=i > 0, keep=k))
    return specs


def synthetic_classes(classes: int, image: Sequence[int], device, seed: int = 0):
    """A function that draws (images, labels): a class is a grating of its own frequency and colours, which
    comes at a random phase and under noise."""
    c, h, w = image
    gen = torch.Generator(device=device).manual_seed(seed)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device=device)
    wave, colour = (uniform(classes, 2) * 2 - 1) * 2.5, uniform(classes, c) * 2 - 1
    rows, cols = torch.arange(h, device=device)[:, None], torch.arange(w, device=device)

    def draw(n: int):
        labels = torch.randint(0, classes, (n,), generator=gen, device=device)
        at = wave[labels].view(n, 2, 1, 1)
        grating = torch.cos(at[:, 0] * rows + at[:, 1] * cols + 2 * math.pi * uniform(n, 1, 1))
        noise = torch.randn(n, c, h, w, generator=gen, device=device)
        return grating[:, None] * colour[labels].view(n, c, 1, 1) + 0.25 * noise, labels
    return draw


def dense_net(channels: Sequence[int] = (3, 64, 128, 128), seed: int = 0) -> List[admm.ConvSpec]:
    """The same net before anything is pruned."""
    rng = np.random.default_rng(seed)
    return [admm.ConvSpec((rng.standard_normal((cout, cin, 3, 3)) * math.sqrt(2.0 / (9 * cin))).astype(np.float32), np.zeros(cout, np.float32),
                          pool_after=i > 0 and cin != cout) for i, (cin, cout) in enumerate(zip(channels, channels[1:]))]


def pruned_from(net: Retrainer, keep: float = 0.4) -> List[admm.ConvSpec]:
    """A trained net's layers inside the pattern and connectivity constraints; the first one keeps all kernels."""
    specs = []
    for i, (w, spec) in enumerate(zip(net.weights, net.specs)):
        k = 1.0 if i == 0 else keep
        specs.append(admm.ConvSpec(admm.project(w.detach().cpu().numpy(), net.patterns, k, spec.stride), spec.bias, spec.stride,
                                   spec.pool_after, k))
    return specs


def main() -> None:
    ap = argparse.ArgumentParser(description="retrain a small pruned net on synthetic classes")
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    ap.add_argument("--residual", action="store_true", help="a net with residual blocks")
    ap.add_argument("--distill", action="store_true", help="train a dense net first, prune it, and retrain beside its top logits")
    args = ap.parse_args()
    draw = synthetic_classes(10, (3, 32, 32), "cuda")
    options = dict(classes=10, act="silu", state_bits=args.state_bits, residual=args.residual)
    channels = (3, 64, 64, 64, 128, 128) if args.residual else (3, 64, 128, 128)

    def train(net, what, teacher=None):
        for i in range(args.steps):
            x, labels = draw(args.batch)
            top = None
            if teacher is not None:
                with torch.no_grad():
                    top = distill.pp_top_logits(teacher.logits(x), 4, net.temperature)
            loss, total = net.step(x, labels, top)
            if i % 10 == 0 or i == args.steps - 1:
                print(f"{what}step {i}: loss {float(loss.detach()):.4f}, gradient norm {float(total):.4f}")

    teacher = None
    if args.distill:
        teacher = Retrainer(dense_net(channels), **options)
        train(teacher, "dense net, ")
        net = Retrainer(pruned_from(teacher), **options)
    else:
        specs = pruned_net(channels)
        for spec in specs if args.residual else ():
            spec.pool_after = spec.weight.shape[0] != spec.weight.shape[1] and spec.weight.shape[1] > 3
        net = Retrainer(specs, **options)
    train(net, "", teacher)
    x, labels = draw(256)
    right = (net.predict(net.pack(), x).argmax(1) == labels).float().mean()
    print(f"packed layers: {float(right):.3f} of 256 new images right")


if __name__ == "__main__":
    main()
