"""Retraining with residual blocks and beside a teacher, end to end on the GPU: the new operators used together."""
import subprocess
import sys

import numpy as np
import pytest
import torch
import torch.nn.functional as F

from paper_2003_06513_gb300 import distill, retrain

pytestmark = pytest.mark.gpu


def _specs(channels, seed):
    specs = retrain.pruned_net(channels, seed=seed)
    for s in specs:
        s.pool_after = s.weight.shape[0] != s.weight.shape[1] and s.weight.shape[1] > 3
    return specs


def _rms(v, w=None, b=None):
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-5)
    v = v if w is None else v * w.view(1, -1, 1, 1)
    return v if b is None else v + b.view(1, -1, 1, 1)


def _plain_logits(net, params, x):
    """The residual net in the parameters' own type with torch's elementary operators."""
    n, stream = len(net.specs), None
    act = {"none": lambda t: t, "relu": torch.relu, "silu": F.silu}[net.act]
    for i, spec in enumerate(net.specs):
        x = F.conv2d(x, params[i], stride=spec.stride, padding=1)
        if i in net.blocks:
            pw, scale, gw, gb = params[net.blocks[i]:net.blocks[i] + 4]
            gate = torch.sigmoid(x.mean((2, 3)) * gw + gb)
            stream = stream + _rms(x, pw) * (scale * gate)[:, :, None, None]
        else:
            stream = F.max_pool2d(x, 2) if spec.pool_after else x
        x = act(_rms(stream, params[n + i], params[2 * n + i]))
    return F.linear(x.mean((2, 3)), params[3 * n], params[3 * n + 1])


def _plain_loss(logits, teacher, k, labels, t, alpha):
    values, at = torch.sort(teacher, dim=1, descending=True, stable=True)
    left = torch.logsumexp(values[:, k:] / t, 1, keepdim=True)
    p = torch.log_softmax(torch.cat([values[:, :k] / t, left], 1), 1)
    q = torch.log_softmax(logits / t, 1)
    others = torch.logsumexp(q.scatter(1, at[:, :k], -np.inf), 1, keepdim=True)
    q = torch.cat([q.gather(1, at[:, :k]), others], 1)
    kl = (p.exp() * (p - q)).sum(1)
    ce = F.cross_entropy(logits, labels, reduction="none", ignore_index=-100)
    return (alpha * t * t * kl + torch.where(labels >= 0, (1 - alpha) * ce, torch.zeros_like(ce))).mean()


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("taught", [False, True])
def test_first_step_is_the_plain_one(taught, act):
    """One fp32 step against fp64 on the CPU, as for the net without blocks: norms and losses of fp32 sums of some 1e4 terms agree to
    1e-4, and the first AdamW step of a gradient g is lr g / (|g| + eps') whatever its size, so that elements are compared whose
    gradient is well above the fp32 gradients' error."""
    tf32 = torch.backends.cudnn.allow_tf32
    torch.backends.cudnn.allow_tf32 = False
    try:
        net = retrain.Retrainer(_specs((3, 24, 24, 40, 40), 1), classes=12, act=act, dtype=torch.float32, lr=1e-2, weight_decay=0.0,
                                max_norm=0.5, state_bits=32, residual=True, temperature=3.0, alpha=0.7)
        assert sorted(net.blocks) == [1, 3]
        draw = retrain.synthetic_classes(12, (3, 14, 10), "cuda", seed=2)
        x, labels = draw(6)
        teacher = torch.randn(6, 12, device="cuda", generator=torch.Generator("cuda").manual_seed(5)) * 2
        before = [p.detach().double().cpu().requires_grad_(True) for p in net.params]
        if taught:
            labels[1] = -100
            loss, total = net.step(x, labels, distill.pp_top_logits(teacher, 4, 3.0))
            ref = _plain_loss(_plain_logits(net, before, x.double().cpu()), teacher.double().cpu(), 4, labels.cpu(), 3.0, 0.7)
        else:
            loss, total = net.step(x, labels)
            ref = F.cross_entropy(_plain_logits(net, before, x.double().cpu()), labels.cpu())
        grads = list(torch.autograd.grad(ref, before))
        for i in range(len(net.specs)):
            grads[i] = grads[i] * (before[i].detach() != 0)
        norm = torch.sqrt(sum((g ** 2).sum() for g in grads))
        ref = float(ref.detach())
        assert abs(float(loss) - ref) <= 1e-4 * abs(ref) and abs(float(total) - float(norm)) <= 1e-4 * float(norm)
        scale = min(1.0, 0.5 / (float(norm) + 1e-6))
        for p, b, g in zip(net.params, before, grads):
            g = g * scale
            wanted = b.detach() - 1e-2 * g / (g.abs() + 1e-8)
            clear = g.abs() > 1e-3 * max(float(g.abs().max()), 1e-5)
            assert clear.any() and torch.all((p.detach().double().cpu() - wanted).abs()[clear] <= 1e-2 * 1e-3)
    finally:
        torch.backends.cudnn.allow_tf32 = tf32


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_the_pruned_structure_stays_and_everything_has_a_gradient(dtype):
    specs = _specs((3, 32, 32, 64, 64), 3)
    net = retrain.Retrainer(specs, classes=6, act="silu", dtype=dtype, residual=True)
    draw = retrain.synthetic_classes(6, (3, 16, 16), "cuda", seed=4)
    first = [p.detach().clone() for p in net.params]
    for _ in range(5):
        x, labels = draw(16)
        with torch.no_grad():
            top = distill.pp_top_logits(net.logits(x) + torch.randn(16, 6, device="cuda"), 3, net.temperature)
        loss, total = net.step(x, labels, top)
        assert torch.isfinite(loss) and torch.isfinite(total)
    assert all(not torch.equal(a, b) for a, b in zip(first, net.params))
    for w, spec in zip(net.weights, specs):
        assert np.array_equal(w.detach().cpu().numpy() != 0, spec.weight != 0)
    assert len(net.pack()) == len(specs)


def test_packed_layers_predict_what_the_net_does():
    """fp32 activations on both sides without TF32: scores agree to fp32 rounding of sums of some 1e3 terms, kept well below
    1e-3 of their size."""
    tf32 = torch.backends.cudnn.allow_tf32
    torch.backends.cudnn.allow_tf32 = False
    try:
        net = retrain.Retrainer(_specs((3, 32, 32, 64, 64), 5), classes=4, dtype=torch.float32, lr=3e-3, residual=True)
        draw = retrain.synthetic_classes(4, (3, 16, 16), "cuda", seed=6)
        for _ in range(5):
            net.step(*draw(16))
        x, _ = draw(16)
        with torch.no_grad():
            want = net.logits(x)
        assert (net.predict(net.pack(), x) - want).abs().max() <= 1e-3 * want.abs().max()
    finally:
        torch.backends.cudnn.allow_tf32 = tf32


def test_a_teacher_without_labels():
    net = retrain.Retrainer(retrain.pruned_net((3, 16, 32), seed=7), classes=5)
    x = torch.randn(4, 3, 12, 12, device="cuda")
    loss, _ = net.step(x, None, distill.pp_top_logits(torch.randn(4, 5, device="cuda"), 5, net.temperature))
    assert torch.isfinite(loss)


@pytest.mark.parametrize("options", [["--residual"], ["--distill"], ["--residual", "--distill"]], ids=" ".join)
def test_the_command(options):
    r = subprocess.run([sys.executable, "-m", "paper_2003_06513_gb300.retrain", "--steps", "3", "--batch", "8"] + options, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stderr
    assert "packed layers" in r.stdout and "nan" not in r.stdout
