"""Masked retraining end to end on the GPU: the operators of the training side used together."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from paper_2003_06513_gb300 import admm, retrain

pytestmark = pytest.mark.gpu


def _plain_loss(net, params, x, labels):
    """The net in the parameters' own type with torch's operators."""
    n = len(net.specs)
    for i, spec in enumerate(net.specs):
        x = F.conv2d(x, params[i], stride=spec.stride, padding=1)
        x = F.group_norm(x, net.groups[i], params[n + i], params[2 * n + i], 1e-5)
        x = {"none": lambda t: t, "relu": torch.relu, "silu": F.silu}[net.act](x)
        x = F.max_pool2d(x, 2) if spec.pool_after else x
    return F.cross_entropy(F.linear(x.mean((2, 3)), params[3 * n], params[3 * n + 1]), labels)


@pytest.mark.parametrize("act", ["relu", "silu"])
def test_first_step_is_the_plain_one(act):
    """One fp32 step against fp64 on the CPU.  The first AdamW step of a gradient g is lr g / (|g| + eps') whatever
    its size, so that an element's step differs by eps / |g| of it at most where |g| is well above the fp32
    gradients' error; elements whose gradient is within 1e-3 of the largest are compared.  Norms and losses of
    fp32 sums of some 1e4 terms: 1e-4."""
    tf32 = torch.backends.cudnn.allow_tf32
    torch.backends.cudnn.allow_tf32 = False
    try:
        specs = retrain.pruned_net((3, 24, 40), seed=1)
        net = retrain.Retrainer(specs, classes=5, groups=8, act=act, dtype=torch.float32, lr=1e-2, weight_decay=0.0,
                                max_norm=0.5, state_bits=32)
        draw = retrain.synthetic_classes(5, (3, 13, 11), "cuda", seed=2)
        x, labels = draw(6)
        before = [p.detach().double().cpu().requires_grad_(True) for p in net.params]
        loss, total = net.step(x, labels)
        ref = _plain_loss(net, before, x.double().cpu(), labels.cpu())
        grads = list(torch.autograd.grad(ref, before))
        for i in range(len(specs)):
            grads[i] = grads[i] * (before[i].detach() != 0)
        norm = torch.sqrt(sum((g ** 2).sum() for g in grads))
        assert abs(float(loss) - float(ref)) <= 1e-4 * abs(float(ref))
        assert abs(float(total) - float(norm)) <= 1e-4 * float(norm)
        scale = min(1.0, 0.5 / (float(norm) + 1e-6))
        for p, b, g in zip(net.params, before, grads):
            g = g * scale
            wanted = b.detach() - 1e-2 * g / (g.abs() + 1e-8)
            clear = g.abs() > 1e-3 * max(float(g.abs().max()), 1e-5)
            assert torch.all((p.detach().double().cpu() - wanted).abs()[clear] <= 1e-2 * 1e-3)
            assert clear.any()
    finally:
        torch.backends.cudnn.allow_tf32 = tf32


@pytest.mark.parametrize("state_bits", [8, 32])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_retraining_learns_and_keeps_the_pruned_structure(dtype, state_bits):
    specs = retrain.pruned_net((3, 32, 64), seed=3)
    net = retrain.Retrainer(specs, classes=4, act="silu", dtype=dtype, lr=3e-3, state_bits=state_bits)
    draw = retrain.synthetic_classes(4, (3, 16, 16), "cuda", seed=4)
    losses = [float(net.step(*draw(32))[0]) for _ in range(40)]
    assert all(np.isfinite(losses)) and np.mean(losses[-5:]) < 0.5 * np.mean(losses[:3]), losses
    for w, spec, layer in zip(net.weights, specs, net.pack()):
        w = w.detach().cpu().numpy()
        assert np.array_equal(w != 0, spec.weight != 0)
        # the packer finds the same patterns and kernels again, and nothing to prune
        np.testing.assert_array_equal(admm.project(w, None, spec.keep), w)
        np.testing.assert_array_equal(layer.export("dense").reshape(w.shape), w)
    if dtype != torch.float32:
        for w, c in zip(net.weights, net.copies):
            assert torch.equal(w.detach().to(dtype), c.detach())


def test_packed_layers_predict_what_the_net_does():
    """fp32 activations on both sides (torch's convolutions without TF32): scores agree to fp32 rounding of sums
    of some 1e3 terms, kept well below 1e-3 of their size."""
    tf32 = torch.backends.cudnn.allow_tf32
    torch.backends.cudnn.allow_tf32 = False
    try:
        net = retrain.Retrainer(retrain.pruned_net((3, 32, 64), seed=5), classes=4, dtype=torch.float32, lr=3e-3)
        draw = retrain.synthetic_classes(4, (3, 16, 16), "cuda", seed=6)
        for _ in range(10):
            net.step(*draw(16))
        x, _ = draw(16)
        with torch.no_grad():
            want = net.logits(x)
        got = net.predict(net.pack(), x)
        assert (got - want).abs().max() <= 1e-3 * want.abs().max()
    finally:
        torch.backends.cudnn.allow_tf32 = tf32


OTHER = [0x115, 0x151, 0x154, 0x055]                 # the centre and three corners: no pattern of the default library


def _pruned_with(patterns, keep=0.5):
    rng = np.random.default_rng(31)
    specs = []
    for cin, cout, k in ((3, 16, 1.0), (16, 32, keep)):
        w = (rng.standard_normal((cout, cin, 3, 3)) * np.sqrt(2.0 / (9 * cin))).astype(np.float32)
        specs.append(admm.ConvSpec(admm.project(w, patterns, k), np.zeros(cout, np.float32), keep=k))
    return specs


def test_another_pattern_library_comes_back_from_the_packer():
    """fp32 activations without TF32, as above: scores agree to 1e-3 of their size."""
    tf32 = torch.backends.cudnn.allow_tf32
    torch.backends.cudnn.allow_tf32 = False
    try:
        net = retrain.Retrainer(_pruned_with(OTHER), classes=4, dtype=torch.float32, lr=3e-3, patterns=OTHER)
        draw = retrain.synthetic_classes(4, (3, 16, 16), "cuda", seed=32)
        for _ in range(5):
            net.step(*draw(16))
        layers = net.pack()
        for w, spec, layer in zip(net.weights, net.specs, layers):
            w = w.detach().cpu().numpy()
            assert np.array_equal(w != 0, spec.weight != 0)
            np.testing.assert_array_equal(layer.export("dense").reshape(w.shape), w)
        x, _ = draw(16)
        with torch.no_grad():
            want = net.logits(x)
        assert (net.predict(layers, x) - want).abs().max() <= 1e-3 * want.abs().max()
    finally:
        torch.backends.cudnn.allow_tf32 = tf32


def test_pack_refuses_what_the_packer_would_prune():
    net = retrain.Retrainer(_pruned_with(OTHER), classes=4)          # not told of its library
    with pytest.raises(ValueError, match="constraints"):
        net.pack()
    specs = _pruned_with(None, 0.6)
    specs[1].keep = 0.3                                              # fewer kernels than it has
    with pytest.raises(ValueError, match="layer 1"):
        retrain.Retrainer(specs, classes=4).pack()
    assert len(retrain.Retrainer(_pruned_with(None), classes=4).pack()) == 2
