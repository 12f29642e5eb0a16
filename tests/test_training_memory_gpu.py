"""What the training operators owe torch's memory and autograd: memory that a call on another stream uses is not
handed out again before, and tensors written in place are known to be changed."""
import pytest
import torch

from paper_2003_06513_gb300 import norm, optim

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("state_bits", [8, 32])
def test_memory_used_on_another_stream_is_recorded(monkeypatch, state_bits):
    p = torch.ones(600, device="cuda")
    opt = optim.AdamW([p], state_bits=state_bits)
    g = [torch.full((600,), 0.5, device="cuda")]
    recorded = []
    real = torch.Tensor.record_stream
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: (recorded.append((t.data_ptr(), s.cuda_stream)), real(t, s))[1])
    opt.grad_norm(g)
    opt.step(g)
    assert not recorded                                  # its own stream
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    own = {t.data_ptr() for t in (opt._t._table, opt.m, opt.v, opt.m_scale, opt.v_scale) if t is not None}
    opt.step(g, stream=side)
    assert {a for a, s in recorded if s == side.cuda_stream} == own
    recorded.clear()
    with torch.cuda.stream(side):
        opt.grad_norm(g)
    assert recorded == [(opt._t._table.data_ptr(), side.cuda_stream)]
    torch.cuda.synchronize()
    assert opt.steps == 2 and bool((p < 1).all())


def test_what_a_step_writes_has_a_new_version():
    p = torch.ones(40, device="cuda")
    c = p.half().requires_grad_(True)
    opt = optim.AdamW([p], copies=[c], grad_dtypes=torch.float16)
    square = (c * c).sum()                               # keeps c for its backward pass
    versions = p._version, c._version
    opt.step([torch.ones_like(c)])
    assert p._version > versions[0] and c._version > versions[1]
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        square.backward()


def test_out_has_a_new_version():
    x = torch.randn(2, 8, 4, 4, device="cuda").contiguous(memory_format=torch.channels_last)
    out, both = torch.empty_like(x), torch.empty(2, device="cuda")
    before = out._version, both._version
    _, mean, rstd = norm.pp_group_norm(x, 2, out=out)
    assert out._version > before[0]
    between = out._version
    norm.pp_group_norm_backward(x, x, mean, rstd, 2, out=out)
    assert out._version > between
    optim.GradNorm([(4,)])([torch.ones(4, device="cuda")], out=both)
    assert both._version > before[1] and float(both[0]) == 2.0


def _pruned():
    w = torch.ones(6, 4, 3, 3, device="cuda")
    w[:, :, 0] = 0
    return w


@pytest.mark.parametrize("state_bits", [8, 32])
@pytest.mark.parametrize("which", ["parameter", "copy", "parameter's order", "module"])
def test_a_parameter_that_was_given_other_memory_is_refused(which, state_bits):
    """Its old memory may be another tensor's: nothing is written, and the step is not counted."""
    p, q = torch.ones(40, device="cuda"), torch.ones(7, 6, device="cuda")
    c = p.half()
    net = torch.nn.Linear(3, 5, device="cuda")
    opt = optim.AdamW([p, q, net.weight], state_bits=state_bits, copies=[c, None, None])
    grads = [torch.ones_like(p), torch.ones_like(q), torch.ones_like(net.weight)]
    opt.step(grads)
    old = {"parameter": p, "copy": c, "parameter's order": q, "module": net.weight}[which]
    before = old.detach()                                # its memory as it was
    if which == "module":
        torch.nn.utils.vector_to_parameters(torch.full((20,), 3.0, device="cuda"), net.parameters())
    elif which == "parameter's order":
        q.data = q.data.view(6, 7).t()                   # the same address and shape, columns first
        assert q.shape == (7, 6) and q.stride() == (1, 7)
    else:
        old.data = old.data.clone()
    kept = [t.clone() for t in (p, q, c, net.weight, before, opt.m.view(torch.uint8))]
    with pytest.raises(ValueError, match="other memory"):
        opt.step(grads)
    assert opt.steps == 1
    assert all(torch.equal(a, b) for a, b in zip(kept, (p, q, c, net.weight, before, opt.m.view(torch.uint8))))
    again = optim.AdamW([p, q, net.weight], state_bits=state_bits, copies=[c, None, None], state=opt.state_dict())
    again.step([torch.ones_like(p), torch.ones_like(q), torch.ones_like(net.weight)])
    assert again.steps == 2 and bool((p < kept[0]).all()) and bool((net.weight < kept[3]).all()) and torch.equal(c, p.half())


def test_masks_are_read_where_they_were():
    """Masks that were given other memory: the handle holds what it reads."""
    w = _pruned()
    taps = optim.taps_of(w)
    opt = optim.AdamW([w], taps=[taps], weight_decay=0.0)
    n = optim.GradNorm([w.shape], taps=[taps])
    taps.data = torch.zeros(5, dtype=torch.int16, device="cuda")
    junk = [torch.full((24,), -1, dtype=torch.int16, device="cuda") for _ in range(64)]      # would take freed memory
    g = torch.ones_like(w)
    for norm_of in (opt.grad_norm, n):
        assert float(norm_of([g])[0]) == pytest.approx(144 ** 0.5)                          # six of nine taps
    opt.step([g])
    assert bool((w[:, :, 0] == 0).all()) and bool((w[:, :, 1:] < 1).all()) and len(junk) == 64


@pytest.mark.parametrize("state_bits", [8, 32])
def test_states_of_another_size_or_type_are_refused(state_bits):
    """m, v and their scales are the object's attributes, which a program may set."""
    p = torch.ones(600, device="cuda")
    opt = optim.AdamW([p], state_bits=state_bits)
    g = [torch.ones_like(p)]
    for name in ("m", "v") + (("m_scale", "v_scale") if state_bits == 8 else ()):
        right = getattr(opt, name)
        for wrong in (right[:-1], right.view(torch.uint8), right.cpu(), torch.empty(2 * right.numel(), dtype=right.dtype, device="cuda")[::2], None):
            setattr(opt, name, wrong)
            with pytest.raises(ValueError, match=name):
                opt.step(g)
        setattr(opt, name, right.clone())
    assert opt.steps == 0 and bool((p == 1).all())
    opt.step(g)
    assert opt.steps == 1 and bool((p < 1).all())


@pytest.mark.parametrize("own_stream", [False, True])
@pytest.mark.parametrize("state_bits", [8, 32])
def test_a_new_object_is_ready_for_calls_on_any_stream(monkeypatch, state_bits, own_stream):
    """The states' zeros come after 0.1 s of other work on the constructor's stream: the constructor waits for them."""
    p = torch.ones(600, device="cuda")
    stream = torch.cuda.Stream() if own_stream else None
    torch.cuda.synchronize()
    zeros = torch.zeros

    def late(*args, **kw):
        torch.cuda._sleep(200_000_000)
        return zeros(*args, **kw)
    monkeypatch.setattr(torch, "zeros", late)
    opt = optim.AdamW([p], state_bits=state_bits, stream=stream)
    assert (stream or torch.cuda.current_stream()).query()
    g = [torch.ones_like(p)]
    torch.cuda.synchronize()
    opt.step(g, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert torch.allclose(opt.state_of(0)[0], torch.full_like(p, 0.1), rtol=0.07)
