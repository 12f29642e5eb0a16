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
