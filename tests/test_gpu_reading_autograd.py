"""attend on inputs that require gradients: torch's backward gives what attend_backward gives."""
import pytest
import torch

import paper_2604_18913_amd as lkg
from test_gpu_reading import _attend, _gpu, _inputs

pytestmark = pytest.mark.gpu


def _case(seed, **kw):
    a, dout = _inputs(seed, torch.bfloat16, [70, 20], [90, 33], 4, 2, 64, bias=True)
    a |= dict(causal=True, cap=20.0, prefix=torch.tensor([5, 0], dtype=torch.int32), **kw)
    return a, dout


@pytest.mark.parametrize("needed", [("q", "k", "v", "bias"), ("q",), ("bias",), ("k", "v")])
def test_gradients_by_torch(needed):
    a, dout = _case(61)
    want = _attend(a, dout)
    b = {k: _gpu(x) for k, x in a.items()}
    for n in needed:
        b[n].requires_grad_()
    out, lse = lkg.attend(**b)
    assert out.requires_grad and torch.equal(out, want["out"]) and torch.equal(lse, want["lse"])
    out.backward(_gpu(dout))
    for n in ("q", "k", "v", "bias"):
        assert torch.equal(b[n].grad, want["d" + n]) if n in needed else b[n].grad is None


def test_gradients_through_layers_on_another_stream():
    # weights in front and behind, the gradient of out in any layout
    a, _ = _case(62)
    b = {k: _gpu(x) for k, x in a.items()}
    w = torch.randn(64, 64, device="cuda") / 8
    v = torch.randn(64, 4, device="cuda")
    grads = []
    for stream in (None, torch.cuda.Stream()):
        x = w.clone().requires_grad_()
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            out, _ = lkg.attend(**{**b, "q": (b["q"].float() @ x).to(torch.bfloat16)})
            (out.float().transpose(0, 1) @ v).square().sum().backward()
        torch.cuda.synchronize()
        grads.append(x.grad)
    assert torch.isfinite(grads[0]).all() and grads[0].abs().max() > 0 and torch.equal(*grads)


def test_without_gradients_nothing_is_kept():
    a, _ = _case(63)
    b = {k: _gpu(x) for k, x in a.items()}
    assert not lkg.attend(**b)[0].requires_grad
    b["q"].requires_grad_()
    with torch.no_grad():
        assert not lkg.attend(**b)[0].requires_grad
    assert not lkg.attend(**{**b, "q": b["q"].detach()})[0].requires_grad


def test_the_gradient_of_lse_is_refused():
    a, _ = _case(64)
    b = {k: _gpu(x) for k, x in a.items()}
    b["k"].requires_grad_()
    out, lse = lkg.attend(**b)
    with pytest.raises(RuntimeError, match="lse has no gradient"):
        (out.float().sum() + lse[lse > -1e30].sum()).backward()
    out, lse = lkg.attend(**b)
    out.float().sum().backward()
    assert b["k"].grad is not None
