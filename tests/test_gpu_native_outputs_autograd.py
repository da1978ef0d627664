"""Output tensors that the binding's native half puts together take part in autograd as any leaf does: themselves, not copies of them."""
import pytest
import torch

from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu


def outputs():
    x = torch.randn(3, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    hidden, _, scale = tb.tbik_rmsnorm_fp8(x, w, residual=x)
    return {"hidden": hidden, "row scale": scale, "product": tb.tbik_gemm_epilogue(x, torch.randn(64, 64, device="cuda").bfloat16(), 64, 1, out_dtype=torch.float32)}


@pytest.mark.parametrize("name", ["hidden", "row scale", "product"])
def test_outputs_are_leaves(name, monkeypatch):
    tb.lib()
    native = []
    real = tb._native
    spy = lambda g: (lambda *a: native.append(g(*a)) or native[-1])
    monkeypatch.setattr(tb, "_native", type("Spy", (), {k: staticmethod(spy(getattr(real, k))) for k in ("epilogue", "eight_bits")}))
    t = outputs()[name]
    made = [o for a in native for o in (a if isinstance(a, tuple) else (a,))]
    assert any(t is o for o in made)                              # the native half's own tensor
    assert t.is_leaf and not t.requires_grad and t.grad_fn is None and t._version == 0
    t.requires_grad_()
    (t * t).sum().backward()
    assert t.grad is not None and torch.equal(t.grad, 2 * t.detach())
    with torch.no_grad():
        t.mul_(2)
    assert t._version == 1
    y = t * t                                                     # saves t
    with torch.no_grad():
        t.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    v = t.detach().view(-1)                                       # a view shares memory and version
    v.zero_()
    assert bool((t == 0).all()) and v.untyped_storage().data_ptr() == t.untyped_storage().data_ptr()
