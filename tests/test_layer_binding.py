"""What the binding's layer operators refuse on the host: arguments that a call would lose without a word."""
import pytest
import torch

from paper_1803_04209_b200 import binding, build


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    binding._load_torch()
    return binding.load_library()


def _with_gradient(name):
    t = torch.ones(4, 8) if name in ("x", "h", "gate", "residual", "d_residual", "d_norm", "out") else torch.ones(8)
    return t.requires_grad_()


# autograd does not see these calls: a tensor that wants a gradient would not get the part that goes through them
@pytest.mark.parametrize("call", [
    lambda t: binding.dropout(t("x"), 0.5, 1),
    lambda t: binding.residual_norm(t("x")),
    lambda t: binding.residual_norm(t("x"), t("x")),
    lambda t: binding.residual_norm_grad(t("x"), t("x"), t("x"), t("x")),
    lambda t: binding.quantize_rows(t("x")),
    lambda t: binding._vector(t("scale"), "scale", 8, 0),
    lambda t: binding._same(t("gate"), "gate", 4, 8, 0, torch.float32),
])
def test_tensors_that_require_a_gradient(call):
    with pytest.raises(ValueError, match="requires a gradient"):
        call(_with_gradient)
    with torch.no_grad(), pytest.raises(ValueError) as e:            # then it is their being on the CPU that is refused
        call(_with_gradient)
    assert "requires a gradient" not in str(e.value)


# results that the call would not write, and numbers that would arrive as others
@pytest.mark.parametrize("call,what", [
    (lambda x: binding.residual_norm(x, residual_out=x), "residual_out"),
    (lambda x: binding.residual_norm(x, x, want_norm=False, norm_out=x), "norm_out"),
    (lambda x: binding.residual_norm(x, x, quantize=True, norm_out=x), "norm_out"),
    (lambda x: binding.residual_norm(x, x, gate=x, gate_rows=1 << 63), "gate_rows"),
    (lambda x: binding.residual_norm_grad(x, x, x, x, gate=x, gate_rows=1 << 64), "gate_rows"),
    (lambda x: binding.dropout(x, 0.5, 1, first_row=1 << 64), "first_row"),
    (lambda x: binding.dropout(x, 0.5, 1, first_row=(1 << 63) + 5), "first_row"),
    (lambda x: binding.dropout(x, 0.5, 1, first_row=-(1 << 64)), "first_row"),
])
def test_what_a_call_would_ignore(call, what):
    with pytest.raises(ValueError, match=what):
        call(torch.ones(4, 8))
