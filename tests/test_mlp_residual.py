"""GaussWSMLP on the CPU, with the linear layer's calls replaced by plain forms: its residual."""
import pytest
import torch

import paper_2505_11170_b200 as gws
from paper_2505_11170_b200 import binding, module


@pytest.fixture
def block(monkeypatch):
    """A block whose weights are sampled by nobody and whose products are torch's."""
    monkeypatch.setattr(module.GaussWSLinear, "sampled_weight", lambda self: self.weight)

    def linear_fwd(x, w, bias=None, residual=None, activation=gws.ACT_NONE, save=gws.SAVE_NONE):
        z = torch.nn.functional.linear(x, w, bias)
        y = z if activation == gws.ACT_NONE else torch.nn.functional.gelu(z, approximate="tanh")
        return (y if residual is None else y + residual).detach(), None

    monkeypatch.setattr(binding, "linear_fwd", linear_fwd)
    layer = module.GaussWSMLP(32, 64, group=(1, 32), device="cpu", bias=False)
    return layer.requires_grad_(False)


@pytest.mark.parametrize("shape", [(3, 4, 32), (12, 32), (1, 12, 32), (4, 96), (4, 3, 1, 32), (4, 3, 31), (32,)])
def test_a_residual_of_another_shape_is_refused(block, shape):
    """Of as many elements (and tokens in another order) it would be added in the wrong places."""
    x = torch.randn(4, 3, 32).to(torch.bfloat16)
    with pytest.raises(ValueError, match="shape"):
        block(x, torch.zeros(shape, dtype=torch.bfloat16))


@pytest.mark.parametrize("shape", [(4, 3, 32), (7, 32), (32,)])
def test_a_residual_of_the_shape_of_x_is_added(block, shape):
    x, r = (torch.randn(shape).to(torch.bfloat16) for _ in range(2))
    strided = torch.randn(*shape[:-1], 40).to(torch.bfloat16)[..., :32]
    for residual in (r, strided):
        y = block(x, residual)
        assert y.shape == x.shape and torch.equal(y, block(x) + residual)
