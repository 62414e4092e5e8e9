"""GaussWSLinear(keep=...) and GaussWSGatedMLP on the CPU, with the kernels' calls replaced by plain products that carry no graph (as the
kernels' results do not): what of them is the modules' own."""
import pytest
import torch

import act_reference as ref
import paper_2505_11170_b200 as gws
from paper_2505_11170_b200 import binding, module


class Kept:
    def __init__(self, rows):
        self.rows, self.buffer = rows, rows


@pytest.fixture
def plain(monkeypatch):
    """The library's calls in 64 bits and without rounding."""

    def gated_fwd(x, w_gate, w_up, activation, save):
        g, u = x @ w_gate.t(), x @ w_up.t()
        return (ref.act(g, activation)[0] * u).detach(), Kept(torch.stack([g, u]).detach())

    def gated_bwd(grad_h, x, w_gate, w_up, saved, activation, want_h=False, want_grad_x=True, want_grad_w=True):
        with torch.no_grad():
            g, u = saved.rows
            a, slope = ref.act(g, activation)
            dg, du = grad_h * u * slope, grad_h * a
            x = x.rows if isinstance(x, Kept) else x
            return tuple(t.detach() for t in (dg @ w_gate + du @ w_up, dg.t() @ x, du.t() @ x, a * u))

    monkeypatch.setattr(binding, "act8_save", lambda x, fmt: Kept(x.detach()))
    monkeypatch.setattr(binding, "wgrad_act8", lambda grad_y, x8: (grad_y.t() @ x8.rows).detach())
    monkeypatch.setattr(binding, "Act8", lambda buffer, *shape: Kept(buffer))
    monkeypatch.setattr(binding, "GatedSaved", lambda buffer, *shape: Kept(buffer))
    monkeypatch.setattr(binding, "gated_fwd", gated_fwd)
    monkeypatch.setattr(binding, "gated_bwd", gated_bwd)


def _rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def _block(x, weights, act=gws.GATED_SILU):
    return module._GatedMLP.apply(x, *weights, act, gws.ACT8_INT8)


def _composed(x, weights, act=gws.GATED_SILU):
    w_gate, w_up, w_down = weights
    g, u = x @ w_gate.t(), x @ w_up.t()
    return (g * torch.sigmoid(g) * u) @ w_down.t()


def _leaves():
    return _rand(1, 6, 8).requires_grad_(), [_rand(2, 12, 8).requires_grad_(), _rand(3, 12, 8).requires_grad_(), _rand(4, 8, 12).requires_grad_()]


def test_first_derivatives_of_the_block(plain):
    x, weights = _leaves()
    got = torch.autograd.grad(_block(x, weights).pow(2).sum(), [x, *weights])
    want = torch.autograd.grad(_composed(x, weights).pow(2).sum(), [x, *weights])
    for p, q in zip(got, want):
        assert torch.allclose(p, q, rtol=1e-10, atol=1e-10)


def test_a_second_derivative_through_the_block_is_refused(plain):
    x, weights = _leaves()
    y = _block(x, weights)
    grad_x, = torch.autograd.grad(y.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        (grad_x.pow(2).sum() + y.sum()).backward()


@pytest.mark.parametrize("of", ["x", "w"])
def test_a_second_derivative_through_a_layer_with_a_kept_input_is_refused(plain, of):
    x, w = _rand(1, 6, 8).requires_grad_(), _rand(2, 12, 8).requires_grad_()
    y = module._KeptLinear.apply(x, w, None, gws.ACT8_INT8)
    grad, = torch.autograd.grad(y.pow(2).sum(), {"x": x, "w": w}[of], create_graph=True)
    with pytest.raises(RuntimeError):
        (grad.pow(2).sum() + y.sum()).backward()


def test_create_graph_alone_changes_nothing(plain):
    x, weights = _leaves()
    want = torch.autograd.grad(_block(x, weights).pow(2).sum(), [x, *weights])
    got = torch.autograd.grad(_block(x, weights).pow(2).sum(), [x, *weights], create_graph=True)
    assert all(torch.equal(p, q) and p.requires_grad for p, q in zip(got, want))
    frozen = [w.detach() for w in weights]
    grad_x, = torch.autograd.grad(_block(x, frozen).sum(), x, create_graph=True)
    assert grad_x.shape == x.shape and grad_x.requires_grad


def test_a_second_derivative_through_the_gradient_of_the_bit_widths_is_refused(monkeypatch):
    monkeypatch.setattr(binding, "bitwidth", lambda bi, *_: bi)
    monkeypatch.setattr(binding, "sample_fwd", lambda desc, w, bt: (w.clone(), torch.ones_like(bt)))
    monkeypatch.setattr(binding, "sample_bwd", lambda desc, g, scale: (None, g.detach().sum(1)))
    monkeypatch.setattr(binding, "bitwidth_grad", lambda grad_bt, *_: grad_bt.detach())
    w, bi = _rand(1, 6, 8).requires_grad_(), _rand(2, 6).requires_grad_()
    w_hat = module._SampledWeight.apply(w, bi, None, 6.0, 4.0, 0.0, {"lambda_term_due": True})
    grad_w, grad_bi = torch.autograd.grad(w_hat.pow(2).sum(), [w, bi], create_graph=True)
    second, = torch.autograd.grad(grad_w.sum(), w, retain_graph=True)       # dL/dw is dL/dw_hat: its graph is torch's
    assert torch.equal(second, torch.full_like(w, 2.0))
    with pytest.raises(RuntimeError):
        (grad_bi.pow(2).sum() + w_hat.sum()).backward()


@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("shape", [(40, 96), (2, 3, 96), (1, 96)])
def test_a_layer_with_a_kept_input_rounds_its_output_once(plain, monkeypatch, bias, shape):
    layer = module.GaussWSLinear(96, 72, bias=bias, group=(1, 24), device="cpu", keep=gws.ACT8_INT8)
    monkeypatch.setattr(layer, "sampled_weight", lambda: layer.weight)
    if bias:
        torch.nn.init.normal_(layer.bias)
    x = _rand(1, *shape).to(torch.bfloat16).requires_grad_()
    y = layer(x)
    assert torch.equal(y, torch.nn.functional.linear(x, layer.weight, layer.bias))
    grad_y = _rand(2, *y.shape).to(torch.bfloat16)
    tensors = [x, layer.weight] + ([layer.bias] if bias else [])
    got = torch.autograd.grad(y, tensors, grad_y)
    want = torch.autograd.grad(torch.nn.functional.linear(x, layer.weight, layer.bias), tensors, grad_y)
    for p, q in zip(got, want):
        assert p.shape == q.shape and torch.allclose(p, q, rtol=2.0 ** -6, atol=2.0 ** -6)


def test_a_layer_pickled_before_it_had_a_choice_of_keep_still_runs(monkeypatch):
    layer = module.GaussWSLinear(32, 16, group=(1, 32), device="cpu")
    del layer.__dict__["keep"]                                  # as such a pickle restores it
    monkeypatch.setattr(layer, "sampled_weight", lambda: layer.weight)
    x = _rand(1, 4, 32).to(torch.bfloat16)
    assert torch.equal(layer(x), torch.nn.functional.linear(x, layer.weight, layer.bias))
