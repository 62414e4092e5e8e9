"""GaussWSGatedMLP and GaussWSLinear(keep=...): the activation operators through autograd, next to the sampling pass."""
import math

import pytest
import torch

import act_reference as ref
import paper_2505_11170_b200 as gws
from paper_2505_11170_b200 import binding
from paper_2505_11170_b200.module import GaussWSGatedMLP, GaussWSLinear, GaussWSSet

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _x(shape, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(torch.bfloat16).to(DEV)


def _block(features=96, hidden=160, **kw):
    torch.manual_seed(3)
    block = GaussWSGatedMLP(features, hidden, **kw)
    for layer in block.layers:
        torch.nn.init.normal_(layer.weight, std=1.0 / math.sqrt(layer.in_features))
    return block


def _plain(block, x, grad_y, weights):
    """Forward and backward of the block in 64 bits from its sampled weights, with x, g and u kept in the block's format."""
    wg, wu, wd = (w.detach().double() for w in weights)
    x64 = x.double().reshape(-1, x.shape[-1])
    g, u = x64 @ wg.t(), x64 @ wu.t()
    a, _ = ref.act(g, block.activation)
    y = (a * u) @ wd.t()
    keep = (lambda t: t.to(torch.bfloat16).double()) if block.keep == gws.SAVE_BF16 else (lambda t: ref.values(*ref.encode(t, block.keep), t.shape[1]))
    g, u, x64 = keep(g), keep(u), keep(x64)
    a, slope = ref.act(g, block.activation)
    dy = grad_y.double().reshape(-1, grad_y.shape[-1])
    dh = dy @ wd
    dg, du = dh * u * slope, dh * a
    return y, dg @ wg + du @ wu, dg.t() @ x64, du.t() @ x64, dy.t() @ (a * u)


def _close(got, want, what):
    # independent BF16 roundings (each at most 2^-8 of a number, 2^-9 and a half on average) of the result, of h or dh, of dg and du and, in
    # BF16 copies, of g and u: five of them, with norms adding in squares
    err = float((got.double().reshape(want.shape) - want).norm() / want.norm())
    assert err <= math.sqrt(5) * 2.0 ** -8, (what, err)


@pytest.mark.parametrize("keep", [gws.ACT8_INT8, gws.ACT8_E4M3, gws.SAVE_BF16])
@pytest.mark.parametrize("activation", [gws.GATED_SILU, gws.GATED_GELU_TANH, gws.GATED_RELU])
@pytest.mark.parametrize("shape", [(64, 96), (2, 31, 96), (1, 96)])
def test_block_forward_and_gradients(keep, activation, shape):
    block = _block(activation=activation, keep=keep)
    x = _x(shape, 1).requires_grad_()
    grad_y = _x(shape, 2)
    weights = [layer.sampled_weight() for layer in block.layers]
    y = block(x)
    y.backward(grad_y)
    want = _plain(block, x.detach(), grad_y, weights)
    assert y.shape == x.shape and x.grad.shape == x.shape
    for got, exact, what in zip((y, x.grad, block.gate.weight.grad, block.up.weight.grad, block.down.weight.grad), want, ("y", "x", "gate", "up", "down")):
        _close(got.detach(), exact, what)
    assert all(layer.b_i.grad is not None and bool(torch.isfinite(layer.b_i.grad).all()) for layer in block.layers)


def test_block_in_a_set_gives_the_bits_of_the_block_alone():
    alone, together = _block(lam=0.1, user_seed=4), _block(lam=0.1, user_seed=4)
    together.load_state_dict(alone.state_dict())
    sampler = GaussWSSet(together.layers)
    for update in range(2):
        x, grad_y = _x((50, 96), 10 + update), _x((50, 96), 20 + update)
        sampler.sample()
        outs = []
        for block in (alone, together):
            leaf = x.clone().requires_grad_()
            y = block(leaf)
            y.backward(grad_y)
            outs.append((y, leaf.grad, *[layer.weight.grad for layer in block.layers]))
        sampler.finish_backward()
        assert all(torch.equal(p, q) for p, q in zip(*outs))
        for a, b in zip(alone.layers, together.layers):
            assert torch.allclose(a.b_i.grad, b.b_i.grad, rtol=1e-5, atol=1e-12)
            a.weight.grad = b.weight.grad = a.b_i.grad = b.b_i.grad = None
        alone.advance()
        sampler.advance()


def test_block_keeps_one_byte_per_element():
    m, features, hidden = 512, 256, 704
    x = _x((m, features), 5).requires_grad_()
    seen = {}
    for keep in (gws.ACT8_INT8, gws.SAVE_BF16):
        block = _block(features, hidden, keep=keep)
        weights = [layer.sampled_weight().detach() for layer in block.layers]
        for layer, w in zip(block.layers, weights):
            layer.sampled_weight = lambda w=w: w.requires_grad_()
        kept = []
        with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t.numel() * t.element_size()) or t, lambda t: t):
            block(x)
        seen[keep] = sum(kept) - sum(w.numel() * w.element_size() for w in weights)
    elements = m * (features + 2 * hidden)
    assert seen[gws.ACT8_INT8] <= elements * 33 // 32 + 2048 and seen[gws.SAVE_BF16] >= 2 * elements


def test_gradients_that_are_not_needed_are_not_formed():
    block = _block()
    for layer in block.layers:
        layer.weight.requires_grad_(False)
        layer.b_i.requires_grad_(False)
    x = _x((20, 96), 6).requires_grad_()
    y = block(x)
    y.backward(_x((20, 96), 7))
    assert x.grad is not None and all(layer.weight.grad is None for layer in block.layers)
    with torch.no_grad():
        assert torch.equal(block(x), y)
    assert not block(x.detach()).requires_grad


@pytest.mark.parametrize("keep", [gws.ACT8_INT8, gws.ACT8_E4M3])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("shape", [(40, 96), (2, 3, 5, 96)])
def test_linear_layer_with_a_kept_input(keep, bias, shape):
    torch.manual_seed(2)
    kept = GaussWSLinear(96, 72, bias=bias, group=(1, 24), keep=keep)
    plain = GaussWSLinear(96, 72, bias=bias, group=(1, 24))
    plain.load_state_dict(kept.state_dict())
    x = _x(shape, 8)
    grad_y = _x((*shape[:-1], 72), 9)
    grads = []
    for layer in (kept, plain):
        leaf = x.clone().requires_grad_()
        y = layer(leaf)
        y.backward(grad_y)
        grads.append((y, leaf.grad, layer.weight.grad, layer.bias.grad if bias else None))
    _close(grads[0][0].detach(), grads[1][0].detach().double(), "y")
    _close(grads[0][1], grads[1][1].double(), "x")
    rows = x.double().reshape(-1, 96)
    want = grad_y.double().reshape(-1, 72).t() @ ref.values(*ref.encode(rows, keep), 96)
    _close(grads[0][2], want, "weight")
    if bias:
        _close(grads[0][3], grads[1][3].double(), "bias")


def test_broadcast_gradient_and_refusals():
    block = _block()
    x = _x((30, 96), 11).requires_grad_()
    block(x).sum().backward()                       # the gradient arrives as one number broadcast over the block's output
    assert bool(torch.isfinite(x.grad.float()).all()) and bool(x.grad.any())
    with pytest.raises(ValueError):
        GaussWSGatedMLP(96, 160, keep=gws.SAVE_NONE)
    with pytest.raises(ValueError):
        GaussWSGatedMLP(96, 160, activation=5)
    with pytest.raises(ValueError):
        GaussWSLinear(96, 72, keep=binding.SAVE_BF16)
    with pytest.raises(ValueError):
        block(x.float())


def test_training_lowers_the_loss():
    # the operators as they are used: sampled weights, 8-bit activations, an optimizer; a target the block can fit
    torch.manual_seed(0)
    block = GaussWSGatedMLP(64, 128, b_init=8.0, b_target=6.0)
    for layer in block.layers:
        torch.nn.init.normal_(layer.weight, std=0.1)
    sampler = GaussWSSet(block.layers)
    opt = torch.optim.AdamW(block.parameters(), lr=2e-3)
    x = _x((256, 64), 30)
    target = _x((256, 64), 31, 0.3)
    losses = []
    for _ in range(120):
        sampler.sample()
        loss = (block(x).float() - target.float()).square().mean()
        loss.backward()
        sampler.finish_backward()
        opt.step()
        opt.zero_grad(set_to_none=False)
        sampler.advance()
        losses.append(float(loss))
    assert losses[-1] < 0.5 * losses[0]


@pytest.mark.parametrize("shape", [(40, 96), (2, 3, 5, 96), (515, 96)])
def test_a_kept_input_leaves_the_output_of_the_layer_as_it_was(shape):
    torch.manual_seed(4)
    kept = GaussWSLinear(96, 72, group=(1, 24), keep=gws.ACT8_INT8)
    plain = GaussWSLinear(96, 72, group=(1, 24))
    torch.nn.init.normal_(kept.bias)
    plain.load_state_dict(kept.state_dict())
    x = _x(shape, 8)
    assert torch.equal(kept(x), plain(x))


def test_no_tokens_and_one():
    for keep in (gws.ACT8_INT8, gws.SAVE_BF16):
        block = _block(keep=keep)
        for shape in ((0, 96), (2, 0, 96), (1, 96)):
            x = _x(shape, 12).requires_grad_()
            y = block(x)
            assert y.shape == x.shape
            y.sum().backward()
            assert x.grad.shape == x.shape and all(bool(torch.isfinite(layer.weight.grad.float()).all()) for layer in block.layers)
    layer = GaussWSLinear(96, 72, keep=gws.ACT8_INT8)
    x = _x((0, 96), 13).requires_grad_()
    layer(x).sum().backward()
    assert x.grad.shape == (0, 96) and not bool(layer.weight.grad.any()) and not bool(layer.bias.grad.any())
