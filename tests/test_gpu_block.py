"""GaussWSLayerNorm, GaussWSMLP and GaussWSAdamW: the norm, the linear layers with their epilogues and the optimizer as a training step uses them, next to the sampling pass."""
import math

import numpy as np
import pytest
import torch

import act_reference as ref
import paper_2505_11170_b200 as gws
import step_reference as step_ref
from paper_2505_11170_b200.module import GaussWSLayerNorm, GaussWSLinear, GaussWSMLP, GaussWSSet
from paper_2505_11170_b200.optimizer import GaussWSAdamW

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _x(shape, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(torch.bfloat16).to(DEV)


def _mlp(features=96, hidden=160, **kw):
    torch.manual_seed(3)
    block = GaussWSMLP(features, hidden, **kw)
    for layer in block.layers:
        torch.nn.init.normal_(layer.weight, std=1.0 / math.sqrt(layer.in_features))
        if layer.bias is not None:
            torch.nn.init.normal_(layer.bias, std=0.2)
    return block


def _close(got, want, what, roundings=5):
    # independent BF16 roundings (each at most 2^-8 of a number, 2^-9 and a half on average) of the result, of h or dh, of dz and, in BF16 copies, of z and x, with norms
    # adding in squares
    err = float((got.double().reshape(want.shape) - want).norm() / want.norm())
    assert err <= math.sqrt(roundings) * 2.0 ** -8, (what, err)


def _plain_mlp(block, x, residual, grad_y, weights):
    """Forward and backward of the block in 64 bits from its sampled weights, with x and z kept in the block's format."""
    wu, wd = (w.detach().double() for w in weights)
    bu, bd = (0.0 if layer.bias is None else layer.bias.detach().double() for layer in block.layers)
    x64, dy = x.double().reshape(-1, x.shape[-1]), grad_y.double().reshape(-1, grad_y.shape[-1])
    z = x64 @ wu.t() + bu
    y = ref.act(z, block.activation)[0] @ wd.t() + bd
    if residual is not None:
        y = y + residual.double().reshape(y.shape)
    keep = (lambda t: t.to(torch.bfloat16).double()) if block.keep == gws.SAVE_BF16 else (lambda t: ref.values(*ref.encode(t, block.keep), t.shape[1]))
    a, slope = ref.act(keep(z), block.activation)
    dz = (dy @ wd) * slope
    return y, dz @ wu, dz.t() @ keep(x64), dz.sum(0), dy.t() @ a, dy.sum(0)


@pytest.mark.parametrize("keep", [gws.ACT8_INT8, gws.ACT8_E4M3, gws.SAVE_BF16])
@pytest.mark.parametrize("activation", [gws.GATED_SILU, gws.GATED_GELU_TANH, gws.GATED_RELU])
@pytest.mark.parametrize("shape", [(64, 96), (2, 31, 96), (1, 96)])
def test_block_forward_and_gradients(keep, activation, shape):
    for bias, stream in ((True, True), (False, False)):
        block = _mlp(activation=activation, keep=keep, bias=bias)
        x, grad_y = _x(shape, 1).requires_grad_(), _x(shape, 2)
        residual = _x(shape, 5).requires_grad_() if stream else None
        weights = [layer.sampled_weight() for layer in block.layers]
        y = block(x, residual)
        y.backward(grad_y)
        want = _plain_mlp(block, x.detach(), None if residual is None else residual.detach(), grad_y, weights)
        got = [y, x.grad, block.up.weight.grad, block.up.bias.grad if bias else None, block.down.weight.grad, block.down.bias.grad if bias else None]
        for p, q, what in zip(got, want, ("y", "x", "up", "up bias", "down", "down bias")):
            if p is not None:
                _close(p.detach(), q, what)
        if stream:
            assert torch.equal(residual.grad, grad_y)
        assert all(layer.b_i.grad is not None and bool(torch.isfinite(layer.b_i.grad).all()) for layer in block.layers)


def test_block_in_a_set_gives_the_bits_of_the_block_alone():
    alone, together = _mlp(lam=0.1, user_seed=4), _mlp(lam=0.1, user_seed=4)
    together.load_state_dict(alone.state_dict())
    sampler = GaussWSSet(together.layers)
    for update in range(2):
        x, grad_y = _x((50, 96), 10 + update), _x((50, 96), 20 + update)
        sampler.sample()
        outs = []
        for block in (alone, together):
            leaf = x.clone().requires_grad_()
            y = block(leaf, x)
            y.backward(grad_y)
            outs.append((y, leaf.grad, *[t.grad for layer in block.layers for t in (layer.weight, layer.bias)]))
        sampler.finish_backward()
        assert all(torch.equal(p, q) for p, q in zip(*outs))
        for a, b in zip(alone.layers, together.layers):
            a.weight.grad = b.weight.grad = a.b_i.grad = b.b_i.grad = a.bias.grad = b.bias.grad = None
        alone.advance()
        sampler.advance()


def test_block_keeps_one_byte_per_element():
    m, features, hidden = 512, 256, 704
    x = _x((m, features), 5).requires_grad_()
    seen = {}
    for keep in (gws.ACT8_INT8, gws.SAVE_BF16):
        block = _mlp(features, hidden, keep=keep)
        weights = [layer.sampled_weight().detach() for layer in block.layers]
        for layer, w in zip(block.layers, weights):
            layer.sampled_weight = lambda w=w: w.requires_grad_()
        kept = []
        with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t.numel() * t.element_size()) or t, lambda t: t):
            block(x)
        seen[keep] = sum(kept) - sum(w.numel() * w.element_size() for w in weights)
    elements = m * (features + hidden)
    assert seen[gws.ACT8_INT8] <= elements * 33 // 32 + 2048 and seen[gws.SAVE_BF16] >= 2 * elements


def test_no_tokens_and_frozen_parameters():
    block, norm = _mlp(), GaussWSLayerNorm(96)
    for shape in ((0, 96), (2, 0, 96), (1, 96)):
        x = _x(shape, 12).requires_grad_()
        y, s = norm(x, x.detach())
        out = block(y, s)
        assert out.shape == x.shape
        out.sum().backward()
        assert x.grad.shape == x.shape and all(bool(torch.isfinite(p.grad.float()).all()) for p in (*block.parameters(), *norm.parameters()))
    frozen, x = _mlp(), _x((20, 96), 6).requires_grad_()
    for p in frozen.parameters():
        p.requires_grad_(False)
    frozen(x).backward(_x((20, 96), 7))
    assert x.grad is not None and all(p.grad is None for p in frozen.parameters())
    with torch.no_grad():
        assert not frozen(x).requires_grad and not norm(x).requires_grad
    only = _mlp()
    for p in only.parameters():
        p.requires_grad_(p is only.down.weight)
    only(x.detach()).sum().backward()
    assert bool(only.down.weight.grad.any()) and only.up.weight.grad is None


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bias", [True, False])
def test_norm_and_its_gradients(dtype, bias):
    norm = GaussWSLayerNorm(200, bias=bias, dtype=dtype)
    torch.nn.init.normal_(norm.weight, 1.0, 0.3)
    x, r, gy, gs = (_x((3, 7, 200), i) for i in range(4))
    x.requires_grad_()
    r.requires_grad_()
    y, s = norm(x, r)
    torch.autograd.backward([y, s], [gy, gs])
    leaves = [t.detach().double().requires_grad_() for t in (s, norm.weight)] + ([norm.bias.detach().double().requires_grad_()] if bias else [])
    want_y = torch.nn.functional.layer_norm(leaves[0], (200,), leaves[1], leaves[2] if bias else None, 1e-5)
    want = torch.autograd.grad(want_y, leaves, gy.double())
    _close(y.detach(), want_y.detach(), "y", 1)
    _close(x.grad, want[0] + gs.double(), "x", 1)
    assert torch.equal(x.grad, r.grad) and x.grad.data_ptr() != r.grad.data_ptr()
    _close(norm.weight.grad, want[1], "weight", 1)
    if bias:
        _close(norm.bias.grad, want[2], "bias", 1)
    alone = norm(s.detach())
    assert torch.equal(alone, y)


class Block(torch.nn.Module):
    def __init__(self, features, hidden, k):
        super().__init__()
        self.norm, self.mlp = GaussWSLayerNorm(features), GaussWSMLP(features, hidden, layer_index=2 * k, user_seed=7, lam=0.05)

    def forward(self, stream):
        return self.mlp(self.norm(stream), stream)


@pytest.mark.parametrize("moments", [gws.ADAMW_F32, gws.ADAMW_8BIT])
def test_updates_of_a_stack_of_blocks(moments):
    """Sampling, norms, blocks, gradients and the step over all tensors; the step is the specified one for the gradients that the backward pass left."""
    torch.manual_seed(5)
    model = torch.nn.Sequential(*[Block(96, 200, k) for k in range(3)])
    sampler = GaussWSSet([layer for block in model for layer in block.mlp.layers])
    decayed = [p for p in model.parameters() if p.dim() > 1]
    others = [p for p in model.parameters() if p.dim() <= 1]
    optimizer = GaussWSAdamW([dict(params=decayed, weight_decay=0.1), dict(params=others, weight_decay=0.0)], lr=2e-3, betas=(0.9, 0.95), moments=moments)
    params = decayed + others
    w = [p.detach().float().cpu().numpy().ravel() for p in params]
    m, v = ([np.zeros(-(-t.size // 256) * 256, np.float32) for t in w] for _ in range(2))
    for update in range(1, 4):
        x = _x((300, 96), 40 + update)
        sampler.sample()
        out = model(x)
        out.backward(_x((300, 96), 50 + update, 1e-2))
        sampler.finish_backward()
        grads = [p.grad.float().cpu().numpy().ravel() for p in params]
        before = gws.launch_count()
        optimizer.step()
        assert gws.launch_count() - before == 1
        for i, p in enumerate(params):
            pad = lambda t: np.concatenate([t, np.zeros(m[i].size - t.size, np.float32)])
            new, m[i], v[i], r = step_ref.adamw32(pad(w[i]), pad(grads[i]), m[i], v[i], 2e-3, 0.9, 0.95, 1e-8, 0.1 if i < len(decayed) else 0.0, update)
            if moments == gws.ADAMW_8BIT:
                m[i] = step_ref.decode_m(*step_ref.encode_m(m[i])).ravel()
                r = step_ref.decode_r(*step_ref.encode_r(r)).ravel()
                v[i] = r * r
            w[i] = new[:w[i].size].astype(np.float32)
            assert np.array_equal(optimizer.weight(p).cpu().numpy().ravel(), w[i]), (update, i)
            got = optimizer.moments(p)
            assert np.array_equal(got[0].cpu().numpy().ravel(), m[i][:w[i].size]) and np.array_equal(got[1].cpu().numpy().ravel(), v[i][:w[i].size])
        optimizer.zero_grad()
        sampler.advance()
    gws.check_waits()


def test_a_stack_goes_on_from_its_state_as_it_would_have():
    def build():
        torch.manual_seed(6)
        layer = GaussWSLinear(64, 48, bias=True)
        return layer, GaussWSAdamW(layer.parameters(), lr=1e-2, moments=gws.ADAMW_8BIT)

    def update(layer, optimizer, k):
        layer(_x((30, 64), k)).backward(_x((30, 48), 100 + k))
        optimizer.step()
        optimizer.zero_grad()
        layer.advance()

    (a, oa), (b, ob) = build(), build()
    for k in range(3):
        update(a, oa, k)
    b.load_state_dict(a.state_dict())
    b.step = a.step
    ob.load_state_dict(oa.state_dict())
    for k in range(3, 5):
        update(a, oa, k)
        update(b, ob, k)
    assert all(torch.equal(p, q) for p, q in zip(a.parameters(), b.parameters()))
    assert torch.equal(oa._state.moments, ob._state.moments) and torch.equal(oa._state.rest, ob._state.rest)


def test_a_captured_step_of_the_optimizer():
    def build(capturable):
        torch.manual_seed(8)
        params = [torch.nn.Parameter(torch.randn(n, device=DEV).to(t)) for n, t in ((1000, torch.bfloat16), (77, torch.float32))]
        for p in params:
            p.grad = torch.randn_like(p)
        lr = torch.full((1,), 1e-3, device=DEV) if capturable else 1e-3
        return params, GaussWSAdamW(params, lr=lr, capturable=capturable, weight_decay=0.0)

    (p, o), (q, e) = build(True), build(False)
    o.step()
    e.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o.step()
    for rate in (1e-3, 5e-4):
        o.param_groups[0]["lr"].fill_(rate)
        for a, b in zip(p, q):
            a.grad.mul_(-0.5)
            b.grad.mul_(-0.5)
        graph.replay()
        e.param_groups[0]["lr"] = float(np.float32(rate))
        e.step()
    torch.cuda.synchronize()
    # alpha is rounded from lr / (1 - b1^t) in double on either side, with a power that may differ in its last place
    assert o.state_dict()["gws"]["count"] == 3
    for a, b in zip(p, q):
        assert torch.allclose(o.weight(a), e.weight(b), rtol=2.0 ** -22, atol=1e-9)
