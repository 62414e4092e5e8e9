"""GaussWSLayerNorm, GaussWSMLP and GaussWSAdamW on the CPU, with the kernels' calls replaced by plain forms that carry no graph (as the kernels' results do not): what of
them is the modules' own."""
import copy
import pickle

import pytest
import torch

import act_reference as ref
import paper_2505_11170_b200 as gws
from paper_2505_11170_b200 import binding, module
from paper_2505_11170_b200.optimizer import GaussWSAdamW

EPS = 1e-5


class Kept:
    def __init__(self, rows):
        self.rows, self.buffer = rows, rows


def _act(z, kind):
    return (z, torch.ones_like(z)) if kind == gws.ACT_NONE else ref.act(z, kind)


@pytest.fixture
def plain(monkeypatch):
    """The library's calls in 64 bits and without rounding."""

    def linear_fwd(x, w, bias=None, residual=None, activation=gws.ACT_NONE, save=gws.SAVE_NONE):
        z = x @ w.t() if bias is None else x @ w.t() + bias
        y = _act(z, activation)[0]
        return (y if residual is None else y + residual).detach(), None if save == gws.SAVE_NONE else Kept(z.detach())

    def linear_bwd(grad_y, x, w, saved=None, activation=gws.ACT_NONE, want_grad_x=True, want_grad_w=True, want_grad_bias=False, want_act=False, bias_dtype=None):
        a, slope = (None, 1.0) if saved is None else _act(saved.rows, activation)
        dz = (grad_y * slope).detach()
        x = x.rows if isinstance(x, Kept) else x
        return dz @ w if want_grad_x else None, dz.t() @ x if want_grad_w else None, dz.sum(0) if want_grad_bias else None, a.detach() if want_act else None

    def layernorm_fwd(x, weight, bias, eps, residual=None, want_stats=True):
        s = (x if residual is None else x + residual).detach()
        return torch.nn.functional.layer_norm(s, s.shape[-1:], weight, bias, eps).detach(), s, torch.zeros(())

    def layernorm_bwd(grad_y, s, weight, stats, grad_sum=None, want_grad_x=True, want_grad_weight=True, want_grad_bias=True):
        with torch.enable_grad():
            leaves = [s.detach().requires_grad_(), weight.detach().requires_grad_(), torch.zeros_like(weight).requires_grad_()]
            y = torch.nn.functional.layer_norm(leaves[0], s.shape[-1:], leaves[1], leaves[2], EPS)
            gx, gw, gb = torch.autograd.grad(y, leaves, grad_y)
        gx = gx if grad_sum is None else gx + grad_sum
        return gx if want_grad_x else None, gw if want_grad_weight else None, gb if want_grad_bias else None

    monkeypatch.setattr(binding, "act8_save", lambda x, fmt: Kept(x.detach()))
    monkeypatch.setattr(binding, "Act8", lambda buffer, *shape: Kept(buffer))
    for f in (linear_fwd, linear_bwd, layernorm_fwd, layernorm_bwd):
        monkeypatch.setattr(binding, f.__name__, f)


def _rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def _mlp_leaves(bias=True):
    return [_rand(1, 6, 8), _rand(2, 6, 8), _rand(3, 12, 8), _rand(4, 12) if bias else None, _rand(5, 8, 12), _rand(6, 8) if bias else None]


def _leaf(t):
    return None if t is None else t.requires_grad_()


def _composed_mlp(x, residual, wu, bu, wd, bd):
    y = torch.nn.functional.linear(torch.nn.functional.silu(torch.nn.functional.linear(x, wu, bu)), wd, bd)
    return y if residual is None else y + residual


@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("stream", [True, False])
def test_first_derivatives_of_the_block(plain, bias, stream):
    leaves = [_leaf(t) for t in _mlp_leaves(bias)]
    if not stream:
        leaves[1] = None
    real = [t for t in leaves if t is not None]
    got = torch.autograd.grad(module._MLP.apply(*leaves, gws.GATED_SILU, gws.ACT8_INT8).pow(2).sum(), real)
    want = torch.autograd.grad(_composed_mlp(*leaves).pow(2).sum(), real)
    for p, q in zip(got, want):
        assert torch.allclose(p, q, rtol=1e-10, atol=1e-10)


@pytest.mark.parametrize("wanted", range(6))
def test_one_derivative_of_the_block_alone(plain, wanted):
    leaves = _mlp_leaves()
    leaves[wanted].requires_grad_()
    got, = torch.autograd.grad(module._MLP.apply(*leaves, gws.GATED_SILU, gws.ACT8_INT8).pow(2).sum(), leaves[wanted])
    want, = torch.autograd.grad(_composed_mlp(*leaves).pow(2).sum(), leaves[wanted])
    assert torch.allclose(got, want, rtol=1e-10, atol=1e-10)


def _norm_leaves():
    return [_rand(1, 2, 3, 8), _rand(2, 2, 3, 8), _rand(3, 8), _rand(4, 8)]


@pytest.mark.parametrize("use", ["y", "s", "both", "alone"])
def test_first_derivatives_of_the_norm(plain, use):
    x, r, w, b = [_leaf(t) for t in _norm_leaves()]
    if use == "alone":
        r = None
    out = module._LayerNorm.apply(x, r, w, b, EPS)
    s = x if r is None else x + r
    y = torch.nn.functional.layer_norm(s, (8,), w, b, EPS)
    loss = {"y": lambda y, s: y.pow(2).sum(), "s": lambda y, s: s.pow(3).sum(), "both": lambda y, s: (y * s).sum(), "alone": lambda y, s: y.pow(3).sum()}[use]
    real = [t for t in (x, r, w, b) if t is not None]
    got = torch.autograd.grad(loss(*(out if r is not None else (out, None))), real, allow_unused=True)
    want = torch.autograd.grad(loss(y, s), real, allow_unused=True)
    for p, q in zip(got, want):
        assert (p is None and q is None) or torch.allclose(p, q, rtol=1e-9, atol=1e-9)


def test_second_derivatives_are_refused(plain):
    leaves = [_leaf(t) for t in _mlp_leaves()]
    y = module._MLP.apply(*leaves, gws.GATED_SILU, gws.ACT8_INT8)
    grad, = torch.autograd.grad(y.sum(), leaves[0], create_graph=True)
    with pytest.raises(RuntimeError):
        (grad.pow(2).sum() + y.sum()).backward()
    x, r, w, b = [_leaf(t) for t in _norm_leaves()]
    y, s = module._LayerNorm.apply(x, r, w, b, EPS)
    grad, = torch.autograd.grad(y.pow(2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        (grad.pow(2).sum() + y.sum()).backward()


def test_modules_check_their_choices():
    for bad in (dict(keep=gws.SAVE_NONE), dict(activation=gws.ACT_NONE), dict(activation=7)):
        with pytest.raises(ValueError):
            module.GaussWSMLP(32, 64, group=(1, 32), device="cpu", **bad)
    with pytest.raises(ValueError):
        module.GaussWSLayerNorm(8, dtype=torch.float16, device="cpu")
    with pytest.raises(ValueError):
        module.GaussWSLayerNorm(8, device="cpu")(torch.zeros(2, 8), torch.zeros(1, 8))
    block = module.GaussWSMLP(32, 64, group=(1, 32), device="cpu", layer_index=5)
    assert block.layers == [block.up, block.down] and block.up.bias.shape == (64,) and block.down.weight.shape == (32, 64)
    block.advance()
    assert block.up.step == block.down.step == 1


# ---- the optimizer ---------------------------------------------------------------------------------------------------
@pytest.fixture
def recorded(monkeypatch):
    """adamw_step with its arguments written down and a plain step of size lr."""
    calls = []

    def adamw_step(params, grads, state, **more):
        calls.append(dict(grads=[g is not None for g in grads], sizes=state.sizes, **more))
        for p, g in zip(params, grads):
            if g is not None:
                p -= float(more["lr"]) * g.sign()

    monkeypatch.setattr(binding, "adamw_step", adamw_step)
    return calls


def _parameter(*shape, dtype=torch.bfloat16):
    p = torch.nn.Parameter(torch.ones(*shape, dtype=dtype))
    p.grad = torch.ones_like(p)
    return p


def test_groups_that_share_their_rates_are_one_call(recorded):
    a, b, c = _parameter(3, 4), _parameter(5, dtype=torch.float32), _parameter(7)
    optimizer = GaussWSAdamW([dict(params=[a], weight_decay=0.1), dict(params=[b], weight_decay=0.0), dict(params=[c], lr=1e-2)], lr=1e-3)
    optimizer.step()
    assert [(k["grads"], k["lr"], k["weight_decay"], k["step"]) for k in recorded] == [([True, True, False], 1e-3, [0.1, 0.0, 0.01], 1), ([False, False, True], 1e-2, [0.1, 0.0, 0.01], 1)]
    b.grad = None
    scheduler = torch.optim.lr_scheduler.LambdaLR(optimizer, lambda k: 0.5)
    optimizer.step()
    scheduler.step()
    assert recorded[2]["grads"] == [True, False, False] and recorded[2]["lr"] == 0.5e-3 and recorded[2]["step"] == 2
    for p in (a, c):
        p.grad = None
    optimizer.step()
    assert len(recorded) == 4 and optimizer.state_dict()["gws"]["count"] == 2          # nothing to do is no step
    with pytest.raises(RuntimeError):
        optimizer.add_param_group(dict(params=[_parameter(2)]))


def test_closure_and_refusals(recorded):
    p = _parameter(4)
    optimizer = GaussWSAdamW([p], lr=1e-3)
    assert optimizer.step(lambda: 3.0) == 3.0
    for bad in (dict(lr=-1.0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(weight_decay=-0.1), dict(moments=5)):
        with pytest.raises(ValueError):
            GaussWSAdamW([p], **bad)
    with pytest.raises(KeyError):
        optimizer.weight(_parameter(4))
    p.grad = torch.ones(4).to_sparse().to(torch.bfloat16)
    with pytest.raises(RuntimeError):
        optimizer.step()


def test_a_capture_wants_a_count_on_the_device_and_a_step_before(recorded, monkeypatch):
    plain, ready = GaussWSAdamW([_parameter(4)]), GaussWSAdamW([_parameter(4)], capturable=True)
    early = GaussWSAdamW([_parameter(4)], capturable=True)
    plain.step()
    ready.step()
    assert ready._count.dtype == torch.int64 and int(ready._count) == 1
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    for refused in (plain, early):
        with pytest.raises(RuntimeError):
            refused.step()
    ready.step()
    assert int(ready._count) == 2 and recorded[-1]["step"] is ready._count and len(recorded) == 3


@pytest.mark.parametrize("capturable", [False, True])
def test_a_refused_step_does_not_count(recorded, capturable, monkeypatch):
    optimizer = GaussWSAdamW([_parameter(4)], capturable=capturable)
    optimizer.step()

    def refuses(*args, **more):
        raise ValueError

    with monkeypatch.context() as m:
        m.setattr(binding, "adamw_step", refuses)
        with pytest.raises(ValueError):
            optimizer.step()
    assert int(optimizer._count) == 1
    optimizer.step()
    assert int(recorded[-1]["step"]) == 2


def test_a_refused_state_changes_nothing(recorded):
    source, other = GaussWSAdamW([_parameter(300)], lr=2e-3), GaussWSAdamW([_parameter(300)], lr=1e-3, rest=False)
    source.step()
    with pytest.raises(ValueError):
        other.load_state_dict(source.state_dict())
    assert other._count == 0 and other.param_groups[0]["lr"] == 1e-3


@pytest.mark.parametrize("moments", [gws.ADAMW_F32, gws.ADAMW_8BIT])
def test_state_travels(recorded, moments):
    p = _parameter(300)
    optimizer = GaussWSAdamW([p], lr=1e-3, moments=moments)
    optimizer.step()
    state = optimizer._state
    state.moments.random_(0, 100)
    state.rest.random_(-100, 100)
    for other in (pickle.loads(pickle.dumps(optimizer)), copy.deepcopy(optimizer)):
        assert other._count == 1 and torch.equal(other._state.moments, state.moments) and torch.equal(other._state.rest, state.rest)
        assert other._state._c.moments == other._state.moments.data_ptr() != state.moments.data_ptr()
    fresh = GaussWSAdamW([_parameter(300)], lr=5.0, moments=moments)
    fresh.load_state_dict(optimizer.state_dict())
    assert fresh._count == 1 and fresh.param_groups[0]["lr"] == 1e-3 and torch.equal(fresh._state.moments, state.moments) and torch.equal(fresh._state.rest, state.rest)
    assert (fresh._state.units is None) == (moments == gws.ADAMW_F32)
    for wrong in (GaussWSAdamW([_parameter(301)], moments=moments), GaussWSAdamW([_parameter(300)], moments=1 - moments), GaussWSAdamW([_parameter(300)], moments=moments, rest=False)):
        with pytest.raises(ValueError):
            wrong.load_state_dict(optimizer.state_dict())
    with pytest.raises(ValueError):
        fresh.load_state_dict(torch.optim.AdamW([_parameter(300)]).state_dict())


def test_layout_of_the_state():
    state = gws.AdamWState([1, 256, 257, 0, 300], gws.ADAMW_8BIT, rest=True, device="cpu")
    assert state.starts == (0, 256, 512, 1024, 1024) and state.total == 1536
    assert state.moments.shape == (2, 1536) and state.moments.dtype == torch.uint8 and state.units.shape == (2, 6) and state.rest.shape == (1536,)
    with pytest.raises(AttributeError):
        state.moments = state.moments.clone()              # the address is kept
    flat = gws.AdamWState([5], device="cpu")
    assert flat.moments.shape == (2, 256) and flat.units is None and flat.rest is None
    assert [t.shape for t in flat.values()] == [(256,), (256,)]
    p = torch.tensor([1.0, -2.0], dtype=torch.bfloat16)
    kept = gws.AdamWState([2], rest=True, device="cpu")
    kept.rest[:2] = torch.tensor([5, -7])
    ulp = 2.0 ** -23
    assert torch.equal(kept.weight(0, p), torch.tensor([1 + 5 * ulp, -2 + 7 * ulp]))       # below a power of two the numbers are twice as dense
    for call in (lambda: gws.AdamWState([5], 3), lambda: gws.AdamWState([-1], device="cpu"), lambda: gws.AdamWState([5], moments=torch.zeros(2, 255)),
                 lambda: gws.AdamWState([5], units=torch.zeros(2, 1), device="cpu")):
        with pytest.raises(ValueError):
            call()
