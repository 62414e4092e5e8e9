"""The state of the AdamW step and its optimizer on the CPU: the calls that they refuse, and states that are loaded."""
import weakref

import pytest
import torch

import paper_2505_11170_b200 as gws
from paper_2505_11170_b200 import binding
from paper_2505_11170_b200.optimizer import GaussWSAdamW


@pytest.fixture
def recorded(monkeypatch):
    """adamw_step with its arguments written down, and nothing done."""
    calls = []
    monkeypatch.setattr(binding, "adamw_step", lambda params, grads, state, **more: calls.append(dict(grads=[g is not None for g in grads], **more)))
    return calls


def _parameter(*shape, dtype=torch.bfloat16):
    p = torch.nn.Parameter(torch.ones(*shape, dtype=dtype))
    p.grad = torch.ones_like(p)
    return p


def _rate(value):
    return torch.full((1,), value)


def _two_groups(first, second, **more):
    return GaussWSAdamW([dict(params=[_parameter(300)], lr=first), dict(params=[_parameter(7)], lr=second)], **more)


def _tensors(fmt, device):
    bits8 = fmt == gws.ADAMW_8BIT
    return dict(moments=torch.zeros(2, 768, dtype=torch.uint8 if bits8 else torch.float32, device=device), units=torch.zeros(2, 3, device=device) if bits8 else None,
                rest=torch.zeros(768, dtype=torch.int16, device=device))


@pytest.mark.parametrize("fmt", [gws.ADAMW_F32, gws.ADAMW_8BIT])
def test_the_tensors_of_a_state_live_on_one_device(fmt):
    """A kernel reads them all by address, and is launched on the device of the moments."""
    here, there = _tensors(fmt, "cpu"), _tensors(fmt, "meta")
    gws.AdamWState([300, 40], fmt, **here)
    for name in ("units", "rest"):
        if here[name] is not None:
            with pytest.raises(ValueError, match="one device"):
                gws.AdamWState([300, 40], fmt, **{**here, name: there[name]})
    with pytest.raises(ValueError, match="one device"):
        gws.AdamWState([300, 40], fmt, device="cpu", rest=there["rest"])


def test_a_loaded_rate_goes_where_the_present_one_is(recorded):
    """A captured step reads a rate on the device by its address."""
    source, shared = _two_groups(5e-4, _rate(2e-3)), _rate(1e-3)
    source.step()
    optimizer = _two_groups(_rate(1e-3), _rate(1e-3), capturable=True)
    optimizer.step()
    held = [g["lr"] for g in optimizer.param_groups]
    optimizer.load_state_dict(source.state_dict())
    assert [g["lr"] for g in optimizer.param_groups] == held and all(g["lr"] is lr for g, lr in zip(optimizer.param_groups, held))
    assert torch.equal(held[0], _rate(5e-4)) and torch.equal(held[1], _rate(2e-3))
    source.param_groups[1]["lr"].fill_(9.0)                   # the loaded one is a copy
    optimizer.step()
    assert [c["lr"] for c in recorded[-2:]] == held and torch.equal(held[1], _rate(2e-3))
    # one tensor for both groups stays one where both take the same
    alike = _two_groups(3e-3, 3e-3)
    optimizer = _two_groups(shared, shared, capturable=True)
    optimizer.step()
    optimizer.load_state_dict(alike.state_dict())
    assert all(g["lr"] is shared for g in optimizer.param_groups) and torch.equal(shared, _rate(3e-3))


def test_rates_that_a_shared_tensor_cannot_hold(recorded):
    source, shared = _two_groups(5e-4, 2e-3), _rate(1e-3)
    source.step()
    optimizer = _two_groups(shared, shared, capturable=True)
    optimizer.step()
    with pytest.raises(ValueError):
        optimizer.load_state_dict(source.state_dict())
    assert torch.equal(shared, _rate(1e-3)) and int(optimizer._count) == 1 and all(g["lr"] is shared for g in optimizer.param_groups)
    fresh = _two_groups(shared, shared)                       # no captured step can know of it: each group its own
    fresh.load_state_dict(source.state_dict())
    assert fresh.param_groups[0]["lr"] is shared and [float(g["lr"]) for g in fresh.param_groups] == [float(_rate(5e-4)), float(_rate(2e-3))]
    state = source.state_dict()
    state["param_groups"][0]["lr"] = torch.ones(2)
    with pytest.raises(ValueError):
        fresh.load_state_dict(state)


def test_a_loaded_rate_beside_the_parameters(recorded):
    """Where the present rate is a number: a tensor stays one, of FP32 and shared as it was."""
    shared = torch.full((1,), 2e-3, dtype=torch.float64)
    source, optimizer = _two_groups(shared, shared), _two_groups(1e-3, 1e-3)
    optimizer.load_state_dict(source.state_dict())
    rates = [g["lr"] for g in optimizer.param_groups]
    assert rates[0] is rates[1] and rates[0].dtype == torch.float32 and rates[0].device == optimizer.param_groups[0]["params"][0].device
    optimizer.step()
    assert len(recorded) == 1


@pytest.mark.parametrize("capturable", [False, True])
def test_a_step_is_refused_as_a_whole(recorded, capturable):
    """Groups of different rates are calls of their own: none is made where one would be refused."""
    optimizer = _two_groups(1e-3, 2e-3, capturable=capturable)
    optimizer.step()
    recorded.clear()
    second = optimizer.param_groups[1]
    strided = torch.nn.Parameter(torch.ones(4, 14, dtype=torch.bfloat16)[:, ::2])
    strided.grad = torch.ones(4, 7, dtype=torch.bfloat16)
    for wrong in (dict(lr=torch.ones(1, dtype=torch.float64)), dict(lr=torch.ones(2)), dict(lr="fast"), dict(betas=(0.9,)), dict(params=[strided])):
        present = {k: second[k] for k in wrong}
        second.update(wrong)
        with pytest.raises((ValueError, TypeError, IndexError)):
            optimizer.step()
        second.update(present)
        assert not recorded and int(optimizer._count) == 1
    optimizer.step()
    assert [(c["grads"], int(c["step"])) for c in recorded] == [([True, False], 2), ([False, True], 2)]


@pytest.mark.parametrize("capturable", [False, True])
def test_a_launch_that_fails_in_the_middle_of_a_step(recorded, capturable, monkeypatch):
    """The groups before it have been stepped, so the step counts: they are not stepped under the same count again."""
    optimizer = _two_groups(1e-3, 2e-3, capturable=capturable)
    optimizer.step()
    taken = binding.adamw_step

    def fails(params, grads, state, **more):
        if more["lr"] == 2e-3:
            raise RuntimeError
        taken(params, grads, state, **more)

    with monkeypatch.context() as m:
        m.setattr(binding, "adamw_step", fails)
        with pytest.raises(RuntimeError):
            optimizer.step()
    assert int(optimizer._count) == 2


def test_check_of_a_step():
    """What adamw_step refuses, but that the tensors are on the CPU."""
    p, g, state = torch.ones(300), torch.ones(300), gws.AdamWState([300], device="cpu")
    gws.adamw_check([p], [g], state, lr=1e-3)
    for call in (lambda: gws.adamw_check([p], [g, g], state, lr=1e-3), lambda: gws.adamw_check([p[:299]], [g[:299]], state, lr=1e-3), lambda: gws.adamw_check([p], [g.half()], state, lr=1e-3),
                 lambda: gws.adamw_check([torch.ones(600)[::2]], [g], state, lr=1e-3), lambda: gws.adamw_check([p], [g], state, lr=1e-3, weight_decay=[0.1, 0.1]),
                 lambda: gws.adamw_check([p], [g], state, lr=1e-3, grad_scale=0.5), lambda: gws.adamw_check([p], [g], state, lr=1e-3, step=torch.ones(1))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        gws.adamw_step([p], [g], state, lr=1e-3)


def test_the_weight_of_a_parameter_set_to_zero_from_outside():
    """A zero over a negative rest, which no step leaves, counts as zero, as the step takes it; its bits joined would be a NaN's."""
    state = gws.AdamWState([6], rest=True, device="cpu")
    state.rest[:6] = torch.tensor([-3, -3, 4, 0, -5, -5], dtype=torch.int16)
    p = torch.tensor([0.0, -0.0, 0.0, -0.0, 1.0, -1.0], dtype=torch.bfloat16)
    below = 1 - 5 * 2.0 ** -24                                 # under a power of two the numbers are twice as dense
    want = torch.tensor([0.0, -0.0, 4 * 2.0 ** -149, -0.0, below, -below])
    got = state.weight(0, p)
    assert torch.equal(got.view(torch.int32), want.view(torch.int32))
    assert state.weight(0, p.view(2, 3)).shape == (2, 3)


def test_a_loaded_rate_of_a_group_without_parameters(recorded):
    groups = lambda lr: [dict(params=[]), dict(params=[_parameter(300)], lr=lr)]
    source, optimizer = GaussWSAdamW(groups(_rate(1e-3)), lr=_rate(2e-3)), GaussWSAdamW(groups(5e-4), lr=5e-4)
    optimizer.load_state_dict(source.state_dict())
    assert [float(g["lr"]) for g in optimizer.param_groups] == [float(_rate(2e-3)), float(_rate(1e-3))]


def test_a_check_is_of_its_own_arguments():
    """adamw_step takes addresses from it: of tensors that it holds, and for the same ones alone."""
    made = lambda: ([torch.ones(300), torch.ones(7)], [torch.ones(300), None], gws.AdamWState([300, 7], device="cpu"))
    (p, g, state), (q, h, other) = made(), made()
    checked = gws.adamw_check(p, g, state, lr=1e-3, step=5)
    for call in (lambda: gws.adamw_step(q, g, state, lr=1e-3, step=5, checked=checked), lambda: gws.adamw_step(p, h, state, lr=1e-3, step=5, checked=checked),
                 lambda: gws.adamw_step(p, g, other, lr=1e-3, step=5, checked=checked), lambda: gws.adamw_step(p, g, state, lr=1e-3, step=torch.ones(1), checked=checked),
                 lambda: gws.adamw_step(p[:1], g[:1], state, lr=1e-3, step=5, checked=checked)):
        with pytest.raises(ValueError, match="other arguments"):
            call()
    with pytest.raises(ValueError, match="device pointers"):                  # as without it
        gws.adamw_step(p, g, state, lr=float("1e-3"), step=5, checked=checked)
    held = weakref.ref(p[0])
    p[0] = q[0]
    assert held() is not None
