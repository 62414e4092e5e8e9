"""States of GaussWSAdamW that are loaded between replays of a captured step."""
import copy

import numpy as np
import pytest
import torch

import paper_2505_11170_b200 as gws
from paper_2505_11170_b200.optimizer import GaussWSAdamW

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _optimizer(rate, capturable, moments):
    torch.manual_seed(8)
    params = [torch.nn.Parameter(torch.randn(n, device=DEV).to(t)) for n, t in ((1000, torch.bfloat16), (77, torch.float32))]
    for p in params:
        p.grad = torch.randn_like(p)
    return params, GaussWSAdamW(params, lr=torch.full((1,), rate, device=DEV) if capturable else rate, capturable=capturable, weight_decay=0.0, moments=moments)


@pytest.mark.parametrize("moments", [gws.ADAMW_F32, gws.ADAMW_8BIT])
def test_a_captured_step_goes_on_from_a_loaded_state(moments):
    (p, o), (q, e) = _optimizer(1e-3, True, moments), _optimizer(1e-3, True, moments)
    o.step()
    e.step()
    weights, kept = [t.detach().clone() for t in p], copy.deepcopy(o.state_dict())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o.step()
    graph.replay()
    for where in ("cuda", "cpu"):
        there = copy.deepcopy(kept)
        there["param_groups"][0]["lr"] = kept["param_groups"][0]["lr"].to(where) * 2
        there["gws"]["state"] = {k: t.to(where) if isinstance(t, torch.Tensor) else t for k, t in kept["gws"]["state"].items()}
        o.load_state_dict(there)
        e.load_state_dict(there)
        with torch.no_grad():
            for a, b, w in zip(p, q, weights):
                a.copy_(w)
                b.copy_(w)
        rate = e.param_groups[0]["lr"]
        assert rate.device.type == "cuda" and float(rate) == float(np.float32(1e-3) * 2)
        for factor in (1.0, 0.5):
            o.param_groups[0]["lr"].mul_(factor)
            rate.mul_(factor)
            graph.replay()
            e.step()
            torch.cuda.synchronize()
            for a, b in zip(p, q):
                assert torch.equal(a, b) and torch.equal(o.weight(a), e.weight(b))
        assert o.state_dict()["gws"]["count"] == e.state_dict()["gws"]["count"] == 3
        assert torch.equal(o._state.moments, e._state.moments)


def test_a_step_of_several_groups_is_refused_as_a_whole():
    a, b = (torch.nn.Parameter(torch.ones(300, dtype=torch.bfloat16, device=DEV)) for _ in range(2))
    optimizer = GaussWSAdamW([dict(params=[a], lr=1e-3), dict(params=[b], lr=2e-3)])
    a.grad, b.grad = torch.ones_like(a), torch.ones_like(b)
    optimizer.step()
    tensors = [a, b, optimizer._state.moments, optimizer._state.rest]
    before = [t.detach().clone() for t in tensors]
    second, launches = optimizer.param_groups[1], gws.launch_count()
    for wrong in (dict(betas=(1.0, 0.9)), dict(betas=(0.9, float("nan"))), dict(eps=-1.0), dict(lr=torch.ones(1)), dict(lr=torch.ones(1, dtype=torch.float64, device=DEV))):
        present = {k: second[k] for k in wrong}
        second.update(wrong)
        with pytest.raises((ValueError, gws.GwsError)):
            optimizer.step()
        second.update(present)
    grad, b.grad = b.grad, b.detach()                          # a gradient that is the parameter itself
    with pytest.raises(gws.GwsError):
        optimizer.step()
    b.grad = grad
    assert gws.launch_count() == launches and all(torch.equal(t, u) for t, u in zip(tensors, before))
    optimizer.step()
    assert optimizer.state_dict()["gws"]["count"] == 2 and gws.launch_count() == launches + 2


@pytest.mark.parametrize("on_side", [False, True])
def test_a_checked_step_is_the_step(on_side):
    """On the stream of the call, with gradients that need a copy, and places without one."""
    def made(seed):
        torch.manual_seed(seed)
        params = [torch.randn(40, 30, device=DEV), torch.randn(300, device=DEV).bfloat16(), torch.randn(7, device=DEV)]
        return params, [torch.randn(30, 40, device=DEV).t(), torch.randn(300, device=DEV).bfloat16(), None], gws.AdamWState([1200, 300, 7], gws.ADAMW_8BIT, rest=True)

    (p, g, s), (q, h, t) = made(1), made(1)
    more = dict(lr=torch.full((1,), 1e-3, device=DEV), step=3, grad_scale=torch.full((1,), 0.5, device=DEV))
    launches = gws.launch_count()
    checked = gws.adamw_check(p, g, s, **more)
    assert gws.launch_count() == launches
    side = torch.cuda.Stream() if on_side else None
    if on_side:
        side.wait_stream(torch.cuda.current_stream())
    gws.adamw_step(p, g, s, **more, checked=checked, stream=side)
    gws.adamw_step(q, h, t, **more)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*p, s.moments, s.units, s.rest), (*q, t.moments, t.units, t.rest)))
