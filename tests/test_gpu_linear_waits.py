"""What follows when a wait inside the linear layer's products runs out: with a limit of a few cycles a sound launch gives up, reports it, and leaves the device and every later
call as they were."""
import contextlib

import pytest
import torch

import paper_2505_11170_b200 as gws
from paper_2505_11170_b200.module import GaussWSMLP

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _rand(rows, cols, seed, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(rows, cols, generator=g, device=DEV) * std).to(torch.bfloat16)


@contextlib.contextmanager
def _no_patience():
    assert gws.set_wait_limit(1) == 2_000_000_000
    try:
        yield
    finally:
        torch.cuda.synchronize()
        assert gws.set_wait_limit(0) == 1


def _path(p):
    return p.blocks, p.columns, "cluster" if p.clustered else "whole+cut" if p.cut and p.whole else "cut" if p.cut else "whole*" if p.waves > 1 else "whole"


# Contractions (or parts of one) of 64 stages and more: 30,000 cycles and more to the first finished tile, against the 16,000 or so that two tries of a wait take.
FORWARD = [((1, 128, "cluster"), 5, 2048, 32768, gws.ACT8_INT8), ((1, 128, "cut"), 70, 2048, 131072, gws.ACT8_E4M3), ((2, 256, "whole*"), 2100, 4096, 16384, gws.SAVE_BF16),
           ((2, 256, "whole*"), 2100, 4096, 16384, gws.ACT8_INT8), ((2, 256, "whole+cut"), 1500, 4096, 16384, gws.ACT8_INT8)]


@pytest.mark.parametrize("path,m,n,k,save", FORWARD)
def test_forward(path, m, n, k, save):
    assert _path(gws.linear_plan(m, n, k)) == path
    x, w, b, r = _rand(m, k, 1), _rand(n, k, 2, 0.01), _rand(1, n, 3)[0], _rand(m, n, 4)
    call = lambda status: gws.linear_fwd(x, w, b, residual=r, activation=gws.GATED_GELU_TANH, save=save, status=status)[0]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    want = call(status)
    assert int(status) == 0
    with _no_patience():
        call(status)
    assert int(status) == 1
    status.zero_()
    assert torch.equal(call(status), want) and int(status) == 0


def test_a_training_step_of_the_module_raises():
    block = GaussWSMLP(16384, 2048)
    x = _rand(2100, 16384, 1).requires_grad_()
    with _no_patience():
        with pytest.raises(gws.GwsError):                       # by the block's second product at the earliest, by advance at the latest
            block(x)
            torch.cuda.synchronize()
            block.advance()
    with contextlib.suppress(gws.GwsError):                     # what the second product may have reported after that
        gws.check_waits()
    block(x).sum().backward()
    gws.check_waits()
    block.advance()
