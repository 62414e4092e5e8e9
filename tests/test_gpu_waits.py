"""What follows when a wait inside the block GEMM runs out: with a limit of a few cycles a sound launch gives up (its epilogue asks for the
first tile long before a contraction of many steps is through), reports it, and leaves the device and every later call as they were."""
import contextlib
import time

import pytest
import torch

import paper_2505_11170_b200 as gws
from paper_2505_11170_b200.module import GaussWSGatedMLP
from test_tilings import _path

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


# Contractions (or parts of one) of 64 stages and more: 30,000 cycles and more to the first finished tile, against the 16,000 or so that two
# tries of a wait take.
# forward: (path, m, n, k, what is kept)
FORWARD = [((1, "narrow", "whole"), 2, 4096, 16384, gws.SAVE_NONE), ((1, 128, "cut"), 16, 2048, 65536, gws.ACT8_INT8),
           ((1, 128, "whole"), 128, 9472, 8192, gws.ACT8_E4M3), ((2, 128, "cut"), 1, 64, 262144, gws.ACT8_INT8),
           ((2, 256, "whole+cut"), 700, 4096, 16384, gws.ACT8_E4M3), ((2, 256, "whole*"), 2100, 2048, 16384, gws.SAVE_BF16),
           ((2, 256, "whole*"), 300, 9000, 8192, gws.ACT8_INT8)]


@pytest.mark.parametrize("path,m,n,k,save", FORWARD)
def test_forward(path, m, n, k, save):
    assert _path(gws.gated_plan(m, n, k, "h", save=save)) == path
    x, wg, wu = _rand(m, k, 1), _rand(n, k, 2, 0.01), _rand(n, k, 3, 0.01)
    want = gws.gated_fwd(x, wg, wu, save=save)[0]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    t = time.perf_counter()
    with _no_patience():
        gws.gated_fwd(x, wg, wu, save=save, status=status)
    assert int(status) == 1 and time.perf_counter() - t < 5.0
    status.zero_()
    assert torch.equal(gws.gated_fwd(x, wg, wu, save=save, status=status)[0], want) and int(status) == 0


# backward: (product, path, m, n, k, format of x and of what is kept)
BACKWARD = [("grad_x", (1, 128, "cluster"), 1, 8359, 6280, gws.ACT8_INT8), ("grad_x", (1, 128, "cut"), 1, 98304, 648, gws.ACT8_E4M3),
            ("grad_x", (2, 128, "whole"), 300, 8047, 3728, gws.SAVE_BF16), ("grad_x", (2, 256, "whole+cut"), 16384, 4096, 1024, gws.ACT8_E4M3),
            ("grad_w", (2, 256, "whole*"), 16384, 4096, 1024, gws.ACT8_E4M3), ("grad_w", (2, 256, "cut"), 65536, 520, 520, gws.SAVE_BF16)]


@pytest.mark.parametrize("product,path,m,n,k,fmt", BACKWARD)
def test_backward(product, path, m, n, k, fmt):
    assert _path(gws.gated_plan(m, n, k, product, x_format=fmt)) == path
    x, wg, wu, dh = _rand(m, k, 1), _rand(n, k, 2, 0.05), _rand(n, k, 3, 0.05), _rand(m, n, 4, 0.01)
    _, saved = gws.gated_fwd(x, wg, wu, save=fmt)
    x_in = x if fmt == gws.SAVE_BF16 else gws.act8_save(x, fmt)
    call = lambda status: gws.gated_bwd(dh, x_in, wg, wu, saved, want_grad_x=product == "grad_x", want_grad_w=product == "grad_w", status=status)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    want = call(status)
    assert int(status) == 0
    with _no_patience():
        call(status)
    assert int(status) == 1
    status.zero_()
    assert all(p is q is None or torch.equal(p, q) for p, q in zip(call(status), want)) and int(status) == 0


# a layer's weight gradient, X converted inside the product or restored before it: (path, inside, m, n, k)
WGRAD = [((1, 128, "cut"), True, 74240, 8, 1851), ((2, 128, "cut"), True, 262144, 12, 250), ((2, 256, "cut"), True, 16384, 512, 2048),
         ((2, 256, "cut*"), True, 65536, 536, 1256), ((2, 256, "whole"), False, 32768, 2048, 2048)]


@pytest.mark.parametrize("path,inside,m,n,k", WGRAD)
def test_weight_gradient(path, inside, m, n, k):
    plan = gws.wgrad_act8_plan(m, n, k)
    assert (_path(plan), bool(plan.inside)) == (path, inside)
    gy, a = _rand(m, n, 1, 1e-3), gws.act8_save(_rand(m, k, 2))
    want = gws.wgrad_act8(gy, a)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    with _no_patience():
        gws.wgrad_act8(gy, a, status=status)
    assert int(status) == 1
    assert torch.equal(gws.wgrad_act8(gy, a), want)


def test_calls_without_a_status_word_raise_afterwards():
    x, w = _rand(2100, 16384, 1), _rand(2048, 16384, 2, 0.01)
    want = gws.gated_fwd(x, w, w)[0]
    gws.check_waits()
    with _no_patience():
        gws.gated_fwd(x, w, w)
    with pytest.raises(gws.GwsError):
        gws.check_waits()
    gws.check_waits()                                     # reported once
    with _no_patience():
        gws.gated_fwd(x, w, w)
    with pytest.raises(gws.GwsError):
        gws.gated_fwd(x, w, w)
    assert torch.equal(gws.gated_fwd(x, w, w)[0], want)
    gws.check_waits()


def test_a_training_step_of_the_module_raises():
    block = GaussWSGatedMLP(16384, 2048)
    x = _rand(2100, 16384, 1).requires_grad_()
    with _no_patience():
        block(x)
    with pytest.raises(gws.GwsError):
        block.advance()
    block(x).sum().backward()
    gws.check_waits()
    block.advance()
