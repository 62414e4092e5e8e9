"""Argument checks of the linear layer's C entry points: host arithmetic on pointers and sizes, nothing is launched."""
import ctypes

import pytest

import paper_2505_11170_b200 as gws
from paper_2505_11170_b200 import _build, binding
from paper_2505_11170_b200.binding import LinearDesc

P = [0x10000000 + 0x4000000 * i for i in range(14)]      # never dereferenced: every call below fails validation
M, N, K = 100, 72, 64


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return gws.load_library()


def desc(m=M, n=N, k=K, ld_x=K, ld_w=K, ld_y=N, ld_r=N, act=0, save=0, x_format=2, bias_type=0):
    return LinearDesc(m, n, k, ld_x, ld_w, ld_y, ld_r, act, save, x_format, bias_type)


def test_sizes_and_kinds(lib):
    size = lambda backward=0, **k: lib.gws_linear_workspace_bytes(ctypes.byref(desc(**k)), backward)
    assert size() >= 0 and size(1) > 0 and size(m=0) == size(n=0) == size(1, m=0) == 0
    assert size(m=-1) == size(k=0) == size(k=-1) == size(ld_x=K - 1) == size(ld_w=K - 1) == size(ld_y=N - 1) == size(ld_r=-1) == binding.ERR_SHAPE
    assert size(m=1 << 31) == size(ld_x=1 << 31) == binding.ERR_LIMIT
    assert size(act=4) == size(act=-1) == size(bias_type=2) == binding.ERR_UNSUPPORTED
    assert lib.gws_linear_workspace_bytes(None, 0) == binding.ERR_NULL
    plan = binding.ProductPlan()
    assert lib.gws_linear_plan(ctypes.byref(desc()), 3, ctypes.byref(plan)) == binding.ERR_UNSUPPORTED
    assert lib.gws_linear_plan(ctypes.byref(desc()), 0, None) == binding.ERR_NULL
    for product in ("y", "grad_x", "grad_w"):
        p = gws.linear_plan(M, N, K, product)
        assert p.whole + p.cut > 0


def test_forward_validates_before_any_launch(lib):
    before = gws.launch_count()
    need = lib.gws_linear_workspace_bytes(ctypes.byref(desc(ld_x=K + 1)), 0)
    assert need > 0

    def fwd(x=P[0], w=P[1], b=P[2], r=P[3], y=P[4], s=P[5], ws=P[6], nbytes=need, status=None, **k):
        return lib.gws_linear_fwd(ctypes.byref(desc(**{"ld_x": K + 1, **k})), x, w, b, r, y, s, ws, nbytes, status, None)

    assert fwd(save=4) == binding.ERR_UNSUPPORTED and fwd(ld_r=N - 1) == binding.ERR_SHAPE
    assert fwd(x=None) == fwd(w=None) == fwd(y=None) == fwd(s=None) == binding.ERR_NULL
    assert fwd(x=P[0] + 1) == fwd(ld_x=K + 8, x=P[0] + 2) == fwd(w=P[1] + 2) == fwd(y=P[4] + 1) == fwd(s=P[5] + 16) == fwd(b=P[2] + 2, bias_type=1) == fwd(r=P[3] + 1) == \
        fwd(status=P[7] + 2) == binding.ERR_ALIGN
    assert fwd(y=P[0]) == fwd(y=P[3]) == fwd(s=P[4]) == fwd(y=P[2] - 64) == fwd(ws=P[1]) == fwd(ws=P[4]) == binding.ERR_ALIAS
    assert fwd(ws=None) == fwd(nbytes=need - 1) == fwd(ws=P[6] + 64) == binding.ERR_WORKSPACE
    assert fwd(m=0, x=None, y=None) == binding.OK
    assert gws.launch_count() == before


def test_backward_validates_before_any_launch(lib):
    before = gws.launch_count()
    need = lib.gws_linear_workspace_bytes(ctypes.byref(desc()), 1)

    def bwd(dy=P[0], x=P[1], w=P[2], s=P[3], dx=P[4], dw=P[5], db=P[6], a=P[7], ws=P[8], nbytes=need, status=None, **k):
        return lib.gws_linear_bwd(ctypes.byref(desc(**k)), dy, x, w, s, dx, dw, db, a, ws, nbytes, status, None)

    assert bwd(save=3) == bwd(save=7) == bwd(x_format=3) == bwd(act=3, save=3) == binding.ERR_UNSUPPORTED
    assert bwd(dy=None) == bwd(x=None) == bwd(w=None) == bwd(s=None) == bwd(dw=None, dx=None, dy=None) == bwd(act=3, s=None) == binding.ERR_NULL
    assert bwd(dy=P[0] + 1) == bwd(act=3, save=3, a=None, dy=P[0] + 2) == bwd(x=P[1] + 2) == bwd(w=P[2] + 8) == bwd(s=P[3] + 8) == bwd(dx=P[4] + 1) == bwd(dw=P[5] + 1) == \
        bwd(db=P[6] + 2, bias_type=1) == bwd(a=P[7] + 1) == bwd(x_format=0, x=P[1] + 16) == binding.ERR_ALIGN
    assert bwd(dx=P[0]) == bwd(dw=P[1]) == bwd(db=P[2]) == bwd(a=P[3]) == bwd(dx=P[5]) == bwd(ws=P[3]) == bwd(a=P[8]) == binding.ERR_ALIAS
    assert bwd(ws=None) == bwd(nbytes=need - 1) == bwd(ws=P[8] + 128) == binding.ERR_WORKSPACE
    assert bwd(dx=None, dw=None, db=None, a=None) == binding.OK
    assert gws.launch_count() == before
