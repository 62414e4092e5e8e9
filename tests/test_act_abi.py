"""Argument checks of the activation operators' C entry points: host arithmetic on pointers and sizes, nothing is launched."""
import ctypes

import pytest

import paper_2505_11170_b200 as gws
from paper_2505_11170_b200 import _build, binding
from paper_2505_11170_b200.binding import GatedDesc

P = [0x10000000 + 0x4000000 * i for i in range(14)]      # never dereferenced: every call below fails validation


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return gws.load_library()


def test_checkpoint_layout(lib):
    assert gws.act8_layout(1, 32) == (32, 256, 257)
    assert gws.act8_layout(5, 33) == (320, 512, 522)
    assert gws.act8_layout(0, 64) == (0, 0, 0)
    assert gws.act8_layout(16384, 5632) == (16384 * 5632, 16384 * 5632, 16384 * 5632 // 32 * 33)
    for rows, cols in ((1, 1), (7, 31), (64, 2730), (3, 0)):
        assert gws.act8_layout(rows, cols)[2] == binding._act8_bytes(rows, cols)
    with pytest.raises(gws.GwsError):
        gws.act8_layout(-1, 4)


def test_save_and_load_validate_before_any_launch(lib):
    before = gws.launch_count()
    save, load = lib.gws_act8_save, lib.gws_act8_load
    assert save(4, 64, 64, 2, P[0], P[1], None) == binding.ERR_UNSUPPORTED
    assert save(-1, 64, 64, 0, P[0], P[1], None) == binding.ERR_SHAPE
    assert save(4, 64, 63, 0, P[0], P[1], None) == binding.ERR_SHAPE
    assert save(4, 1 << 31, 1 << 31, 0, P[0], P[1], None) == binding.ERR_LIMIT
    assert save(4, 64, 64, 0, None, P[1], None) == binding.ERR_NULL
    assert save(4, 64, 64, 0, P[0], None, None) == binding.ERR_NULL
    assert save(4, 64, 64, 0, P[0] + 1, P[1], None) == binding.ERR_ALIGN
    assert save(4, 64, 64, 0, P[0], P[1] + 16, None) == binding.ERR_ALIGN
    assert save(4, 64, 64, 0, P[0], P[0] + 256, None) == binding.ERR_ALIAS
    assert load(4, 64, 64, 0, P[0], P[0] + 256, None) == binding.ERR_ALIAS
    assert load(4, 64, 64, 0, P[0], None, None) == binding.ERR_NULL
    assert save(0, 64, 64, 0, None, None, None) == binding.OK
    assert gws.launch_count() == before


def test_weight_gradient_validates_before_any_launch(lib):
    before = gws.launch_count()
    need = lib.gws_wgrad_act8_workspace_bytes(100, 33, 64, 33)
    assert need > 0 and lib.gws_wgrad_act8_workspace_bytes(-1, 1, 1, 1) == binding.ERR_SHAPE

    def call(m=100, n=33, k=64, fmt=0, gy=P[0], ld_y=33, x8=P[1], gw=P[2], ld_w=64, ws=P[3], nbytes=need, status=None):
        return lib.gws_wgrad_act8(m, n, k, fmt, gy, ld_y, x8, gw, ld_w, ws, nbytes, status, None)

    assert call(fmt=2) == binding.ERR_UNSUPPORTED
    assert call(ld_y=32) == binding.ERR_SHAPE and call(ld_w=63) == binding.ERR_SHAPE and call(n=-3) == binding.ERR_SHAPE
    assert call(gy=None) == binding.ERR_NULL and call(x8=None) == binding.ERR_NULL and call(gw=None) == binding.ERR_NULL
    assert call(gy=P[0] + 1) == binding.ERR_ALIGN and call(x8=P[1] + 8) == binding.ERR_ALIGN and call(ld_y=40, gy=P[0] + 2) == binding.ERR_ALIGN
    assert call(gw=P[0]) == binding.ERR_ALIAS and call(ws=P[1]) == binding.ERR_ALIAS and call(gw=P[3] + 64) == binding.ERR_ALIAS
    assert call(ws=None) == binding.ERR_WORKSPACE and call(nbytes=need - 1) == binding.ERR_WORKSPACE and call(ws=P[3] + 16) == binding.ERR_WORKSPACE
    assert call(n=0) == binding.OK and call(k=0) == binding.OK
    assert gws.launch_count() == before


def _desc(**kw):
    base = dict(m=100, n=96, k=64, ld_x=64, ld_w=64, ld_h=96, activation=0, save=0, x_format=2)
    base.update(kw)
    return GatedDesc(base["m"], base["n"], base["k"], base["ld_x"], base["ld_w"], base["ld_h"], base["activation"], base["save"], base["x_format"], 0)


def _fwd(lib, d, x=P[0], wg=P[1], wu=P[2], h=P[3], sg=P[4], su=P[5], ws=P[6], nbytes=1 << 25, status=None):
    return lib.gws_gated_fwd(ctypes.addressof(d), x, wg, wu, h, sg, su, ws, nbytes, status, None)


def _bwd(lib, d, dh=P[0], x=P[1], wg=P[2], wu=P[3], sg=P[4], su=P[5], gx=P[6], gg=P[7], gu=P[8], h=P[9], ws=P[10], nbytes=1 << 25, status=None):
    return lib.gws_gated_bwd(ctypes.addressof(d), dh, x, wg, wu, sg, su, gx, gg, gu, h, ws, nbytes, status, None)


def test_gated_forward_validates_before_any_launch(lib):
    before = gws.launch_count()
    assert lib.gws_gated_fwd(None, *[None] * 7, 0, None, None) == binding.ERR_NULL
    assert _fwd(lib, _desc(m=-1)) == binding.ERR_SHAPE and _fwd(lib, _desc(ld_x=63)) == binding.ERR_SHAPE
    assert _fwd(lib, _desc(ld_w=63)) == binding.ERR_SHAPE and _fwd(lib, _desc(ld_h=95)) == binding.ERR_SHAPE
    assert _fwd(lib, _desc(m=1 << 31)) == binding.ERR_LIMIT
    assert _fwd(lib, _desc(activation=3)) == binding.ERR_UNSUPPORTED and _fwd(lib, _desc(save=4)) == binding.ERR_UNSUPPORTED
    for name in ("x", "wg", "wu", "h", "sg", "su"):
        assert _fwd(lib, _desc(), **{name: None}) == binding.ERR_NULL, name
    for name in ("x", "wg", "wu"):
        assert _fwd(lib, _desc(), **{name: P[12] + 8}) == binding.ERR_ALIGN, name
    assert _fwd(lib, _desc(), h=P[3] + 1) == binding.ERR_ALIGN and _fwd(lib, _desc(), sg=P[4] + 16) == binding.ERR_ALIGN
    assert _fwd(lib, _desc(), status=P[11] + 2) == binding.ERR_ALIGN
    assert _fwd(lib, _desc(), h=P[0]) == binding.ERR_ALIAS and _fwd(lib, _desc(), su=P[4]) == binding.ERR_ALIAS
    assert _fwd(lib, _desc(), sg=P[1] + 32) == binding.ERR_ALIAS and _fwd(lib, _desc(save=2), su=P[3]) == binding.ERR_ALIAS
    odd = _desc(k=63, ld_x=63, ld_w=63)                       # rows a tensor map cannot read: copies in the workspace
    need = lib.gws_gated_workspace_bytes(ctypes.addressof(odd), 0)
    assert need >= 2 * 63 * (100 + 2 * 96)
    assert _fwd(lib, odd, nbytes=need - 1) == binding.ERR_WORKSPACE and _fwd(lib, odd, ws=None) == binding.ERR_WORKSPACE
    assert _fwd(lib, odd, ws=P[6] + 128) == binding.ERR_WORKSPACE and _fwd(lib, odd, ws=P[2]) == binding.ERR_ALIAS
    assert _fwd(lib, _desc(m=0), x=None, wg=None, wu=None, h=None, sg=None, su=None) == binding.OK
    assert gws.launch_count() == before


def test_gated_backward_validates_before_any_launch(lib):
    before = gws.launch_count()
    d = _desc()
    need = lib.gws_gated_workspace_bytes(ctypes.addressof(d), 1)
    assert need >= 2 * 2 * 100 * 96
    assert _bwd(lib, _desc(save=3)) == binding.ERR_UNSUPPORTED and _bwd(lib, _desc(x_format=3)) == binding.ERR_UNSUPPORTED
    for name in ("dh", "x", "wg", "wu", "sg", "su", "gg", "gu"):
        assert _bwd(lib, d, **{name: None}) == binding.ERR_NULL, name
    assert _bwd(lib, d, x=P[1] + 8) == binding.ERR_ALIGN and _bwd(lib, _desc(x_format=0), x=P[1] + 16) == binding.ERR_ALIGN
    assert _bwd(lib, d, dh=P[0] + 1) == binding.ERR_ALIGN and _bwd(lib, d, gx=P[6] + 1) == binding.ERR_ALIGN
    for out in ("gx", "gg", "gu", "h", "ws"):
        for over in (P[0], P[1], P[2], P[4]):
            assert _bwd(lib, d, **{out: over}) == binding.ERR_ALIAS, (out, over)
    assert _bwd(lib, d, gg=P[8]) == binding.ERR_ALIAS and _bwd(lib, d, ws=P[9]) == binding.ERR_ALIAS
    assert _bwd(lib, d, nbytes=need - 1) == binding.ERR_WORKSPACE and _bwd(lib, d, ws=None) == binding.ERR_WORKSPACE
    assert gws.launch_count() == before


def test_library_refusals_come_back_as_errors_of_the_binding():
    import torch

    cpu = torch.zeros(4, 64, dtype=torch.bfloat16)
    for call in (lambda: gws.act8_save(cpu), lambda: gws.gated_fwd(cpu, cpu, cpu), lambda: gws.act8_load(gws.Act8(torch.zeros(1024, dtype=torch.uint8), 4, 64, 0)),
                 lambda: gws.wgrad_act8(cpu, gws.Act8(torch.zeros(1024, dtype=torch.uint8), 4, 64, 0))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        gws.Act8(torch.zeros(100, dtype=torch.uint8), 4, 64, 0)
