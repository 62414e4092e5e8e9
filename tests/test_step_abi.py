"""Argument checks of the C entry points of the layer norm and of the AdamW step: host arithmetic on pointers and sizes, nothing is launched."""
import ctypes

import pytest

import paper_2505_11170_b200 as gws
from paper_2505_11170_b200 import _build, binding
from paper_2505_11170_b200.binding import NormDesc

P = [0x10000000 + 0x4000000 * i for i in range(14)]      # never dereferenced: every call below fails validation


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return gws.load_library()


def test_layer_norm_validates_before_any_launch(lib):
    before = gws.launch_count()

    def fwd(rows=8, cols=64, ld=64, ld_r=64, kind=0, x=P[0], r=P[1], w=P[2], b=P[3], y=P[4], s=P[5], stats=P[6]):
        d = NormDesc(rows, cols, ld, ld_r, 0, 0, kind, 1e-5)
        return lib.gws_layernorm_fwd(ctypes.addressof(d), x, r, w, b, y, s, stats, None)

    assert lib.gws_layernorm_fwd(None, *P[:7], None) == binding.ERR_NULL
    assert fwd(rows=-1) == fwd(cols=-1) == fwd(ld=63) == fwd(ld_r=63) == fwd(ld=-1) == binding.ERR_SHAPE
    assert fwd(rows=1 << 31) == fwd(cols=1 << 31, ld=1 << 31) == fwd(ld=1 << 40) == binding.ERR_LIMIT
    assert fwd(kind=2) == fwd(w=None) == binding.ERR_UNSUPPORTED
    assert fwd(x=None) == fwd(y=None) == fwd(s=None) == binding.ERR_NULL
    assert fwd(x=P[0] + 1) == fwd(r=P[1] + 1) == fwd(w=P[2] + 2, kind=1) == fwd(stats=P[6] + 2) == fwd(y=P[4] + 1) == fwd(s=P[5] + 1) == binding.ERR_ALIGN
    assert fwd(y=P[0]) == fwd(s=P[1] + 1022) == fwd(y=P[5] + 2) == fwd(stats=P[2]) == fwd(stats=P[4] + 1020) == binding.ERR_ALIAS
    assert fwd(rows=0, x=None, y=None) == fwd(cols=0, x=None, y=None) == binding.OK

    d = NormDesc(8, 64, 64, 0, 64, 64, 0, 0.0)
    need = lib.gws_layernorm_workspace_bytes(ctypes.addressof(d))
    assert need > 0 and need % 256 == 0

    def bwd(rows=8, cols=64, ld=64, ld_dy=64, ld_d=64, kind=0, dy=P[0], s=P[1], w=P[2], stats=P[3], g=P[4], dx=P[5], dw=P[6], db=P[7], ws=P[8], nbytes=need):
        d = NormDesc(rows, cols, ld, 0, ld_dy, ld_d, kind, 0.0)
        return lib.gws_layernorm_bwd(ctypes.addressof(d), dy, s, w, stats, g, dx, dw, db, ws, nbytes, None)

    assert bwd(ld=63) == bwd(ld_dy=63) == bwd(ld_d=63) == bwd(rows=-2) == binding.ERR_SHAPE
    assert bwd(kind=7) == binding.ERR_UNSUPPORTED
    assert bwd(dy=None) == bwd(s=None) == bwd(stats=None) == binding.ERR_NULL
    assert bwd(dy=P[0] + 1) == bwd(dx=P[5] + 1) == bwd(dw=P[6] + 1) == bwd(kind=1, db=P[7] + 2) == bwd(g=P[4] + 1) == bwd(stats=P[3] + 1) == binding.ERR_ALIGN
    assert bwd(dx=P[0]) == bwd(dx=P[4]) == bwd(dw=P[2]) == bwd(dw=P[7]) == bwd(ws=P[1]) == bwd(dx=P[8] + 256) == binding.ERR_ALIAS
    assert bwd(ws=None) == bwd(nbytes=need - 1) == bwd(ws=P[8] + 128) == binding.ERR_WORKSPACE
    assert bwd(dx=None, dw=None, db=None) == bwd(rows=0, cols=0) == binding.OK
    assert gws.launch_count() == before


def test_adamw_validates_before_any_launch(lib):
    before = gws.launch_count()

    def step(params=(P[0], P[1]), grads=(P[2], P[3]), sizes=(300, 40), starts=(0, 512), types=(0, 0), n=None, moments=P[4], units=P[5], rest=P[6], total=768, fmt=1,
             args=True, lists=True, **over):
        n = len(params) if n is None else n
        st = binding._AdamwState(moments, units, rest, total, fmt, 0)
        a = binding._AdamwArgs(1e-3, 0.9, 0.95, 1e-8, 1, None, None, None, None)
        for k, v in over.items():
            setattr(a, k, v)
        arrays = [(ctypes.c_void_p * len(params))(*params), (ctypes.c_void_p * len(params))(*grads), (ctypes.c_int64 * len(params))(*sizes),
                  (ctypes.c_int64 * len(params))(*starts), (ctypes.c_int32 * len(params))(*types), (ctypes.c_double * len(params))()]
        if not lists:
            arrays[3] = None
        return lib.gws_adamw_step(n, *arrays, ctypes.addressof(st), ctypes.addressof(a) if args else None, None)

    assert step(args=False) == step(lists=False) == step(moments=None) == step(units=None) == step(params=(None, P[1])) == step(lr_dev=P[9]) == binding.ERR_NULL
    assert step(fmt=2) == step(types=(0, 2)) == step(beta1=1.0) == step(beta2=-0.1) == step(eps=-1.0) == step(beta1=float("nan")) == binding.ERR_UNSUPPORTED
    assert step(n=-1) == step(step=0) == step(total=700) == step(sizes=(-1, 40)) == step(starts=(0, 500)) == step(sizes=(300, 257)) == step(starts=(0, 768)) == \
        step(starts=(-256, 512)) == step(sizes=(300, 1 << 62)) == binding.ERR_SHAPE
    assert step(total=1 << 40) == binding.ERR_LIMIT
    assert step(params=(P[0] + 1, P[1])) == step(types=(1, 0), grads=(P[2] + 2, P[3])) == step(moments=P[4] + 16) == step(rest=P[6] + 8) == step(units=P[5] + 2) == \
        step(grad_scale=P[9] + 2) == step(step_dev=P[9] + 4, scalars=P[10]) == binding.ERR_ALIGN
    # the same tensor twice, a part of the state twice, a parameter on a gradient, on another one, on the state
    assert step(params=(P[0], P[0])) == step(starts=(0, 256)) == step(starts=(512, 512), sizes=(200, 40)) == step(params=(P[2] + 598, P[1])) == step(params=(P[0], P[0] + 598)) == \
        step(params=(P[0], P[4] + 1504)) == step(moments=P[2]) == step(units=P[6] + 1532) == step(grad_scale=P[0] + 4) == step(lr_dev=P[9], scalars=P[9]) == binding.ERR_ALIAS
    assert step(starts=(512, 0), sizes=(40, 300), fmt=3) == binding.ERR_UNSUPPORTED
    assert step(n=0) == step(grads=(None, None)) == step(sizes=(0, 0)) == binding.OK
    st = binding._AdamwState(P[4], P[5], None, 512, 1, 0)
    values = lambda s, m=P[0], v=P[1]: lib.gws_adamw_values(s if s is None else ctypes.addressof(s), m, v, None)
    assert values(None) == values(st, None) == values(st, P[0], None) == binding.ERR_NULL
    assert values(binding._AdamwState(P[4], None, None, 512, 0, 0)) == binding.ERR_UNSUPPORTED
    assert values(binding._AdamwState(P[4], P[5], None, 100, 1, 0)) == binding.ERR_SHAPE
    assert values(st, P[0] + 16) == binding.ERR_ALIGN
    assert values(st, P[4]) == values(st, P[0], P[0] + 2016) == binding.ERR_ALIAS
    assert gws.launch_count() == before
