"""gws_adamw_check answers what gws_adamw_step would: host arithmetic on pointers and sizes, nothing is launched."""
import ctypes

import pytest

import paper_2505_11170_b200 as gws
from paper_2505_11170_b200 import _build, binding

P = [0x10000000 + 0x4000000 * i for i in range(14)]      # never dereferenced


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return gws.load_library()


def test_check_answers_as_the_step_and_launches_nothing(lib):
    before = gws.launch_count()

    def both(params=(P[0], P[1]), grads=(P[2], P[3]), sizes=(300, 40), starts=(0, 512), types=(0, 0), fmt=1, total=768, refused=True, **over):
        state = binding._AdamwState(P[4], P[5], P[6], total, fmt, 0)
        a = binding._AdamwArgs(1e-3, 0.9, 0.95, 1e-8, 1, None, None, None, None)
        for k, v in over.items():
            setattr(a, k, v)
        arrays = [(ctypes.c_void_p * 2)(*params), (ctypes.c_void_p * 2)(*grads), (ctypes.c_int64 * 2)(*sizes), (ctypes.c_int64 * 2)(*starts), (ctypes.c_int32 * 2)(*types),
                  (ctypes.c_double * 2)()]
        code = lib.gws_adamw_check(2, *arrays, ctypes.addressof(state), ctypes.addressof(a))
        if refused:
            assert code != binding.OK and code == lib.gws_adamw_step(2, *arrays, ctypes.addressof(state), ctypes.addressof(a), None)
        return code

    for wrong in (dict(params=(None, P[1])), dict(fmt=2), dict(types=(0, 2)), dict(beta1=1.0), dict(beta2=float("nan")), dict(eps=-1.0), dict(step=0), dict(total=700),
                  dict(sizes=(-1, 40)), dict(starts=(0, 500)), dict(starts=(0, 256)), dict(params=(P[0] + 1, P[1])), dict(grad_scale=P[9] + 2), dict(params=(P[0], P[0])),
                  dict(grads=(P[0], P[3])), dict(grad_scale=P[0] + 4), dict(params=(P[0], P[4] + 1504))):
        both(**wrong)
    assert both(refused=False) == both(refused=False, lr_dev=P[9]) == both(refused=False, grads=(None, None)) == binding.OK       # no room for scalars is wanted
    assert lib.gws_adamw_check(2, None, None, None, None, None, None, None, None) == binding.ERR_NULL
    assert gws.launch_count() == before
