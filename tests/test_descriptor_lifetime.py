"""What the library reads by address during a call is held by the call, not by a cache that another thread may turn over in that time."""
import gc
import weakref

import pytest
import torch

import paper_2505_11170_b200 as gws
from paper_2505_11170_b200 import binding


class Library:
    """In place of the library: its calls empty the caches of descriptors, and see whether the one that they were given is still there."""

    def __init__(self):
        self.held = []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return lambda *args: 256

        def call(at, *rest):
            alive = [weakref.ref(d) for d in gc.get_objects() if type(d) in (binding.NormDesc, binding.LinearDesc, binding.GatedDesc) and binding.ctypes.addressof(d) == at]
            for cache in (binding._norm_plan, binding._linear_plan, binding._gated_plan):
                cache.cache_clear()
            gc.collect()
            self.held.append(len(alive) == 1 and alive[0]() is not None)
            return 0

        return call


@pytest.fixture
def library(monkeypatch):
    fake = Library()
    for name, value in (("_lib", fake), ("load_library", lambda: fake), ("_device_of", lambda *tensors: 0), ("_current_device", lambda: 0), ("_raw_stream", lambda device: None),
                        ("_status_of", lambda status: None)):
        monkeypatch.setattr(binding, name, value)
    for cache in (binding._norm_plan, binding._linear_plan, binding._gated_plan):
        cache.cache_clear()
    yield fake
    for cache in (binding._norm_plan, binding._linear_plan, binding._gated_plan):
        cache.cache_clear()


X, W = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(64, 32, dtype=torch.bfloat16)
Y, Z = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64, dtype=torch.bfloat16)
CALLS = {
    "layernorm_fwd": lambda: gws.layernorm_fwd(X, residual=X.clone()),
    "layernorm_bwd": lambda: gws.layernorm_bwd(X, X, W[0], torch.zeros(2, 4)),
    "linear_fwd": lambda: gws.linear_fwd(X, W),
    "linear_bwd": lambda: gws.linear_bwd(Y, X, W, Z, gws.GATED_SILU),
    "gated_fwd": lambda: gws.gated_fwd(X, W, W.clone()),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_call_holds_its_descriptor(library, name):
    CALLS[name]()
    assert library.held == [True]
