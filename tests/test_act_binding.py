"""Host side of the activation operators' Python calls, on CPU tensors that claim to live on a GPU and a library that only records."""
import contextlib
import ctypes

import pytest
import torch

import paper_2505_11170_b200 as gws
from paper_2505_11170_b200 import binding


class OnDevice(torch.Tensor):
    """A CPU tensor that names GPU 1 as its device."""

    def get_device(self):
        return 1


def _on_gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


class FakeLibrary:
    """Accepts every call and notes its name and the device that was current."""

    def __init__(self, state):
        self.calls, self.state = [], state

    def gws_status_string(self, status):
        return b"status"

    def __getattr__(self, name):
        if not name.startswith("gws_"):
            raise AttributeError(name)

        def call(*args):
            self.calls.append((name, self.state["device"], args[-1]))
            return 0

        return call


@pytest.fixture
def fake(monkeypatch):
    state = {"device": 0}

    @contextlib.contextmanager
    def use(device):
        before, state["device"] = state["device"], device
        yield
        state["device"] = before

    lib = FakeLibrary(state)
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_current_device", lambda: state["device"], raising=False)
    monkeypatch.setattr(binding, "_raw_stream", lambda device: 1000 + device)
    monkeypatch.setattr(binding, "_watch", ctypes.c_int32(0), raising=False)
    monkeypatch.setattr(binding, "_watch_address", 0x7000, raising=False)
    monkeypatch.setattr(torch.cuda, "device", use)
    caches = (binding._wgrad_workspace, binding._gated_plan)
    for cache in caches:
        cache.cache_clear()
    yield lib
    for cache in caches:
        cache.cache_clear()


def _calls():
    x, w, dy = _on_gpu(4, 64), _on_gpu(96, 64), _on_gpu(4, 96)
    x8 = gws.Act8(_on_gpu(1024, dtype=torch.uint8), 4, 64, gws.ACT8_INT8)
    saved = gws.GatedSaved(_on_gpu(4096, dtype=torch.uint8), 4, 96, gws.ACT8_INT8)
    return {"act8_save": lambda **kw: gws.act8_save(x, **kw), "act8_load": lambda **kw: gws.act8_load(x8, **kw),
            "wgrad_act8": lambda **kw: gws.wgrad_act8(dy, x8, **kw), "gated_fwd": lambda **kw: gws.gated_fwd(x, w, w, **kw),
            "gated_bwd": lambda **kw: gws.gated_bwd(dy, x8, w, w, saved, **kw)}


@pytest.mark.parametrize("name", ["act8_save", "act8_load", "wgrad_act8", "gated_fwd", "gated_bwd"])
def test_tensors_of_another_gpu_than_the_current_one(fake, name):
    # a default stream's handle is 0 on every device: the launch, and the sizes that depend on the device, need the tensors' device current
    _calls()[name]()
    assert fake.calls and all(device == 1 for _, device, _ in fake.calls)
    assert fake.calls[-1][0] == "gws_" + name and fake.calls[-1][2] == 1001
    assert fake.state["device"] == 0


@pytest.mark.parametrize("name", ["act8_save", "act8_load", "wgrad_act8", "gated_fwd", "gated_bwd"])
def test_a_stream_of_another_gpu_than_the_tensors_is_refused(fake, name):
    class OtherStream:
        cuda_stream, device_index = 5, 0

    with pytest.raises(ValueError):
        _calls()[name](stream=OtherStream())
    assert not fake.calls


def _bytes(n):
    return torch.zeros(n, dtype=torch.uint8)


@pytest.mark.parametrize("fmt", [gws.ACT8_INT8, gws.ACT8_E4M3, gws.SAVE_BF16])
def test_kept_projections_refuse_a_buffer_that_a_kernel_would_read_past(fmt):
    m, n = 5, 96
    need = 2 * -(-(2 * m * n if fmt == gws.SAVE_BF16 else gws.act8_layout(m, n)[2]) // 256) * 256
    kept = gws.GatedSaved(_bytes(need), m, n, fmt)
    assert tuple(kept.gate.shape) == tuple(kept.up.shape) == (m, n)
    for bad in (_bytes(need - 1), torch.zeros(need, dtype=torch.int8), torch.zeros(need // 2, dtype=torch.bfloat16), _bytes(2 * need)[::2], _bytes(0)):
        with pytest.raises(ValueError):
            gws.GatedSaved(bad, m, n, fmt)
    for shape in ((-m, -n), (-1, n), (m, -1)):
        with pytest.raises(ValueError):
            gws.GatedSaved(_bytes(need), *shape, fmt)


@pytest.mark.parametrize("fmt", [gws.SAVE_NONE, -1, 7])
def test_kept_values_refuse_a_format_they_cannot_have(fmt):
    with pytest.raises(ValueError):
        gws.GatedSaved(_bytes(1 << 16), 4, 32, fmt)
    with pytest.raises(ValueError):
        gws.Act8(_bytes(1 << 16), 4, 32, fmt)


def test_a_checkpoint_refuses_negative_sizes():
    for shape in ((-4, -32), (-1, 32), (4, -32)):
        with pytest.raises(ValueError):
            gws.Act8(_bytes(1 << 16), *shape, gws.ACT8_INT8)


@pytest.mark.parametrize("name", ["wgrad_act8", "gated_fwd", "gated_bwd"])
def test_a_kernel_that_gave_up_is_reported_by_the_next_call(fake, name):
    call = _calls()[name]
    call()
    launched = len(fake.calls)
    binding._watch.value = 1                        # as the kernel writes it
    with pytest.raises(gws.GwsError):
        call()
    assert len(fake.calls) == launched              # before anything is launched, and once
    call()
    assert len(fake.calls) > launched


def test_a_kernel_that_gave_up_is_reported_by_the_modules(fake):
    from paper_2505_11170_b200.module import GaussWSLinear

    layer = GaussWSLinear.__new__(GaussWSLinear)
    torch.nn.Module.__init__(layer)
    layer.step, layer._update = 3, {"lambda_term_due": False}
    binding._watch.value = 1
    with pytest.raises(gws.GwsError):
        layer.advance()
    assert layer.step == 3
    layer.advance()
    assert layer.step == 4


@pytest.mark.parametrize("name", ["wgrad_act8", "gated_fwd", "gated_bwd"])
def test_status_words_of_another_type_are_refused(fake, name):
    call = _calls()[name]
    for bad in (_on_gpu(1, dtype=torch.uint8), _on_gpu(1, dtype=torch.int64), _on_gpu(0, dtype=torch.int32)):
        with pytest.raises(ValueError):
            call(status=bad)
    assert not fake.calls
    call(status=_on_gpu(1, dtype=torch.int32))
