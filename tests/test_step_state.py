"""The state of the AdamW step and its optimizer on the CPU: the calls that they refuse, and states that are loaded."""
import pytest
import torch

import paper_2505_11170_b200 as gws


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
