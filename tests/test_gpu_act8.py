"""8-bit activation checkpoints and the weight gradient taken from one, against plain forms in 64 bits."""
import math

import pytest
import torch

import act_reference as ref
import paper_2505_11170_b200 as gws

pytestmark = pytest.mark.gpu
DEV = "cuda"
FORMATS = [gws.ACT8_INT8, gws.ACT8_E4M3]


def _x(rows, cols, seed=0, spread=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g)
    if spread:                                    # magnitudes from 2^-40 to 2^40 and small elements beside large ones
        x *= torch.exp2(torch.randint(-40, 41, (rows, 1), generator=g).float())
        x *= torch.exp2(torch.randint(-9, 1, (rows, cols), generator=g).float())
    return x.to(torch.bfloat16)


def _same_as_reference(a, x):
    element, byte = ref.encode(x.double(), a.fmt)
    groups = byte.shape[1]
    got_byte = a.scales.long().cpu()
    assert torch.equal(got_byte, byte)
    got = ref.elements_of(a.codes.cpu().reshape(a.rows, groups, 32), a.fmt)
    assert torch.equal(got, element)
    return ref.values(element, byte, a.cols)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (1, 2048), (3, 31), (5, 33), (7, 64), (64, 768), (33, 1365), (257, 96), (2, 5632), (300, 2730)])
def test_codes_scales_and_restored_values_are_exact(fmt, rows, cols):
    x = _x(rows, cols, seed=rows * 7 + cols)
    a = gws.act8_save(x.to(DEV), fmt)
    want = _same_as_reference(a, x)
    got = gws.act8_load(a).cpu()
    assert torch.equal(got.double(), want.to(torch.bfloat16).double())     # rounds only E4M3 values below 2^-126
    if fmt == gws.ACT8_INT8:
        assert torch.equal(got.double(), want)


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_bf16_number_in_a_group_of_its_own_magnitude(fmt):
    # every positive finite BF16 pattern as the largest of a group, with the patterns just below it and their negatives beside it
    patterns = torch.arange(0, 0x7F80, dtype=torch.int32)
    beside = torch.stack([(patterns - i).clamp(min=0) | (0x8000 * (i & 1)) for i in range(32)], 1).to(torch.int16)
    x = beside.view(torch.bfloat16)
    a = gws.act8_save(x.to(DEV), fmt)
    want = _same_as_reference(a, x)
    assert torch.equal(gws.act8_load(a).cpu().double(), want.to(torch.bfloat16).double())


@pytest.mark.parametrize("fmt", FORMATS)
def test_ties_go_to_the_even_code_and_the_largest_is_clamped(fmt):
    if fmt == gws.ACT8_INT8:
        row = [1.0, 0.5 / 64, 1.5 / 64, 2.5 / 64, -0.5 / 64, -1.5 / 64, -2.5 / 64]
        top = [255 / 128, 127 / 64, -255 / 128]
    else:
        row = [256.0, 17.0, 18.0, 19.0, -17.0, -19.0, 2.0 ** -10, 3 * 2.0 ** -10]
        top = [510.0, 448.0, -464.0, 465.0]
    for r in (row, top):
        x = torch.zeros(1, 32)
        x[0, :len(r)] = torch.tensor(r)
        x = x.to(torch.bfloat16)
        _same_as_reference(gws.act8_save(x.to(DEV), fmt), x)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("aligned", [True, False])
def test_groups_with_nan_or_infinity_restore_as_nan_and_leave_their_neighbours_alone(fmt, aligned):
    x = _x(6, 96 if aligned else 90, spread=False)
    x[1, 40], x[2, 0], x[3, 70], x[4] = math.nan, math.inf, -math.inf, 0.0
    a = gws.act8_save(x.to(DEV), fmt)
    want = _same_as_reference(a, x)
    assert int((a.scales == 255).sum()) == 3
    got = gws.act8_load(a).cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isnan(got)], want[~torch.isnan(want)])
    assert torch.equal(got[4], torch.zeros(x.shape[1], dtype=torch.float64))


@pytest.mark.parametrize("fmt", FORMATS)
def test_strides_offsets_and_broadcast_rows(fmt):
    base = _x(40, 200, spread=False)
    dev = base.to(DEV)
    for view in (lambda t: t[:, :64], lambda t: t[:, 16:112], lambda t: t[:, 1:98], lambda t: t[3:4, 5:], lambda t: t[::2, :96], lambda t: t[:1].expand(40, 200),
                 lambda t: t.t(), lambda t: t[:, ::2]):
        x = view(base)
        a = gws.act8_save(view(dev), fmt)
        want = _same_as_reference(a, x)
        out = torch.full((x.shape[0], x.shape[1] + 24), 7.0, dtype=torch.bfloat16, device=DEV)
        for first in (0, 8, 3):                       # written into a wider tensor: nothing beside it changes
            out.fill_(7.0)
            gws.act8_load(a, x=out[:, first:first + x.shape[1]])
            got = out.cpu().double()
            assert torch.equal(got[:, first:first + x.shape[1]], want.to(torch.bfloat16).double())
            assert bool((got[:, :first] == 7).all()) and bool((got[:, first + x.shape[1]:] == 7).all())


def test_empty_tensors_and_refusals():
    for shape in ((0, 64), (5, 0)):
        a = gws.act8_save(torch.empty(shape, dtype=torch.bfloat16, device=DEV))
        assert gws.act8_load(a).shape == shape
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV)
    before = gws.launch_count()
    with pytest.raises(gws.GwsError):
        gws.act8_save(x, 2)
    with pytest.raises(ValueError):
        gws.act8_save(x.float())
    with pytest.raises(ValueError):
        gws.act8_save(x[0])
    with pytest.raises(ValueError):
        gws.act8_save(x.cpu())
    with pytest.raises(ValueError):
        gws.Act8(torch.empty(10, dtype=torch.uint8, device=DEV), 4, 64, gws.ACT8_INT8)
    with pytest.raises(ValueError):
        gws.act8_load(gws.Act8(torch.zeros(1024, dtype=torch.uint8, device=DEV), 4, 64, 0), x=torch.empty(64, 4, dtype=torch.bfloat16, device=DEV).t())
    with pytest.raises(ValueError):
        gws.act8_save(x, out=gws.act8_save(x[:2]))
    assert gws.launch_count() == before + 1


def test_a_tensor_with_more_than_2_to_31_elements():
    rows, cols = 70000, 32768
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    last = _x(1, cols, spread=False).to(DEV)
    x[-1] = last[0]
    a = gws.act8_save(x)
    del x
    back = gws.act8_load(a)
    assert torch.equal(back[-1], gws.act8_load(gws.act8_save(last))[0])
    assert int((back[:-1].view(torch.int16) != 0).any())== 0


# ---- weight gradient -------------------------------------------------------------------------------------------------------

def wgrad_bound(grad_y, x, want):
    """|error| allowed per element: BF16 rounding of the result, and FP32 sums over m products (each product of two BF16 numbers is
    exact; every one of the additions, in whatever order, loses at most 2^-23 of the sum of magnitudes - the tensor cores may
    truncate)."""
    m = grad_y.shape[0]
    return 2.0 ** -8 * want.abs() + (m + 64) * 2.0 ** -23 * (grad_y.abs().t() @ x.abs()) + 1e-38


WGRAD_SHAPES = [(1, 8, 8), (1, 256, 768), (2, 33, 40), (63, 64, 64), (64, 128, 256), (65, 1, 1), (130, 200, 72), (515, 768, 768), (1000, 1023, 341),
                (4096, 320, 512), (2047, 130, 2048), (16384, 96, 128)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m,n,k", WGRAD_SHAPES)
def test_weight_gradient_from_a_checkpoint(fmt, m, n, k):
    gy = (_x(m, n, seed=1, spread=False).float() * 1e-3).to(torch.bfloat16).to(DEV)
    a = gws.act8_save(_x(m, k, seed=2, spread=False).to(DEV), fmt)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = gws.wgrad_act8(gy, a, status=status)
    x = ref.decode(a)
    want = gy.double().t() @ x
    assert bool(((got.double() - want).abs() <= wgrad_bound(gy.double(), x, want)).all())
    assert int(status) == 0
    assert torch.equal(got, gws.wgrad_act8(gy, a))          # the same bits every time


def test_weight_gradient_of_strided_and_unaligned_gradients_and_into_a_given_tensor():
    big = (_x(300, 400, seed=3, spread=False)).to(DEV)
    a = gws.act8_save(_x(300, 96, seed=4, spread=False).to(DEV))
    x = ref.decode(a)
    for view in (big[:, :128], big[:, 8:200], big[:, 3:200], big[:1].expand(300, 400), big[:, ::2]):
        want = view.double().t() @ x
        out = torch.empty(view.shape[1], 96, dtype=torch.bfloat16, device=DEV)
        got = gws.wgrad_act8(view, a, grad_w=out)
        assert got is out
        assert bool(((got.double() - want).abs() <= wgrad_bound(view.double(), x, want)).all())
    with pytest.raises(ValueError):
        gws.wgrad_act8(big[:299], a)
    with pytest.raises(ValueError):
        gws.wgrad_act8(big, a, grad_w=torch.empty(96, 400, dtype=torch.bfloat16, device=DEV))


def test_weight_gradient_over_no_tokens_is_zero():
    a = gws.act8_save(torch.empty(0, 40, dtype=torch.bfloat16, device=DEV))
    got = gws.wgrad_act8(torch.empty(0, 24, dtype=torch.bfloat16, device=DEV), a)
    assert got.shape == (24, 40) and not bool(got.any())


def test_weight_gradient_on_another_stream_than_the_current_one():
    gy = _x(500, 264, seed=5, spread=False).to(DEV)
    a = gws.act8_save(_x(500, 136, seed=6, spread=False).to(DEV))
    want = gws.wgrad_act8(gy, a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [gws.wgrad_act8(gy, a, stream=side) for _ in range(20)]
    noise = [torch.full((1 << 20,), 3, dtype=torch.uint8, device=DEV) for _ in range(20)]   # what the current stream allocates meanwhile
    side.synchronize()
    assert all(torch.equal(o, want) for o in outs) and len(noise) == 20


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m,n,k", [(515, 96, 200), (1072, 76, 17), (4369, 176, 200)])    # converted inside the product, restored before it
def test_a_group_that_restores_as_nan_reaches_its_own_columns_of_the_weight_gradient(fmt, m, n, k):
    gy, x = _x(m, n, seed=7, spread=False).to(DEV), _x(m, k, seed=8, spread=False).to(DEV)
    clean = gws.wgrad_act8(gy, gws.act8_save(x, fmt))
    x[m // 2, k - 1] = math.inf
    got = gws.wgrad_act8(gy, gws.act8_save(x, fmt))
    first = (k - 1) // 32 * 32
    assert bool(torch.isnan(got[:, first:]).all()) and torch.equal(got[:, :first], clean[:, :first])
