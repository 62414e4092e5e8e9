"""Roots and quotients of the AdamW step are rounded as sqrt and / round: steps without a gradient and from a weight of zero show the quotient's bits."""
import numpy as np
import pytest
import torch

import paper_2505_11170_b200 as gws
import step_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


def step(m, v, lr, betas, eps, t):
    """(weights that the step makes of zeros, those that it is specified to make)."""
    n = m.size
    assert n % 256 == 0
    state = gws.AdamWState([n], moments=torch.stack([torch.from_numpy(m).to(DEV), torch.from_numpy(v).to(DEV)]))
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    gws.adamw_step([p], [g], state, lr=lr, betas=betas, eps=eps, weight_decay=0.0, step=t)
    zero = np.zeros(n, np.float32)
    return p.cpu().numpy(), ref.adamw32(zero, zero, m, v, lr, *betas, eps, 0.0, t)[0].astype(np.float32)


def floats(exponent, binades):
    """Every FP32 number of neighbouring binades."""
    return np.arange((exponent + 127) << 23, (exponent + 127 + binades) << 23, dtype=np.uint32).view(np.float32)


# b1 = b2 = 0.5 after many steps: m and v are halved without a rounding, alpha is lr and rho 1
@pytest.mark.parametrize("exponent", [-60, -20, 0, 40, 98])
def test_roots_of_every_significand(exponent):
    v = floats(exponent, 2)
    for m in (1.0, 2 - 2.0 ** -23):                           # a root one unit off changes at least one of the two quotients, if not for every v
        got, want = step(np.full(v.size, 2 * m, np.float32), 2 * v, 1.0, (0.5, 0.5), 2.0 ** -40, 2000)
        assert np.array_equal(got.view(np.uint32), want.view(np.uint32))


def test_roots_at_the_lower_end():
    """The smallest v that the fast arithmetic takes: rho = 4096 keeps the roots' last place in the sum with eps."""
    v = np.maximum(floats(-100, 2), np.float32(2.0 ** -100 * (1 + 2.0 ** -20)))
    got, want = step(np.full(v.size, 2.0 ** -20, np.float32), v, 0.5, (0.5, 1 - 2.0 ** -24), 2.0 ** -40, 1)
    assert np.array_equal(got.view(np.uint32), want.view(np.uint32))


@pytest.mark.parametrize("lr,m_range,v_range", [(1.0, (-99, 39), (-60, 98)), (2.0 ** 29, (-60, 39), (-98, 98)), (2.0 ** -29, (-69, 39), (-60, 98)), (1.0, (0, 0), (0, 0))])
def test_quotients_of_random_significands_and_exponents(lr, m_range, v_range):
    rng = np.random.default_rng(7)
    n = 1 << 24
    number = lambda range_: np.ldexp(1 + rng.integers(0, 1 << 23, n) * 2.0 ** -23, rng.integers(range_[0], range_[1] + 1, n)).astype(np.float32)
    m, v = number(m_range) * np.where(rng.random(n) < 0.5, np.float32(-1), np.float32(1)), number(v_range)
    got, want = step(2 * m, 2 * v, lr, (0.5, 0.5), 2.0 ** -40, 2000)
    normal = np.abs(want) >= 2.0 ** -126
    assert normal.mean() > 0.5
    assert np.array_equal(got[normal].view(np.uint32), want[normal].view(np.uint32))
    assert np.all(np.abs(got[~normal].view(np.int32).astype(np.int64) - want[~normal].view(np.int32)) <= 1)


def test_quotients_next_to_a_border():
    """Numerators of which the quotient is as near to half way between two numbers as it comes: n = d (q + half a unit) rounded, for random d and q, and its neighbours."""
    rng = np.random.default_rng(8)
    n = 1 << 22
    d = (1 + rng.integers(0, 1 << 23, n) * 2.0 ** -23).astype(np.float32)
    v = (d * d).astype(np.float32)
    d = np.sqrt(v)                                             # what the step divides by: eps is below half a unit of it
    q = 1 + rng.integers(0, 1 << 23, n) * 2.0 ** -23 + 2.0 ** -24
    m = (d.astype(np.float64) * q).astype(np.float32)
    for side in (-1, 0, 1):
        got, want = step(2 * (m.view(np.int32) + side).view(np.float32), 2 * v, 1.0, (0.5, 0.5), 2.0 ** -40, 2000)
        assert np.array_equal(got.view(np.uint32), want.view(np.uint32))


def test_quotients_half_way_between_two_of_the_smallest_numbers():
    """Below 2^-126 a quotient may be one unit, 2^-149, off."""
    k = np.arange(1 << 16, dtype=np.float64)
    for d in (3.0, 5.0, 7.0, 1.0):
        m = np.maximum(d * (2 * k + 1) * 2.0 ** (47 - 150), 2.0 ** -99).astype(np.float32)
        got, want = step(2 * m, np.full(k.size, 2 * (d * 2.0 ** 47) ** 2, np.float32), 1.0, (0.5, 0.5), 2.0 ** -40, 2000)
        assert np.all(np.abs(got) < 2.0 ** -126) and np.all(np.abs(got.view(np.int32).astype(np.int64) - want.view(np.int32)) <= 1)


def test_codes_and_units_of_groups_of_any_size():
    """The reciprocals of units: largest values of 2^-90 to beyond what a square in FP32 can hold, where the root's group is not finite and the mean's is."""
    rng = np.random.default_rng(9)
    groups = 1 << 13
    g = np.ldexp(rng.standard_normal((groups, 256)), rng.integers(-90, 120, (groups, 1))).astype(np.float32).ravel()
    state = gws.AdamWState([g.size], gws.ADAMW_8BIT)
    gws.adamw_step([torch.zeros(g.size, device=DEV)], [torch.from_numpy(g).to(DEV)], state, lr=1e-3, betas=(0.9, 0.95), weight_decay=0.0, step=1)
    zero = np.zeros(g.size, np.float32)
    with np.errstate(all="ignore"):
        _, m, _, r = ref.adamw32(zero, g, zero, zero, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1)
        (cm, um), (cr, ur) = ref.encode_m(m), ref.encode_r(r)
    assert np.array_equal(state.units[0].cpu().numpy(), um) and np.array_equal(state.units[1].cpu().numpy(), ur, equal_nan=True) and np.isnan(ur).any()
    codes = state.moments.cpu().numpy()
    sign = lambda c: c & (0x7F | ((c & 0x7F) != 0) * 0x80)      # a zero's sign is free
    assert np.array_equal(sign(codes[0]), sign(cm.ravel())) and np.array_equal(codes[1], cr.ravel())
