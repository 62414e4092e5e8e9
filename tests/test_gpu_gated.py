"""The gated feed-forward block, forward and backward, against plain forms in 64 bits."""
import math

import pytest
import torch

import act_reference as ref
import paper_2505_11170_b200 as gws

pytestmark = pytest.mark.gpu
DEV = "cuda"
ACTS = [gws.GATED_SILU, gws.GATED_GELU_TANH, gws.GATED_RELU]
# (m, n, k): one token to many, widths that are and are not multiples of the tiles, of 32, of 8; all odd
SHAPES = [(1, 64, 64), (1, 5632, 256), (3, 8, 8), (33, 96, 40), (128, 128, 128), (129, 130, 72), (200, 1365, 512), (257, 2048, 96), (300, 33, 31),
          (640, 1000, 333), (1, 1, 1), (2048, 256, 768), (1500, 2730, 64)]


def _rand(rows, cols, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, cols, generator=g) * std).to(torch.bfloat16).to(DEV)


def _problem(m, n, k):
    std = 1.0 / math.sqrt(k)
    return _rand(m, k, 1), _rand(n, k, 2, 1.5 * std), _rand(n, k, 3, 1.5 * std), _rand(m, n, 4, 1e-2)


def projections(x, wg, wu):
    """g, u in 64 bits and the error FP32 sums over k may leave in them."""
    x, wg, wu = x.double(), wg.double(), wu.double()
    eps = (x.shape[1] + 64) * 2.0 ** -23
    return x @ wg.t(), x @ wu.t(), eps * (x.abs() @ wg.abs().t()), eps * (x.abs() @ wu.abs().t())


def h_bound(a, u, slope_most, dg, du, h):
    """BF16 rounding of h, the errors of g (through act, whose slope is at most slope_most) and of u, and 2^-19 for the FP32
    evaluation of the activation (exp and division of a few ulp, arguments up to a few tens)."""
    return 2.0 ** -8 * h.abs() + slope_most * dg * (u.abs() + du) + a.abs() * du + 2.0 ** -19 * h.abs() + 1e-38


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_forward(act, m, n, k):
    x, wg, wu, _ = _problem(m, n, k)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    h, saved = gws.gated_fwd(x, wg, wu, act, status=status)
    assert saved is None and h.shape == (m, n)
    g, u, eg, eu = projections(x, wg, wu)
    a, _ = ref.act(g, act)
    want = a * u
    assert bool(((h.double() - want).abs() <= h_bound(a, u, 1.2, eg, eu, want)).all())
    assert int(status) == 0
    assert torch.equal(h, gws.gated_fwd(x, wg, wu, act)[0])


@pytest.mark.parametrize("save", [gws.ACT8_INT8, gws.ACT8_E4M3, gws.SAVE_BF16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_what_forward_keeps(save, m, n, k):
    x, wg, wu, _ = _problem(m, n, k)
    h, saved = gws.gated_fwd(x, wg, wu, gws.GATED_SILU, save=save)
    assert torch.equal(h, gws.gated_fwd(x, wg, wu, gws.GATED_SILU)[0])
    for kept, exact, err in zip((saved.gate, saved.up), *(lambda p: (p[:2], p[2:]))(projections(x, wg, wu))):
        if save == gws.SAVE_BF16:
            assert bool(((kept.double() - exact).abs() <= 2.0 ** -8 * exact.abs() + err + 1e-38).all())
            continue
        element, byte = ref.encode(exact, save)
        want = ref.values(element, byte, n)
        got = ref.decode(kept)
        # half a step of the group's grid (a whole one where the largest is clamped), as large as the next power of two allows
        top = torch.nn.functional.pad(exact.abs() + err, (0, -n % 32)).view(m, -1, 32).amax(-1)
        per_group = torch.exp2(torch.floor(torch.log2(top.clamp(min=1e-300)))) * (1.0 / 64 if save == gws.ACT8_INT8 else 1.0 / 4)
        step = per_group.repeat_interleave(32, 1)[:, :n]
        assert bool(((got - exact).abs() <= step + err).all())
        assert float((got != want).double().mean()) < 0.01           # a rounding that FP32 sums decide otherwise is rare
        ld = kept.codes.shape[1]
        assert not bool(kept.codes[:, n:ld].any())


def saved_values(saved):
    return [ref.decode(t) if isinstance(t, gws.Act8) else t.double() for t in (saved.gate, saved.up)]


def check_backward(got, grad_h, x, wg, wu, g, u, act):
    """x, g, u: the values that the backward pass reads, in 64 bits."""
    grad_x, grad_wg, grad_wu, h = got
    dh, wg, wu = grad_h.double(), wg.double(), wu.double()
    a, slope = ref.act(g, act)
    dg, du, want_h = dh * u * slope, dh * a, a * u
    (m, k), n = x.shape, g.shape[1]
    # dg and du are rounded to BF16 (8 significant bits: half a spacing is up to 2^-8 of the number) after an FP32 evaluation whose
    # error is far below that: relative to the largest magnitude the slope's terms can have (3, for GELU) it is at most 2^-18
    r = 2.0 ** -8 + 2.0 ** -18
    e_dg, e_du = r * dg.abs() + 2.0 ** -17 * (dh * u).abs(), r * du.abs() + 2.0 ** -18 * dh.abs() * a.abs()
    if grad_x is not None:
        want = dg @ wg + du @ wu
        sums = dg.abs() @ wg.abs() + du.abs() @ wu.abs()
        bound = 2.0 ** -8 * want.abs() + e_dg @ wg.abs() + e_du @ wu.abs() + (2 * n + 64) * 2.0 ** -23 * sums + 1e-38
        assert bool(((grad_x.double() - want).abs() <= bound).all())
    for grad, d, e in ((grad_wg, dg, e_dg), (grad_wu, du, e_du)):
        if grad is not None:
            want = d.t() @ x
            bound = 2.0 ** -8 * want.abs() + e.t() @ x.abs() + (m + 64) * 2.0 ** -23 * (d.abs().t() @ x.abs()) + 1e-38
            assert bool(((grad.double() - want).abs() <= bound).all())
    if h is not None:
        assert bool(((h.double() - want_h).abs() <= (2.0 ** -8 + 2.0 ** -18) * want_h.abs() + 1e-38).all())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("save", [gws.ACT8_INT8, gws.ACT8_E4M3, gws.SAVE_BF16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_backward(act, save, m, n, k):
    x, wg, wu, grad_h = _problem(m, n, k)
    _, saved = gws.gated_fwd(x, wg, wu, act, save=save)
    x_in = x if save == gws.SAVE_BF16 else gws.act8_save(x, save)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = gws.gated_bwd(grad_h, x_in, wg, wu, saved, act, want_h=True, status=status)
    assert [tuple(t.shape) for t in got] == [(m, k), (n, k), (n, k), (m, n)]
    check_backward(got, grad_h, ref.decode(x_in) if isinstance(x_in, gws.Act8) else x.double(), wg, wu, *saved_values(saved), act)
    assert int(status) == 0
    again = gws.gated_bwd(grad_h, x_in, wg, wu, saved, act, want_h=True)
    assert all(torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("act", ACTS)
def test_backward_against_differences_of_the_forward_pass(act):
    # the loss sum(dh * h) in 64 bits, moved along random directions of x, Wg and Wu; central differences of a smooth function
    m, n, k = 48, 96, 64
    x, wg, wu, grad_h = _problem(m, n, k)
    _, saved = gws.gated_fwd(x, wg, wu, act, save=gws.SAVE_BF16)
    grads = gws.gated_bwd(grad_h, x, wg, wu, saved, act)[:3]

    def loss(x_, wg_, wu_):
        return float((grad_h.double() * ref.act(x_ @ wg_.t(), act)[0] * (x_ @ wu_.t())).sum())

    at = [t.double() for t in (x, wg, wu)]
    gen = torch.Generator().manual_seed(9)
    for which in range(3):
        direction = torch.randn(at[which].shape, generator=gen).double().to(DEV)
        eps = 1e-5
        ahead, behind = list(at), list(at)
        ahead[which], behind[which] = at[which] + eps * direction, at[which] - eps * direction
        slope = (loss(*ahead) - loss(*behind)) / (2 * eps)
        inner = grads[which].double() * direction
        # g and u are kept in BF16 (2^-9, entering dg twice), dg and du rounded (2^-9), the gradient rounded (2^-9): at most 5 * 2^-9
        # of each element's sum of magnitudes; as independent errors of the elements, bounded by 6 standard deviations
        x64, wg64, wu64 = at
        a, s = ref.act(x64 @ wg64.t(), act)
        dg, du = (grad_h.double() * (x64 @ wu64.t()) * s).abs(), (grad_h.double() * a).abs()
        mags = [dg @ wg64.abs() + du @ wu64.abs(), dg.t() @ x64.abs(), du.t() @ x64.abs()][which]
        spread = float((5 * 2.0 ** -9 * mags * direction).square().sum().sqrt())
        kink = 0.02 * abs(slope) if act == gws.GATED_RELU else 0.0
        assert abs(float(inner.sum()) - slope) <= 6 * spread + kink + 1e-9


def test_parts_that_are_not_asked_for():
    x, wg, wu, grad_h = _problem(70, 200, 136)
    _, saved = gws.gated_fwd(x, wg, wu, save=gws.ACT8_INT8)
    full = gws.gated_bwd(grad_h, x, wg, wu, saved, want_h=True)
    only_x = gws.gated_bwd(grad_h, x, wg, wu, saved, want_grad_w=False)
    only_w = gws.gated_bwd(grad_h, x, wg, wu, saved, want_grad_x=False)
    assert torch.equal(only_x[0], full[0]) and only_x[1] is None and only_x[2] is None and only_x[3] is None
    assert only_w[0] is None and torch.equal(only_w[1], full[1]) and torch.equal(only_w[2], full[2])


def test_strided_unaligned_and_broadcast_inputs():
    m, n, k = 150, 264, 104
    X, WG, WU, DH = _rand(m, 200, 1), _rand(n, 200, 2, 0.1), _rand(n, 200, 3, 0.1), _rand(m, 400, 4, 1e-2)
    views = [lambda t, c: t[:, :c], lambda t, c: t[:, 8:8 + c], lambda t, c: t[:, 3:3 + c], lambda t, c: t[:1, 5:5 + c].expand(t.shape[0], c),
             lambda t, c: t[:, :2 * c:2] if 2 * c <= t.shape[1] else t[:, 1:1 + c]]
    for v in views:
        for w in (views[0], views[2]):
            x, wg, wu, dh = v(X, k), w(WG, k), views[1](WU, k), v(DH, n)
            h, saved = gws.gated_fwd(x, wg, wu, save=gws.ACT8_INT8)
            g, u, eg, eu = projections(x, wg, wu)
            a, _ = ref.act(g, gws.GATED_SILU)
            assert bool(((h.double() - a * u).abs() <= h_bound(a, u, 1.2, eg, eu, a * u)).all())
            got = gws.gated_bwd(dh, x, wg, wu, saved, want_h=True)
            check_backward(got, dh, x.double(), wg, wu, *saved_values(saved), gws.GATED_SILU)


def test_empty_sizes():
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)
    for save in (gws.ACT8_INT8, gws.SAVE_BF16):
        h, saved = gws.gated_fwd(z(0, 24), z(40, 24), z(40, 24), save=save)
        gx, gg, gu, hb = gws.gated_bwd(z(0, 40), z(0, 24), z(40, 24), z(40, 24), saved, want_h=True)
        assert h.shape == (0, 40) and gx.shape == (0, 24) and not bool(gg.any()) and not bool(gu.any()) and gg.shape == (40, 24)
        h, saved = gws.gated_fwd(z(5, 0), z(40, 0), z(40, 0), save=save)
        assert h.shape == (5, 40) and not bool(h.any()) and all(not bool(v.any()) for v in saved_values(saved))
        gx, gg, gu, hb = gws.gated_bwd(z(5, 40), z(5, 0), z(40, 0), z(40, 0), saved, want_h=True)
        assert gx.shape == (5, 0) and not bool(hb.any())
        h, saved = gws.gated_fwd(z(5, 24), z(0, 24), z(0, 24), save=save)
        gx, gg, gu, hb = gws.gated_bwd(z(5, 0), z(5, 24), z(0, 24), z(0, 24), saved, want_h=True)
        assert h.shape == (5, 0) and not bool(gx.any()) and gx.shape == (5, 24)


def test_nan_and_infinity_stay_in_their_rows():
    m, n, k = 70, 160, 96
    x, wg, wu, grad_h = _problem(m, n, k)
    clean, _ = gws.gated_fwd(x, wg, wu)
    x[5, 3], x[9, 0] = math.nan, math.inf
    h, saved = gws.gated_fwd(x, wg, wu, save=gws.ACT8_INT8)
    keep = [r for r in range(m) if r not in (5, 9)]
    assert torch.equal(h[keep], clean[keep]) and bool(torch.isnan(h[5]).all())
    grad_x = gws.gated_bwd(grad_h, x, wg, wu, saved, want_grad_w=False)[0]
    assert bool(torch.isnan(grad_x[5]).all()) and bool(torch.isfinite(grad_x[keep].float()).all())


def test_large_arguments_of_the_activation():
    # gates of +-300 at 1 and -300 at 0 times the input; exp overflows on one side and vanishes on the other
    x = torch.ones(1, 8, dtype=torch.bfloat16, device=DEV)
    wg = torch.zeros(64, 8, dtype=torch.bfloat16, device=DEV)
    wg[:, 0] = torch.linspace(-300, 300, 64, device=DEV).to(torch.bfloat16)
    wu = torch.zeros_like(wg)
    wu[:, 0] = 1
    for act in ACTS:
        h, saved = gws.gated_fwd(x, wg, wu, act, save=gws.SAVE_BF16)
        want = ref.act(wg[:, 0].double(), act)[0]
        # 2^-15: the argument of exp, up to 300, carries 2^-24 of itself into the exponent
        assert bool(((h[0].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -15) * want.abs() + 1e-30).all())
        got = gws.gated_bwd(torch.ones(1, 64, dtype=torch.bfloat16, device=DEV), x, wg, wu, saved, act, want_h=True)
        assert all(bool(torch.isfinite(t.float()).all()) for t in got)


def test_refusals():
    x, wg, wu, grad_h = _problem(16, 64, 32)
    _, saved = gws.gated_fwd(x, wg, wu, save=gws.ACT8_INT8)
    before = gws.launch_count()
    for bad in (lambda: gws.gated_fwd(x, wg, wu, 3), lambda: gws.gated_fwd(x, wg, wu, save=7), lambda: gws.gated_fwd(x.float(), wg, wu),
                lambda: gws.gated_fwd(x, wg[:, :16], wu), lambda: gws.gated_fwd(x, wg, wu[:32]), lambda: gws.gated_fwd(x.cpu(), wg, wu),
                lambda: gws.gated_fwd(x[0], wg, wu), lambda: gws.gated_fwd(x, wg, wu, h=x), lambda: gws.gated_bwd(grad_h[:8], x, wg, wu, saved),
                lambda: gws.gated_bwd(grad_h, x, wg, wu, saved, 9), lambda: gws.gated_bwd(grad_h[:, :32], x, wg[:32], wu[:32], saved)):
        with pytest.raises((ValueError, gws.GwsError)):
            bad()
    assert gws.launch_count() == before


def test_on_another_stream_than_the_current_one():
    x, wg, wu, grad_h = _problem(300, 520, 264)
    def step(stream=None):
        h, saved = gws.gated_fwd(x, wg, wu, save=gws.ACT8_INT8, stream=stream)
        return (h, *gws.gated_bwd(grad_h, gws.act8_save(x, stream=stream), wg, wu, saved, want_h=True, stream=stream))
    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [step(side) for _ in range(10)]
    noise = [torch.full((1 << 20,), 3, dtype=torch.uint8, device=DEV) for _ in range(40)]
    side.synchronize()
    assert all(torch.equal(p, q) for outs in got for p, q in zip(outs, want)) and len(noise) == 40


# sizes that take many of the tiles (one block of 128 x 128, a pair of 256 x 128 and of 256 x 256) and forms (whole, cut and joined, cut in a
# cluster, whole but for a cut last wave); test_tilings.py holds one for each form of each product and checks that it is taken
TILINGS = [(41, 89, 1076), (10781, 73, 68), (772, 1416, 276), (48, 66, 412), (9722, 235, 1350), (1404, 2389, 260), (32, 312, 89), (7448, 79, 526),
           (170, 4024, 195), (3254, 1779, 686), (6749, 1685, 668), (1487, 90, 139), (34, 3895, 268), (8874, 152, 69), (5522, 3570, 264), (4548, 1834, 1242),
           (2530, 136, 910), (15024, 1213, 192), (19150, 128, 2048)]


@pytest.mark.parametrize("m,n,k", TILINGS)
def test_every_way_to_tile(m, n, k):
    test_forward(gws.GATED_SILU, m, n, k)
    test_what_forward_keeps(gws.ACT8_INT8, m, n, k)
    test_backward(gws.GATED_SILU, gws.ACT8_INT8, m, n, k)


# few tokens: narrow tiles of every width, in one wave and in several, the last one ragged, 1 to 128 rows of A in a copy
FEW = [(1, 2300, 72), (7, 3500, 136), (33, 4713, 64), (128, 5901, 200), (61, 7100, 80), (2, 8202, 96), (100, 9400, 264), (9, 20001, 40), (120, 12000, 1032),
       (128, 9472, 648), (16, 37, 2056), (1, 1, 1), (5, 65, 4100)]


@pytest.mark.parametrize("m,n,k", FEW)
def test_few_tokens(m, n, k):
    for act in ACTS:
        test_forward(act, m, n, k)
    for save in (gws.ACT8_INT8, gws.ACT8_E4M3, gws.SAVE_BF16):
        test_what_forward_keeps(save, m, n, k)


def test_few_tokens_write_inside_their_output():
    for m, n, k in ((1, 5632, 256), (3, 5630, 256), (17, 2300, 72)):
        x, wg, wu, _ = _problem(m, n, k)
        want, _ = gws.gated_fwd(x, wg, wu)
        around = torch.full((m * n + 1024,), 7.0, device="cuda", dtype=torch.bfloat16)
        h = around[512:512 + m * n].view(m, n)
        gws.gated_fwd(x, wg, wu, h=h)
        assert torch.equal(h, want)
        assert bool((around[:512] == 7.0).all()) and bool((around[512 + m * n:] == 7.0).all())


def test_a_captured_step_replays_to_the_same_bits():
    x, wg, wu, grad_h = _problem(300, 520, 263)                 # copies of unaligned rows, cut contractions: several kernels a call

    def step():
        x8 = gws.act8_save(x)
        h, saved = gws.gated_fwd(x, wg, wu, save=gws.ACT8_INT8)
        return (gws.act8_load(x8), h, *gws.gated_bwd(grad_h, x8, wg, wu, saved, want_h=True), gws.wgrad_act8(grad_h, x8))

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_many_steps_in_a_row_without_waiting_give_the_same_bits():
    # kernels of consecutive calls overlap at their ends; outputs and workspaces come from memory that earlier calls still use
    x, wg, wu, grad_h = _problem(700, 1000, 520)
    outs = []
    for _ in range(60):
        h, saved = gws.gated_fwd(x, wg, wu, save=gws.ACT8_E4M3)
        outs.append((h, *gws.gated_bwd(grad_h, gws.act8_save(x, gws.ACT8_E4M3), wg, wu, saved, want_h=True)))
        if len(outs) > 4:
            del outs[1]
    first = outs[0]
    assert all(torch.equal(p, q) for o in outs for p, q in zip(o, first))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,n", [(3, 70), (1200, 2048)])       # eight elements to a lane, a group to a thread
def test_slopes_of_the_largest_finite_gates(act, m, n):
    # from 2^60 to the end of BF16, where the square of a gate passes FP32: the slope is 1 on one side and 0 on the other
    g = torch.exp2(torch.linspace(60, 127.9, n, device=DEV)).to(torch.bfloat16)
    g[::2] = -g[::2]
    buffer = torch.zeros(2 * gws.GatedSaved._part(m, n, gws.SAVE_BF16), dtype=torch.uint8, device=DEV)
    saved = gws.GatedSaved(buffer, m, n, gws.SAVE_BF16)
    saved.gate.copy_(g.expand(m, n))
    saved.up.fill_(1.0)
    x = torch.zeros(m, 8, dtype=torch.bfloat16, device=DEV)
    x[0, 0] = 1.0                                               # dWg of the first input is dg of the first token
    w = torch.zeros(n, 8, dtype=torch.bfloat16, device=DEV)
    grad_h = torch.full((m, n), 2.0 ** -130, dtype=torch.bfloat16, device=DEV)
    _, grad_wg, _, _ = gws.gated_bwd(grad_h, x, w, w, saved, act, want_grad_x=False)
    assert torch.equal(grad_wg[:, 0], torch.where(g > 0, grad_h[0], torch.zeros_like(grad_h[0])))
