"""Every way in which the products of the activation operators are tiled, and the sizes that take it: what the library plans for each size
is checked on the host, what it computes against the 64-bit forms of test_gpu_gated.py and test_gpu_act8.py.

A path is (blocks a tile, columns of its accumulator, form): "whole" tiles in one wave, "whole*" in several, "cut" contractions joined by a
second launch, "cut*" with more parts than fit one wave, "whole+cut" for a last wave that is cut, "cluster" for parts joined in place."""
import ctypes
import threading

import pytest
import torch

import act_reference as ref
import paper_2505_11170_b200 as gws
import test_gpu_act8 as act8_tests
import test_gpu_gated as gated_tests
from paper_2505_11170_b200.binding import GatedDesc

DEV = "cuda"

# forward: (path, operand copied to whole lines first, m, n, k)
FORWARD = [
    ((1, "narrow", "whole"), "", 9, 1200, 264), ((1, "narrow", "whole"), "x", 9, 1200, 2840), ((1, "narrow", "whole*"), "", 35, 13023, 80),
    ((1, 128, "cut"), "", 20, 100, 3080), ((1, 128, "cut"), "w", 1905, 8, 3944), ((1, 128, "cut"), "x", 5, 1096, 2824),
    ((1, 128, "whole"), "w", 3697, 280, 2696), ((1, 128, "whole"), "x", 566, 1616, 2600), ((1, 128, "whole*"), "", 19127, 40, 16),
    ((1, 128, "whole*"), "w", 8863, 919, 24), ((1, 128, "whole*"), "x", 793, 2440, 1048),
    ((2, 128, "cut"), "", 161, 328, 1960), ((2, 128, "cut"), "w", 2044, 80, 2824), ((2, 128, "cut"), "x", 265, 632, 3608),
    ((2, 128, "whole"), "w", 2570, 112, 3096), ((2, 128, "whole"), "x", 324, 840, 3512), ((2, 128, "whole*"), "", 1073, 1080, 264),
    ((2, 128, "whole*"), "w", 2955, 840, 1448), ((2, 128, "whole*"), "x", 774, 3096, 920), ((2, 128, "whole+cut"), "", 1191, 936, 2272),
    ((2, 128, "whole+cut"), "w", 3369, 688, 1880), ((2, 128, "whole+cut"), "x", 1506, 1592, 1896), ((2, 128, "whole+cut"), "xw", 976, 1187, 2589),
    ((2, 256, "whole"), "", 671, 1608, 400), ((2, 256, "whole"), "w", 3105, 328, 2088), ((2, 256, "whole"), "x", 581, 1962, 2056),
    ((2, 256, "whole"), "xw", 904, 1212, 389), ((2, 256, "whole*"), "", 1059, 2912, 288), ((2, 256, "whole*"), "w", 5614, 856, 648),
    ((2, 256, "whole*"), "x", 850, 3944, 856), ((2, 256, "whole+cut"), "", 1044, 1864, 1184), ((2, 256, "whole+cut"), "w", 3761, 1256, 904),
    ((2, 256, "whole+cut"), "x", 1175, 1912, 1304), ((2, 256, "whole+cut"), "xw", 750, 3150, 1206),
    ((1, 128, "whole+cut"), "", 1, 9495, 19848), ((2, 128, "cut*"), "xw", 6537, 9, 12066), ((2, 256, "cut"), "w", 3149, 72, 7304),
    ((2, 256, "cut*"), "xw", 274, 1572, 17165),
]
# dx: (path, m, n, k)
GRAD_X = [
    ((1, 128, "cluster"), 3, 200, 136), ((1, 128, "cut"), 7, 3500, 136), ((1, 128, "whole*"), 1054, 11, 3779), ((2, 128, "cut"), 388, 1678, 140),
    ((2, 128, "cut*"), 1060, 5516, 1034), ((2, 128, "whole"), 129, 130, 72), ((2, 128, "whole*"), 19127, 40, 16), ((2, 128, "whole+cut"), 1259, 1240, 1800),
    ((2, 256, "cut"), 540, 3634, 1552), ((2, 256, "whole"), 9666, 15, 132), ((2, 256, "whole*"), 1157, 154, 3760), ((2, 256, "whole+cut"), 3653, 703, 1223),
    ((1, 128, "whole"), 1, 8, 9), ((1, 128, "cut*"), 1, 3417, 10539), ((1, 128, "whole+cut"), 1, 402, 19330), ((2, 256, "cut*"), 6301, 7360, 132),
]
# the pair of weight gradients: (path, x converted inside, restored before, or in BF16, m, n, k)
GRAD_W = [
    ((1, 128, "cluster"), "bf16", 1487, 90, 139), ((1, 128, "cut"), "bf16", 10781, 73, 68), ((1, 128, "cut*"), "bf16", 12049, 120, 3195),
    ((1, 128, "whole*"), "bf16", 34, 3895, 268), ((2, 128, "cut"), "bf16", 3932, 155, 137), ((2, 128, "cut*"), "bf16", 14699, 275, 875),
    ((2, 128, "whole"), "bf16", 772, 1416, 276), ((2, 128, "whole*"), "bf16", 202, 552, 1816), ((2, 128, "whole+cut"), "bf16", 1611, 1224, 1840),
    ((2, 256, "cut"), "bf16", 7000, 1061, 446), ((2, 256, "cut*"), "bf16", 16533, 335, 1762), ((2, 256, "whole"), "bf16", 148, 513, 1860),
    ((2, 256, "whole*"), "bf16", 261, 1056, 2144), ((2, 256, "whole+cut"), "bf16", 1575, 3184, 696),
    ((1, 128, "cluster"), "inside", 502, 8, 840), ((1, 128, "cut"), "inside", 8085, 9, 122), ((1, 128, "cut*"), "inside", 11593, 9, 2589),
    ((1, 128, "whole"), "inside", 127, 10, 3366), ((2, 128, "cut"), "inside", 10225, 129, 249), ((2, 128, "whole"), "inside", 492, 19, 3950),
    ((2, 256, "cut"), "inside", 4369, 176, 1576), ((2, 256, "cut*"), "inside", 15577, 304, 1712), ((2, 256, "whole"), "inside", 179, 272, 3262),
    ((2, 256, "whole*"), "inside", 124, 1796, 3099),
    ((1, 128, "cluster"), "restored", 1487, 90, 139), ((1, 128, "cut"), "restored", 10781, 73, 68), ((1, 128, "whole*"), "restored", 34, 3895, 268),
    ((2, 128, "cut"), "restored", 3932, 155, 137), ((2, 128, "cut*"), "restored", 13432, 416, 812), ((2, 128, "whole"), "restored", 772, 1416, 276),
    ((2, 128, "whole*"), "restored", 202, 552, 1816), ((2, 128, "whole+cut"), "restored", 1611, 1224, 1840), ((2, 256, "cut"), "restored", 7000, 1061, 446),
    ((2, 256, "cut*"), "restored", 16606, 1720, 408), ((2, 256, "whole"), "restored", 148, 513, 1860), ((2, 256, "whole*"), "restored", 261, 1056, 2144),
    ((2, 256, "whole+cut"), "restored", 1575, 3184, 696),
    ((1, 128, "whole"), "bf16", 33, 97, 41), ((1, 128, "whole+cut"), "bf16", 1018, 10, 9566), ((1, 128, "whole"), "restored", 33, 97, 41),
    ((1, 128, "whole*"), "inside", 79, 8, 10805), ((1, 128, "whole+cut"), "inside", 656, 11, 9537), ((2, 128, "whole*"), "inside", 91, 130, 20221),
    ((2, 128, "whole+cut"), "inside", 4731, 11, 4776), ((2, 256, "whole+cut"), "inside", 1031, 143, 9735),
]
# a layer's weight gradient from a checkpoint; several of the whole waves have an odd number of stages
WGRAD = [
    ((1, 128, "cluster"), "inside", 1152, 56, 145), ((1, 128, "cut"), "inside", 16384, 96, 128), ((1, 128, "cut*"), "inside", 19533, 19, 3955),
    ((1, 128, "whole"), "inside", 65, 40, 72), ((1, 128, "whole*"), "inside", 315, 2056, 2110), ((2, 128, "cut"), "inside", 12306, 152, 24),
    ((2, 128, "whole"), "inside", 394, 56, 16), ((2, 128, "whole*"), "inside", 338, 2696, 1654), ((2, 128, "whole+cut"), "inside", 6016, 528, 3161),
    ((2, 256, "cut"), "inside", 3865, 536, 1256), ((2, 256, "cut*"), "inside", 12128, 525, 2223), ((2, 256, "whole"), "inside", 144, 1808, 1176),
    ((2, 256, "whole*"), "inside", 140, 3736, 1173), ((2, 256, "whole+cut"), "inside", 1292, 1272, 3735),
    ((2, 128, "cut"), "inside", 8192, 768, 768), ((2, 256, "cut"), "inside", 16384, 512, 2048), ((2, 256, "whole+cut"), "restored", 16384, 2048, 5632),
    ((1, 128, "cluster"), "restored", 387, 11, 20), ((1, 128, "cut"), "restored", 1072, 76, 17), ((1, 128, "whole*"), "restored", 16, 4745, 399),
    ((2, 128, "cut"), "restored", 13181, 138, 23), ((2, 128, "cut*"), "restored", 13972, 1138, 529), ((2, 128, "whole"), "restored", 429, 20, 18),
    ((2, 128, "whole*"), "restored", 209, 2051, 1082), ((2, 128, "whole+cut"), "restored", 2427, 1191, 1816), ((2, 256, "cut"), "restored", 7198, 1126, 937),
    ((2, 256, "cut*"), "restored", 15537, 1203, 1195), ((2, 256, "whole"), "restored", 132, 1300, 1725), ((2, 256, "whole*"), "restored", 285, 1826, 2497),
    ((2, 256, "whole+cut"), "restored", 1666, 3829, 1176),
    ((1, 128, "whole"), "restored", 2, 10, 8), ((1, 128, "whole+cut"), "inside", 675, 9, 19652),
]


def _path(plan):
    many = "*" if plan.waves > 1 else ""
    if plan.clustered:
        form = "cluster"
    elif plan.cut and plan.splits > 1:
        form = "whole+cut" if plan.whole else "cut" + many
    else:
        form = "whole" + many
    return plan.blocks, "narrow" if plan.narrow else plan.columns, form


@pytest.mark.parametrize("path,moves,m,n,k", FORWARD)
def test_plan_of_the_forward_pass(path, moves, m, n, k):
    plan = gws.gated_plan(m, n, k, "h")
    assert (_path(plan), "x" * plan.moves_x + "w" * plan.moves_w) == (path, moves)


@pytest.mark.parametrize("path,m,n,k", GRAD_X)
def test_plan_of_the_input_gradient(path, m, n, k):
    assert _path(gws.gated_plan(m, n, k, "grad_x")) == path


@pytest.mark.parametrize("path,x,m,n,k", GRAD_W)
def test_plan_of_the_pair_of_weight_gradients(path, x, m, n, k):
    plan = gws.gated_plan(m, n, k, "grad_w", x_format=gws.SAVE_BF16 if x == "bf16" else gws.ACT8_E4M3)
    assert (_path(plan), bool(plan.inside)) == (path, x == "inside")


@pytest.mark.parametrize("path,x,m,n,k", WGRAD)
def test_plan_of_a_weight_gradient(path, x, m, n, k):
    plan = gws.wgrad_act8_plan(m, n, k)
    assert (_path(plan), bool(plan.inside)) == (path, x == "inside")


def test_the_lists_hold_every_form_of_every_tile():
    # what a search over some million sizes up to 70000 x 40000 x 40000 came upon
    forms = {(1, 128): {"whole", "whole*", "cut", "cut*", "whole+cut", "cluster"}, (2, 128): {"whole", "whole*", "cut", "cut*", "whole+cut"},
             (2, 256): {"whole", "whole*", "cut", "cut*", "whole+cut"}}

    def held(entries, kind=None):
        return {t: {e[0][2] for e in entries if e[0][:2] == t and (kind is None or e[1] == kind)} for t in forms}

    without = lambda *left_out: {t: f - {x for tile, x in left_out if tile == t} for t, f in forms.items()}
    assert {t: f for t, f in held([e for e in FORWARD if e[0][1] != "narrow"]).items()} == without(((1, 128), "cluster"), ((1, 128), "cut*"))
    assert held(GRAD_X) == forms
    assert held(GRAD_W, "bf16") == forms
    assert held(GRAD_W, "restored") == without(((1, 128), "cut*"), ((1, 128), "whole+cut"))
    assert held(GRAD_W, "inside") == without(((2, 128), "cut*"))
    assert held(WGRAD, "restored") == without(((1, 128), "cut*"), ((1, 128), "whole+cut"))
    assert held(WGRAD, "inside") == without(((2, 128), "cut*"))


def test_plans_of_empty_and_impossible_sizes():
    for plan in (gws.gated_plan(0, 8, 8, "h"), gws.gated_plan(4, 0, 8, "grad_x"), gws.wgrad_act8_plan(4, 8, 0)):
        assert plan.blocks == plan.whole == plan.cut == 0
    for call in (lambda: gws.gated_plan(-1, 8, 8, "h"), lambda: gws.gated_plan(4, 8, 8, "h", ld_x=7), lambda: gws.wgrad_act8_plan(1 << 31, 8, 8)):
        with pytest.raises(gws.GwsError):
            call()
    with pytest.raises(ValueError):
        gws.gated_plan(4, 8, 8, "grad_h")


# ---- on the device -----------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("path,moves,m,n,k", FORWARD)
def test_forward(path, moves, m, n, k):
    for act in gated_tests.ACTS:
        gated_tests.test_forward(act, m, n, k)
    for save in (gws.ACT8_INT8, gws.ACT8_E4M3, gws.SAVE_BF16):
        gated_tests.test_what_forward_keeps(save, m, n, k)


def _backward(m, n, k, x_format, want, act):
    x, wg, wu, grad_h = gated_tests._problem(m, n, k)
    save = gws.SAVE_BF16 if x_format == gws.SAVE_BF16 else x_format
    _, saved = gws.gated_fwd(x, wg, wu, act, save=save)
    x_in = x if x_format == gws.SAVE_BF16 else gws.act8_save(x, x_format)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    call = lambda **kw: gws.gated_bwd(grad_h, x_in, wg, wu, saved, act, want_grad_x="x" in want, want_grad_w="w" in want, **kw)
    got = call(status=status)
    gated_tests.check_backward(got, grad_h, x.double() if x_in is x else ref.decode(x_in), wg, wu, *gated_tests.saved_values(saved), act)
    assert int(status) == 0
    assert all(p is q is None or torch.equal(p, q) for p, q in zip(got, call()))


@pytest.mark.gpu
@pytest.mark.parametrize("path,m,n,k", GRAD_X)
def test_input_gradient(path, m, n, k):
    _backward(m, n, k, gws.SAVE_BF16, "x", gws.GATED_GELU_TANH)


@pytest.mark.gpu
@pytest.mark.parametrize("path,x,m,n,k", GRAD_W)
def test_pair_of_weight_gradients(path, x, m, n, k):
    for fmt in (gws.SAVE_BF16,) if x == "bf16" else (gws.ACT8_INT8, gws.ACT8_E4M3):
        _backward(m, n, k, fmt, "w", gws.GATED_SILU)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [gws.ACT8_INT8, gws.ACT8_E4M3])
@pytest.mark.parametrize("path,x,m,n,k", WGRAD)
def test_weight_gradient(path, x, m, n, k, fmt):
    act8_tests.test_weight_gradient_from_a_checkpoint(fmt, m, n, k)


GUARD = 1 << 12


class Guarded:
    """A region of a tensor of known bytes: what a kernel writes beside it shows."""

    def __init__(self, nbytes, offset=0):
        self.nbytes, self.first = nbytes, GUARD + offset
        self.all = torch.full((nbytes + 2 * GUARD,), 0xA5, dtype=torch.uint8, device=DEV)

    @property
    def p(self):
        return self.all.data_ptr() + self.first

    def bf16(self, *shape):
        return self.all[self.first:self.first + self.nbytes].view(torch.bfloat16).view(*shape)

    def untouched(self):
        return bool((self.all[:self.first] == 0xA5).all()) and bool((self.all[self.first + self.nbytes:] == 0xA5).all())


# (m, n, k): odd everywhere; few rows; ragged last group and tile; whole tiles; a cut and a cluster
GUARDED = [(33, 97, 41), (1, 2309, 72), (130, 1364, 511), (300, 520, 264), (257, 256, 128), (1500, 90, 139), (161, 328, 1960), (1191, 937, 2271)]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [gws.ACT8_INT8, gws.ACT8_E4M3, gws.SAVE_BF16])
@pytest.mark.parametrize("m,n,k", GUARDED)
def test_outputs_kept_values_and_workspaces_are_written_inside_their_bounds(m, n, k, fmt):
    lib = gws.load_library()
    x, wg, wu, grad_h = gated_tests._problem(m, n, k)
    h, saved = gws.gated_fwd(x, wg, wu, gws.GATED_SILU, save=fmt)
    x_in = x if fmt == gws.SAVE_BF16 else gws.act8_save(x, fmt)
    want = gws.gated_bwd(grad_h, x_in, wg, wu, saved, gws.GATED_SILU, want_h=True)
    stream = torch.cuda.current_stream().cuda_stream
    part = 2 * m * n if fmt == gws.SAVE_BF16 else gws.act8_layout(m, n)[2]
    odd = 2                                              # outputs at any 2-byte alignment
    # tensor maps read rows on 16-byte boundaries; what torch allocates is
    d = GatedDesc(m, n, k, k, k, n, gws.GATED_SILU, fmt, fmt, 0)
    at = ctypes.addressof(d)
    need = lib.gws_gated_workspace_bytes(at, 0), lib.gws_gated_workspace_bytes(at, 1)
    out, gate, up, ws = Guarded(2 * m * n, odd), Guarded(part), Guarded(part), Guarded(max(need))
    assert lib.gws_gated_fwd(at, x.data_ptr(), wg.data_ptr(), wu.data_ptr(), out.p, gate.p, up.p, ws.p, need[0], None, stream) == 0
    torch.cuda.synchronize()
    assert all(g.untouched() for g in (out, gate, up, ws))
    assert torch.equal(out.bf16(m, n), h)
    for mine, theirs in ((gate, saved.gate), (up, saved.up)):
        if fmt == gws.SAVE_BF16:
            assert torch.equal(mine.bf16(m, n), theirs)
        else:
            codes, scales, total = gws.act8_layout(m, n)
            a = mine.all[mine.first:mine.first + total]
            assert torch.equal(a[:codes], theirs.buffer[:codes]) and torch.equal(a[scales:], theirs.buffer[scales:total])
    gx, gg, gu, hh = Guarded(2 * m * k, odd), Guarded(2 * n * k, odd), Guarded(2 * n * k), Guarded(2 * m * n, odd)
    x_p = x.data_ptr() if fmt == gws.SAVE_BF16 else x_in.buffer.data_ptr()
    assert lib.gws_gated_bwd(at, grad_h.data_ptr(), x_p, wg.data_ptr(), wu.data_ptr(), gate.p, up.p, gx.p, gg.p, gu.p, hh.p, ws.p, need[1], None, stream) == 0
    torch.cuda.synchronize()
    assert all(g.untouched() for g in (gx, gg, gu, hh, gate, up, ws))
    assert all(torch.equal(g.bf16(*w.shape), w) for g, w in zip((gx, gg, gu, hh), want))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [gws.ACT8_INT8, gws.ACT8_E4M3])
@pytest.mark.parametrize("m,n,k", [(33, 97, 41), (515, 768, 768), (1072, 76, 17), (3001, 511, 682), (4439, 133, 1577)])
def test_weight_gradients_and_checkpoints_are_written_inside_their_bounds(m, n, k, fmt):
    lib = gws.load_library()
    gy, x = gated_tests._rand(m, n, 1, 1e-3), gated_tests._rand(m, k, 2)
    kept = gws.act8_save(x, fmt)
    want, back = gws.wgrad_act8(gy, kept), gws.act8_load(kept)
    stream = torch.cuda.current_stream().cuda_stream
    codes, scales, total = gws.act8_layout(m, k)
    x8, xb, need = Guarded(total), Guarded(2 * m * k, 2), lib.gws_wgrad_act8_workspace_bytes(m, n, k, n)
    gw, ws = Guarded(2 * n * k, 2), Guarded(need)
    assert lib.gws_act8_save(m, k, k, fmt, x.data_ptr(), x8.p, stream) == 0
    assert lib.gws_act8_load(m, k, k, fmt, x8.p, xb.p, stream) == 0
    assert lib.gws_wgrad_act8(m, n, k, fmt, gy.data_ptr(), n, x8.p, gw.p, k, ws.p if need else None, need, None, stream) == 0
    torch.cuda.synchronize()
    assert all(g.untouched() for g in (x8, xb, gw, ws))
    a = x8.all[x8.first:x8.first + total]
    assert torch.equal(a[:codes], kept.buffer[:codes]) and torch.equal(a[scales:], kept.buffer[scales:total])
    assert torch.equal(xb.bf16(m, k), back) and torch.equal(gw.bf16(n, k), want)


@pytest.mark.gpu
def test_host_threads_with_streams_of_their_own():
    # plans are kept per thread, workspaces come from each thread's stream
    sizes = [(300, 520, 263), (33, 97, 41), (1, 2309, 72), (700, 1000, 520), (1500, 90, 139), (129, 130, 72)]

    def step(m, n, k, stream=None):
        x, wg, wu, dh = gated_tests._problem(m, n, k)
        torch.cuda.current_stream().synchronize()
        h, saved = gws.gated_fwd(x, wg, wu, save=gws.ACT8_INT8)
        x8 = gws.act8_save(x)
        return (h, *gws.gated_bwd(dh, x8, wg, wu, saved, want_h=True), gws.wgrad_act8(dh, x8))

    want = [step(*s) for s in sizes]
    torch.cuda.synchronize()
    wrong, errors = [], []

    def work(turn):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for i in range(12):
                    at = (i * (turn + 1) + turn) % len(sizes)
                    got = step(*sizes[at])
                    stream.synchronize()
                    if not all(torch.equal(p, q) for p, q in zip(got, want[at])):
                        wrong.append((turn, sizes[at]))
        except Exception as e:                            # shown by the assertion below
            errors.append(e)

    threads = [threading.Thread(target=work, args=(t,)) for t in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors and not wrong
