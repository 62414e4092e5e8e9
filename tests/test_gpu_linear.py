"""Linear layer with bias, activation and residual, forward and backward, against plain forms in 64 bits."""
import math

import pytest
import torch

import act_reference as ref
import paper_2505_11170_b200 as gws

pytestmark = pytest.mark.gpu
DEV = "cuda"
ACTS = [gws.ACT_NONE, gws.GATED_SILU, gws.GATED_GELU_TANH, gws.GATED_RELU]
# (m, n, k): one token to many, widths that are and are not multiples of the tiles, of 32, of 8; all odd
SHAPES = [(1, 64, 64), (1, 5632, 256), (3, 8, 8), (33, 96, 40), (128, 128, 128), (129, 130, 72), (200, 1365, 512), (257, 2048, 96), (300, 33, 31), (640, 1000, 333), (1, 1, 1),
          (2048, 256, 768), (1500, 2730, 64), (65, 768, 2730)]
# every way of tiling the forward product: (blocks, columns, form, m, n, k); warps that stream rows (0 blocks), narrow tiles of 16 to 128 columns, in one wave and in several
TILINGS = [(0, 8, "rows", 1, 5632, 2048), (0, 4, "rows", 1, 9, 2104), (0, 8, "rows", 1, 100, 8), (0, 4, "rows", 2, 1000, 4096), (0, 8, "rows", 2, 5000, 1032), (0, 16, "rows", 2, 9601, 264),
           (0, 16, "rows", 3, 9600, 264), (0, 8, "rows", 3, 770, 768), (0, 4, "rows", 4, 2050, 1032), (0, 16, "rows", 4, 7, 8), (1, 48, "narrow", 5, 5632, 2048), (1, 16, "narrow", 33, 2050, 768), (1, 48, "narrow", 72, 5858, 1807), (1, 80, "narrow", 128, 11008, 264), (1, 16, "narrow", 6, 40, 72),
           (1, 128, "cut", 1, 10, 4009), (1, 128, "cut", 70, 330, 9000), (1, 128, "cluster", 314, 859, 2745), (1, 128, "cluster", 1, 8, 700), (1, 128, "cluster", 40, 130, 1500),
           (2, 128, "whole", 224, 220, 1139), (1, 128, "whole", 268, 5533, 383), (1, 128, "whole*", 796, 2930, 8), (2, 128, "cut", 477, 701, 5986), (2, 128, "whole+cut", 3002, 864, 3835),
           (1, 128, "whole", 213, 532, 102), (2, 128, "whole*", 3955, 534, 294), (2, 256, "cut", 267, 1686, 9306), (2, 256, "whole+cut", 1112, 3767, 1200), (2, 256, "whole", 2650, 920, 445),
           (2, 256, "whole*", 783, 7541, 340)]

def rand(shape, seed, std=1.0, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).to(DEV)


def problem(m, n, k, bias="bf16", residual=True):
    x, w = rand((m, k), 1), rand((n, k), 2, 1.5 / math.sqrt(k))
    b = None if bias is None else rand((n,), 5, 0.5, torch.float32 if bias == "f32" else torch.bfloat16)
    return x, w, b, rand((m, n), 3) if residual else None, rand((m, n), 4, 1e-2)


def act(z, kind):
    return (z, torch.ones_like(z)) if kind == gws.ACT_NONE else ref.act(z, kind)


def pre_activation(x, w, b):
    """z in 64 bits and the error that FP32 sums over k may leave in it."""
    x, w = x.double(), w.double()
    z = x @ w.t()
    e = (x.shape[1] + 64) * 2.0 ** -23 * (x.abs() @ w.abs().t())
    if b is not None:
        z = z + b.double()
        e = e + 2.0 ** -24 * z.abs()
    return z, e


def within(got, want, bound):
    return bool(((got.double() - want).abs() <= bound).all())


def check_forward(x, w, b, r, kind, save=gws.SAVE_NONE, **more):
    y, saved = gws.linear_fwd(x, w, b, residual=r, activation=kind, save=save, **more)
    z, e = pre_activation(x, w, b)
    a, _ = act(z, kind)
    want = a if r is None else a + r.double()
    # rounding of y, the error of z through a slope of at most 1.2, 2^-19 for exp and division, half an ulp of FP32 for the residual
    assert within(y, want, 2.0 ** -8 * want.abs() + 1.2 * e + 2.0 ** -18 * a.abs() + 2.0 ** -23 * want.abs() + 1e-38)
    return y, saved, z, e


def check_kept(saved, save, z, e):
    m, n = z.shape
    if save == gws.SAVE_BF16:
        assert within(saved, z, 2.0 ** -8 * z.abs() + e + 1e-38)
        return saved.double()
    got, want = ref.decode(saved), ref.values(*ref.encode(z, save), n)
    top = torch.nn.functional.pad(z.abs() + e, (0, -n % 32)).view(m, -1, 32).amax(-1)
    step = torch.exp2(torch.floor(torch.log2(top.clamp(min=1e-300)))) * (1.0 / 64 if save == gws.ACT8_INT8 else 1.0 / 4)
    assert within(got, z, step.repeat_interleave(32, 1)[:, :n] + e)
    assert float((got != want).double().mean()) < 0.01             # a rounding that FP32 sums decide otherwise is rare
    assert not bool(saved.codes[:, n:].any())
    return got


def check_backward(dy, x, w, saved, z, kind, grads, bias_dtype=torch.bfloat16):
    """``x`` and ``z`` in 64 bits, as kept."""
    dx, dw, db, again = grads
    m, n = dy.shape
    a, slope = act(z, kind)
    dz = dy.double() * slope
    e = 2.0 ** -18 * dy.double().abs() if kind != gws.ACT_NONE else torch.zeros_like(dz)
    e16 = e + (2.0 ** -8 * dz.abs() if kind != gws.ACT_NONE else 0.0)          # dz is BF16 for the products, dy itself without an activation
    if dx is not None:
        want = dz @ w.double()
        assert within(dx, want, 2.0 ** -8 * want.abs() + 1.01 * (e16 @ w.double().abs()) + (n + 64) * 2.0 ** -23 * (dz.abs() @ w.double().abs()) + 1e-38)
    if dw is not None:
        want = dz.t() @ x
        assert within(dw, want, 2.0 ** -8 * want.abs() + 1.01 * (e16.t() @ x.abs()) + (m + 64) * 2.0 ** -23 * (dz.abs().t() @ x.abs()) + 1e-38)
    if db is not None:
        want = dz.sum(0)
        assert db.dtype == bias_dtype
        assert within(db, want, (2.0 ** -8 if bias_dtype == torch.bfloat16 else 2.0 ** -24) * want.abs() * 1.01 + (m + 64) * 2.0 ** -24 * dz.abs().sum(0) + 1.01 * e.sum(0) + 1e-38)
    if again is not None:
        assert within(again, a, 2.0 ** -8 * a.abs() + 2.0 ** -18 * a.abs() + 1e-38)


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_forward(kind, m, n, k):
    x, w, b, r, _ = problem(m, n, k)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    y = check_forward(x, w, b, r, kind, status=status)[0]
    assert int(status) == 0
    assert torch.equal(y, gws.linear_fwd(x, w, b, residual=r, activation=kind)[0])
    check_forward(x, w, None, None, kind)
    check_forward(x, w, b.float(), None, kind)


@pytest.mark.parametrize("save", [gws.ACT8_INT8, gws.ACT8_E4M3, gws.SAVE_BF16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_training_step(save, m, n, k):
    x, w, b, r, dy = problem(m, n, k, "f32")
    kind = ACTS[1 + (m + n) % 3]
    y, saved, z, e = check_forward(x, w, b, r, kind, save)
    assert torch.equal(y, gws.linear_fwd(x, w, b, residual=r, activation=kind)[0])          # what is kept does not change y
    kept = check_kept(saved, save, z, e)
    for source in (x, gws.act8_save(x, gws.ACT8_INT8), gws.act8_save(x, gws.ACT8_E4M3)):
        grads = gws.linear_bwd(dy, source, w, saved, kind, want_grad_bias=True, want_act=True, bias_dtype=torch.float32)
        check_backward(dy, ref.decode(source) if isinstance(source, gws.Act8) else x.double(), w, saved, kept, kind, grads, torch.float32)
        again = gws.linear_bwd(dy, source, w, saved, kind, want_grad_bias=True, want_act=True, bias_dtype=torch.float32)
        assert all(torch.equal(p, q) for p, q in zip(grads, again))                         # nothing depends on timing


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_without_an_activation(m, n, k):
    x, w, b, _, dy = problem(m, n, k)
    grads = gws.linear_bwd(dy, x, w, want_grad_bias=True)
    check_backward(dy, x.double(), w, None, torch.zeros(m, n, dtype=torch.float64, device=DEV), gws.ACT_NONE, grads)
    y, saved = gws.linear_fwd(x, w, b, save=gws.ACT8_INT8)
    again = gws.linear_bwd(dy, x, w, saved, want_grad_x=False, want_grad_w=False, want_act=True)
    assert again[:3] == (None, None, None) and torch.equal(again[3], gws.act8_load(saved))


@pytest.mark.parametrize("blocks,columns,form,m,n,k", TILINGS)
def test_every_tiling(blocks, columns, form, m, n, k):
    p = gws.linear_plan(m, n, k)
    got = "rows" if not p.blocks else "narrow" if p.narrow else "cluster" if p.clustered else "whole+cut" if p.cut and p.whole else "cut" if p.cut else "whole*" if p.waves > 1 else "whole"
    assert (p.blocks, p.columns, got) == (blocks, columns, form)
    x, w, b, r, _ = problem(m, n, k)
    for save in (gws.ACT8_INT8, gws.ACT8_E4M3, gws.SAVE_BF16):
        _, saved, z, e = check_forward(x, w, b, r, gws.GATED_GELU_TANH, save)
        check_kept(saved, save, z, e)


@pytest.mark.parametrize("blocks,columns,form,m,n,k", TILINGS[14:])
def test_every_tiling_without_a_residual(blocks, columns, form, m, n, k):
    x, w, b, _, _ = problem(m, n, k, "f32")
    for save in (gws.ACT8_INT8, gws.SAVE_BF16):
        _, saved, z, e = check_forward(x, w, b, None, gws.GATED_SILU, save)
        check_kept(saved, save, z, e)


# residuals in rows that a lane reads by whole lines: tiles of 128 and 256 columns, one wave and several, whole and cut, widths that end inside a chunk of 32 columns
@pytest.mark.parametrize("m,n,k", [(300, 528, 136), (2650, 912, 448), (2049, 1008, 64), (1112, 3760, 1200), (3002, 880, 3840), (4100, 2064, 72), (129, 16, 4096)])
def test_residuals_of_whole_lines(m, n, k):
    x, w, b, r, _ = problem(m, n, k)
    first = check_forward(x, w, b, r, gws.ACT_NONE, gws.ACT8_INT8)[0]
    check_forward(x, w, b, r, gws.GATED_GELU_TANH)
    wide = torch.cat([r, r], 1)
    assert torch.equal(gws.linear_fwd(x, w, b, residual=wide[:, n:], save=gws.ACT8_INT8)[0], first)
    assert torch.equal(gws.linear_fwd(x, w, b, residual=wide[:, :n].t().contiguous().t(), save=gws.ACT8_INT8)[0], first)


@pytest.mark.parametrize("n,k", [(136, 72), (137, 71), (64, 2048)])
def test_strides_and_alignments(n, k):
    m = 45
    big_x, big_w, big_r = rand((m, k + 9), 1), rand((n, k + 5), 2, 1.0 / math.sqrt(k)), rand((m, n + 7), 3)
    for x, w, r in ((big_x[:, :k], big_w[:, :k], big_r[:, :n]), (big_x[:, 3:3 + k], big_w[:, 5:5 + k], big_r[:, 7:7 + n]), (rand((k, m), 4).t(), rand((k, n), 5, 0.2).t(), rand((n, m), 6).t()),
                    (big_x[:1, :k].expand(m, k), big_w[:, 1:1 + k], big_r[:1, 1:1 + n].expand(m, n))):
        b = rand((n + 1,), 8)[1:]
        _, saved, z, e = check_forward(x, w, b, r, gws.GATED_SILU, gws.SAVE_BF16)
        kept = check_kept(saved, gws.SAVE_BF16, z, e)
        dy = r
        check_backward(dy, x.double(), w, saved, kept, gws.GATED_SILU, gws.linear_bwd(dy, x, w, saved, gws.GATED_SILU, want_grad_bias=True, want_act=True))
        check_backward(dy, x.double(), w, None, kept, gws.ACT_NONE, (*gws.linear_bwd(dy, x, w, want_grad_bias=True)[:3], None))


def test_values_that_are_not_finite_stay_in_their_rows_and_columns():
    m, n, k = 70, 96, 64
    x, w, b, r, dy = problem(m, n, k)
    clean, kept = gws.linear_fwd(x, w, b, residual=r, activation=gws.GATED_RELU, save=gws.ACT8_INT8)
    x2, b2 = x.clone(), b.clone()
    x2[5, 3] = float("nan")
    b2[40] = float("inf")
    y, saved = gws.linear_fwd(x2, w, b2, residual=r, activation=gws.GATED_RELU, save=gws.ACT8_INT8)
    assert bool(y[5].isnan().all()) and bool((y[:5, 40] == math.inf).all())
    same = torch.ones_like(y, dtype=torch.bool)
    same[5], same[:, 40] = False, False
    assert torch.equal(y[same], clean[same])
    z = gws.act8_load(saved)
    assert bool(z[5].isnan().all()) and bool(z[0, 32:64].isnan().all()) and bool(z[0, :32].isfinite().all()) and bool(z[0, 64:].isfinite().all())
    grads = gws.linear_bwd(dy, x, w, kept, gws.GATED_RELU, want_grad_bias=True, want_act=True)
    dy2 = dy.clone()
    dy2[7, 11] = float("nan")
    z8 = gws.linear_fwd(x, w, b, activation=gws.GATED_SILU, save=gws.ACT8_INT8)[1]
    dx, dw, db, _ = gws.linear_bwd(dy2, x, w, z8, gws.GATED_SILU, want_grad_bias=True)
    bad = torch.zeros(n, dtype=torch.bool, device=DEV)
    bad[11] = True
    assert bool(dx[7].isnan().all()) and bool(dx[:7].isfinite().all()) and bool(dx[8:].isfinite().all())
    assert torch.equal(db.isnan(), bad) and torch.equal(dw.isnan().all(1), bad) and bool(dw[~bad].isfinite().all())
    assert all(bool(t.isfinite().all()) for t in grads)


def test_a_checkpoint_that_is_not_finite_reaches_only_its_own_columns():
    """The last group of a row is short: what stands for the columns past the width must not reach a sum."""
    m, n, k = 40, 70, 32
    x, w, b, _, dy = problem(m, n, k)
    b[69] = float("inf")
    _, saved = gws.linear_fwd(x, w, b, activation=gws.GATED_SILU, save=gws.ACT8_E4M3)
    dx, dw, db, again = gws.linear_bwd(dy, x, w, saved, gws.GATED_SILU, want_grad_bias=True, want_act=True)
    assert bool(db[:64].isfinite().all()) and bool(db[64:].isnan().all()) and bool(dw[:64].isfinite().all()) and bool(again[:, 64:].isnan().all())


def test_sizes_of_zero():
    x, w, b, r, dy = problem(8, 16, 24)
    y, saved = gws.linear_fwd(x[:0], w, b, residual=r[:0], activation=gws.GATED_SILU, save=gws.ACT8_INT8)
    assert y.shape == (0, 16)
    dx, dw, db, a = gws.linear_bwd(dy[:0], x[:0], w, saved, gws.GATED_SILU, want_grad_bias=True, want_act=True)
    assert dx.shape == (0, 24) and a.shape == (0, 16) and not bool(dw.any()) and not bool(db.any())
    y, _ = gws.linear_fwd(x, w[:0], b[:0])
    assert y.shape == (8, 0)
    dx, dw, db, _ = gws.linear_bwd(dy[:, :0], x, w[:0], want_grad_bias=True)
    assert not bool(dx.any()) and dw.shape == (0, 24) and db.shape == (0,)


def test_gradients_against_differences_of_the_forward_pass():
    m, n, k = 9, 12, 10
    x, w, b, _, dy = problem(m, n, k, "f32")
    for kind in (gws.ACT_NONE, gws.GATED_SILU, gws.GATED_GELU_TANH):
        _, saved = gws.linear_fwd(x, w, b, activation=kind, save=gws.SAVE_BF16)
        grads = gws.linear_bwd(dy, x, w, saved, kind, want_grad_bias=True, bias_dtype=torch.float32)
        leaves = [x.double(), w.double(), b.double()]
        for i, (grad, leaf) in enumerate(zip(grads[:3], leaves)):
            for seed in range(3):
                way = torch.randn(leaf.shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).to(DEV)
                ends = []
                for h in (1e-5, -1e-5):
                    p = [t + h * way if j == i else t for j, t in enumerate(leaves)]
                    ends.append((act(p[0] @ p[1].t() + p[2], kind)[0] * dy.double()).sum())
                slope = float((ends[0] - ends[1]) / 2e-5)
                # z is kept in BF16: its rounding moves the slope by the second derivative (at most 1.2) times 2^-8 |z|; then the roundings of dz and of the result
                a, s = act(leaves[0] @ leaves[1].t() + leaves[2], kind)
                z = leaves[0] @ leaves[1].t() + leaves[2]
                e = dy.double().abs() * (2.0 ** -8 * s.abs() + (0.0 if kind == gws.ACT_NONE else 1.2 * 2.0 ** -8 * z.abs()))
                reach = (e @ leaves[1].abs() if i == 0 else e.t() @ leaves[0].abs() if i == 1 else e.sum(0)) + 2.0 ** -8 * grad.double().abs()
                assert abs(float((grad.double() * way).sum()) - slope) <= float((reach * way.abs()).sum()) * 1.01 + 1e-6


def test_another_stream_a_captured_step_and_steps_in_a_row():
    x, w, b, r, dy = problem(300, 768, 512)

    def step(stream=None):
        y, saved = gws.linear_fwd(x, w, b, residual=r, activation=gws.GATED_GELU_TANH, save=gws.ACT8_INT8, stream=stream)
        return (y, *gws.linear_bwd(dy, x, w, saved, gws.GATED_GELU_TANH, want_grad_bias=True, want_act=True, stream=stream))

    want = step()
    for _ in range(50):
        got = step()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    x.copy_(rand((300, 512), 9))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(out, step()))
    gws.check_waits()


def test_offsets_that_pass_32_bits():
    m, n, k, kind = (1 << 20) + 77, 2072, 2056, gws.GATED_GELU_TANH
    ends = torch.cat([torch.arange(200), torch.arange(m - 200, m)]).to(DEV)
    x = torch.empty(m, k, dtype=torch.bfloat16, device=DEV).normal_()
    w, b, dy = rand((n, k), 2, 1.5 / math.sqrt(k)), rand((n,), 5, 0.5, torch.float32), torch.zeros(m, n, dtype=torch.bfloat16, device=DEV)
    dy[ends] = rand((400, n), 4, 1e-2)
    y, saved = gws.linear_fwd(x, w, b, activation=kind, save=gws.ACT8_INT8)
    z, e = pre_activation(x[ends], w, b)
    a, _ = act(z, kind)
    assert within(y[ends], a, 2.0 ** -8 * a.abs() + 1.2 * e + 2.0 ** -18 * a.abs() + 1e-38)
    kept = gws.act8_load(saved)[ends].double()
    top = torch.nn.functional.pad(z.abs() + e, (0, -n % 32)).view(400, -1, 32).amax(-1)
    assert within(kept, z, (torch.exp2(torch.floor(torch.log2(top))) / 64).repeat_interleave(32, 1)[:, :n] + e)
    dx, dw, db, again = gws.linear_bwd(dy, x, w, saved, kind, want_grad_bias=True, want_act=True, bias_dtype=torch.float32)
    # rows without a gradient add nothing to the sums, and no rounding
    check_backward(dy[ends], x[ends].double(), w, None, kept, kind, (dx[ends], dw, db, again[ends]), torch.float32)
    assert not bool(dx[200:m - 200].any())


def test_refusals():
    x, w, b, r, dy = problem(8, 32, 24)
    y, saved = gws.linear_fwd(x, w, b, activation=gws.GATED_SILU, save=gws.ACT8_INT8)
    for call in (lambda: gws.linear_fwd(x.float(), w), lambda: gws.linear_fwd(x, w[:, :23]), lambda: gws.linear_fwd(x, w, b[:31]), lambda: gws.linear_fwd(x, w, b.half()),
                 lambda: gws.linear_fwd(x, w, b, residual=r[:7]), lambda: gws.linear_fwd(x, w, b, residual=r.float()), lambda: gws.linear_fwd(x, w.cpu(), b),
                 lambda: gws.linear_fwd(x, w, y=y.t()), lambda: gws.linear_bwd(dy, x, w, None, gws.GATED_SILU), lambda: gws.linear_bwd(dy, x, w, None, want_act=True),
                 lambda: gws.linear_bwd(dy[:7], x, w, saved, gws.GATED_SILU), lambda: gws.linear_bwd(dy, x[:, :23], w, saved, gws.GATED_SILU),
                 lambda: gws.linear_bwd(dy, x, w, gws.act8_save(x), gws.GATED_SILU), lambda: gws.linear_bwd(dy, x, w, dy.float(), gws.GATED_SILU),
                 lambda: gws.linear_bwd(dy, x, w, saved, gws.GATED_SILU, bias_dtype=torch.float16)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: gws.linear_fwd(x, w, b, activation=4), lambda: gws.linear_fwd(x, w, b, activation=-1), lambda: gws.linear_fwd(x, w, b, save=4),
                 lambda: gws.linear_fwd(x[:, :0], w[:, :0]), lambda: gws.linear_fwd(x, w, b, activation=7)):
        with pytest.raises(gws.GwsError):
            call()
