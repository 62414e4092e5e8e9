"""Layer norm, forward and backward, against plain forms in 64 bits."""
import pytest
import torch

import paper_2505_11170_b200 as gws
import step_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
# one row to many, every kind of team and its border, odd and even widths, rows longer than a block holds
SHAPES = [(1, 1), (1, 8), (3, 7), (1, 2048), (5, 256), (9, 257), (700, 512), (301, 513), (67, 1024), (400, 1365), (300, 2048), (2, 2049), (65, 2730), (33, 4096), (12, 5632),
          (7, 8192), (3, 8193), (5, 16384), (2, 16391), (1, 33000), (2048, 64), (1000, 776)]


def rand(shape, seed, std=1.0, mean=0.0, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype).to(DEV)


def weights(n, kind):
    if kind == "none":
        return None, None
    dtype = torch.float32 if "f32" in kind else torch.bfloat16
    return rand((n,), 5, 0.3, 1.0, dtype), rand((n,), 6, 0.3, 0.0, dtype) if "bias" in kind else None


def within(got, want, bound):
    return bool(((got.double() - want).abs() <= bound).all())


def check_forward(x, w, b, residual=None, eps=1e-5):
    y, s, stats = gws.layernorm_fwd(x, w, b, eps, residual=residual)
    if residual is None:
        assert s.data_ptr() == x.data_ptr()
    else:
        assert torch.equal(s, (x.float() + residual.float()).to(torch.bfloat16))
    want, _, mean, rstd = ref.norm(s, w, b, eps)
    assert within(y, want, ref.norm_forward_bound(s, w, b, eps) + 1e-38)
    e_mean, e_rstd, _ = ref.norm_errors(s, eps)
    assert within(stats[0], mean[:, 0], e_mean[:, 0] + 1e-40) and within(stats[1], rstd[:, 0], (e_rstd * rstd)[:, 0])
    again = gws.layernorm_fwd(x, w, b, eps, residual=residual, want_stats=False)
    assert torch.equal(again[0], y) and again[2] is None
    return y, s, stats


def check_backward(dy, s, w, stats, b=True, grad_sum=None, eps=1e-5):
    dx, dw, db = gws.layernorm_bwd(dy, s, w, stats, grad_sum=grad_sum, want_grad_bias=b)
    (want_x, want_w, want_b), (e_x, e_w, e_b) = ref.norm_backward(dy, s, w, eps, grad_sum)
    assert within(dx, want_x, e_x + 1e-38)
    assert (dw is None) == (w is None) and (db is None) == (w is None or not b)
    for got, want, err in ((dw, want_w, e_w), (db, want_b, e_b)):
        if got is not None:
            assert got.dtype == w.dtype
            half = ref.U32 if got.dtype == torch.float32 else ref.U16
            assert within(got, want, err + half * (want.abs() + err) + 1e-38)
    return dx, dw, db


@pytest.mark.parametrize("kind", ["bf16 bias", "f32", "none"])
@pytest.mark.parametrize("m,n", SHAPES)
def test_forward_and_backward(m, n, kind):
    x, dy = rand((m, n), 1, 1.5, 0.5), rand((m, n), 2, 1e-2)
    w, b = weights(n, kind)
    _, s, stats = check_forward(x, w, b)
    first = check_backward(dy, s, w, stats, b is not None)
    again = gws.layernorm_bwd(dy, s, w, stats, want_grad_bias=b is not None)
    for p, q in zip(first, again):
        assert (p is None and q is None) or torch.equal(p, q)          # nothing depends on timing


@pytest.mark.parametrize("m,n", [(1, 2048), (5, 33), (300, 768), (290, 1365), (40, 4096), (3, 8200), (1100, 2048)])
def test_residual_stream(m, n):
    x, r, dy, d = rand((m, n), 1), rand((m, n), 2, 2.0), rand((m, n), 3, 1e-2), rand((m, n), 4, 1e-2)
    w, b = weights(n, "f32 bias")
    _, s, stats = check_forward(x, w, b, r)
    check_backward(dy, s, w, stats, True, d)


# more rows than the teams of all blocks hold at once, for every kind of team
@pytest.mark.parametrize("m,n", [(5001, 256), (5003, 255), (3001, 768), (3000, 769), (3001, 1360), (2500, 1365), (1501, 3000), (1500, 3001), (1001, 4096), (1000, 4095), (701, 6000), (700, 6001),
                                 (501, 8192), (500, 8191)])
def test_rows_in_turn(m, n):
    x, r, dy, d = rand((m, n), 1), rand((m, n), 2, 2.0), rand((m, n), 3, 1e-2), rand((m, n), 4, 1e-2)
    w, b = weights(n, "f32 bias")
    _, s, stats = check_forward(x, w, b, r)
    first = check_backward(dy, s, w, stats, True, d)
    again = gws.layernorm_bwd(dy, s, w, stats, grad_sum=d)
    assert all(torch.equal(p, q) for p, q in zip(first, again))


@pytest.mark.parametrize("n", [96, 1365, 2048, 9000])
def test_strides_and_alignments(n):
    m = 37
    wide = rand((m, n + 11), 1)
    for x in (wide[:, :n], wide[:, 3:3 + n], wide[::2, 1:1 + n], rand((n, m), 2).t(), wide[:1, 5:5 + n].expand(m, n)):
        rows = x.shape[0]
        buffer = rand((rows * n + 1,), 3)
        r, dy, d = buffer[1:].view(rows, n), wide[:rows, 7:7 + n], wide.flip(0)[:rows, :n]
        w = rand((n + 1,), 4)[1:]
        _, s, stats = check_forward(x, w, None, r)
        check_backward(dy, s, w, stats, False, d)
        y, s2, stats2 = gws.layernorm_fwd(x.contiguous(), w.clone(), None, residual=r.contiguous())
        assert torch.equal(s2, s)


def test_rows_of_large_mean_constant_rows_and_values_that_are_not_finite():
    x = rand((6, 1000), 1)
    x[0] += 300.0
    x[1] = 2.5                         # no variance: eps decides
    x[2] = 0.0
    x[3, 17] = float("inf")
    x[4, 3] = float("nan")
    w, b = weights(1000, "bf16 bias")
    y, s, stats = gws.layernorm_fwd(x, w, b)
    fine = torch.tensor([0, 1, 2, 5], device=DEV)
    want, _, _, _ = ref.norm(x[fine], w, b, 1e-5)
    assert within(y[fine], want, ref.norm_forward_bound(x[fine], w, b, 1e-5))
    assert torch.equal(y[2], b) and bool(y[3:5].isnan().all())
    dy = rand((6, 1000), 2, 1e-2)
    dx, dw, db = gws.layernorm_bwd(dy, s, w, stats)
    (want_x, _, want_b), (e_x, _, e_b) = ref.norm_backward(dy[fine], x[fine], w, 1e-5)
    assert within(dx[fine], want_x, e_x) and bool(dx[3:5].isnan().all())
    assert bool(dw.isnan().all())                                        # a row that is not finite reaches every column of dgamma, none of dbeta
    assert bool(db.isfinite().all())


def test_no_rows_and_no_columns():
    w, b = weights(64, "f32 bias")
    y, s, stats = gws.layernorm_fwd(rand((0, 64), 1), w, b)
    assert y.shape == (0, 64) and stats.shape == (2, 0)
    dx, dw, db = gws.layernorm_bwd(rand((0, 64), 1), s, w, stats)
    assert dx.shape == (0, 64) and not bool(dw.any()) and not bool(db.any())
    y, s, stats = gws.layernorm_fwd(rand((3, 0), 1))
    assert y.shape == (3, 0)
    assert gws.layernorm_bwd(rand((3, 0), 1), s, None, stats)[0].shape == (3, 0)


def test_what_is_not_wanted():
    x, dy = rand((50, 300), 1), rand((50, 300), 2)
    w, b = weights(300, "bf16 bias")
    _, s, stats = gws.layernorm_fwd(x, w, b)
    full = gws.layernorm_bwd(dy, s, w, stats)
    only_x = gws.layernorm_bwd(dy, s, w, stats, want_grad_weight=False, want_grad_bias=False)
    only_w = gws.layernorm_bwd(dy, s, w, stats, want_grad_x=False, want_grad_bias=False)
    assert only_x[1] is None and only_x[2] is None and torch.equal(only_x[0], full[0])
    assert only_w[0] is None and only_w[2] is None and torch.equal(only_w[1], full[1])
    assert gws.layernorm_bwd(dy, s, w, stats, want_grad_x=False, want_grad_weight=False, want_grad_bias=False) == (None, None, None)
    long = rand((4, 9001), 3)
    wl, _ = weights(9001, "bf16")
    _, s, stats = gws.layernorm_fwd(long, wl)
    full = gws.layernorm_bwd(long, s, wl, stats)
    assert torch.equal(gws.layernorm_bwd(long, s, wl, stats, want_grad_x=False)[1], full[1])


def test_gradients_against_differences_of_the_forward_pass():
    m, n, eps = 6, 40, 1e-5
    x, dy, w, b = rand((m, n), 1), rand((m, n), 2), rand((n,), 3, 0.3, 1.0, torch.float32), rand((n,), 4, 0.3, 0.0, torch.float32)
    _, s, stats = gws.layernorm_fwd(x, w, b, eps)
    grads = gws.layernorm_bwd(dy, s, w, stats)
    leaves = [t.double() for t in (x, w, b)]
    for i, grad in enumerate(grads):
        for seed in range(4):
            g = torch.Generator().manual_seed(seed)
            way = torch.randn(leaves[i].shape, generator=g, dtype=torch.float64).to(DEV)
            h = 1e-5
            ends = []
            for sign in (1, -1):
                moved = [t + sign * h * way if k == i else t for k, t in enumerate(leaves)]
                ends.append((ref.norm(moved[0], moved[1], moved[2], eps)[0] * dy.double()).sum())
            slope = float((ends[0] - ends[1]) / (2 * h))
            got = float((grad.double() * way).sum())
            # each entry of dx is off by at most 2^-8 of itself, of the sums by FP32 rounding; h^2 times the third derivative is below 1e-6 here
            assert abs(got - slope) <= float((grad.double().abs() * way.abs()).sum()) * (ref.U16 + 1e-5) + 1e-4


def test_another_stream_and_a_captured_pass():
    x, r, dy = rand((500, 768), 1), rand((500, 768), 2), rand((500, 768), 3)
    w, b = weights(768, "bf16 bias")

    def both(stream=None):
        y, s, stats = gws.layernorm_fwd(x, w, b, residual=r, stream=stream)
        return (y, s, *gws.layernorm_bwd(dy, s, w, stats, grad_sum=dy, stream=stream))

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    x.copy_(rand((500, 768), 9))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(out, both()))


def test_offsets_that_pass_32_bits():
    m, n = (1 << 20) + 77, 2056
    ends = torch.cat([torch.arange(200), torch.arange(m - 200, m)]).to(DEV)
    x, r, dy = (torch.empty(m, n, dtype=torch.bfloat16, device=DEV).normal_() for _ in range(3))
    w, b = weights(n, "f32 bias")
    y, s, stats = gws.layernorm_fwd(x, w, b, residual=r)
    for got, want in zip((y, s), check_forward(x[ends], w, b, r[ends])):
        assert torch.equal(got[ends], want)
    dy[200:m - 200] = 0
    dx, dw, db = gws.layernorm_bwd(dy, s, w, stats)
    alone = check_backward(dy[ends], s[ends], w, stats[:, ends].contiguous())
    assert torch.equal(dx[ends], alone[0]) and not bool(dx[200:m - 200].any())
    (_, want_w, want_b), (_, e_w, e_b) = ref.norm_backward(dy[ends], s[ends], w, 1e-5)          # rows without a gradient add nothing, and no rounding
    assert within(dw, want_w, e_w + ref.U32 * (want_w.abs() + e_w)) and within(db, want_b, e_b + ref.U32 * (want_b.abs() + e_b))


def test_refusals():
    x = rand((4, 64), 1)
    w, b = weights(64, "bf16 bias")
    y, s, stats = gws.layernorm_fwd(x, w, b)
    for call in (lambda: gws.layernorm_fwd(x.float(), w), lambda: gws.layernorm_fwd(x[0], w), lambda: gws.layernorm_fwd(x, w[:63]), lambda: gws.layernorm_fwd(x, None, b),
                 lambda: gws.layernorm_fwd(x, w, b.float()), lambda: gws.layernorm_fwd(x, w.half()), lambda: gws.layernorm_fwd(x, w, residual=x[:3]),
                 lambda: gws.layernorm_fwd(x, w.cpu()), lambda: gws.layernorm_bwd(x[:, :63], s, w, stats), lambda: gws.layernorm_bwd(x, s, w, stats[0]),
                 lambda: gws.layernorm_bwd(x, s, w, stats.double()), lambda: gws.layernorm_bwd(x, s, w, stats, grad_sum=x[:2])):
        with pytest.raises(ValueError):
            call()
