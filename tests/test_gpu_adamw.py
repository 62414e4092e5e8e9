"""AdamW over many tensors: bit for bit against the specified FP32 operations in numpy, and against the formula in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2505_11170_b200 as gws
import step_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
HYPER = dict(lr=3e-3, betas=(0.9, 0.95), eps=1e-8)
SIZES = [1, 7, 255, 256, 257, 4096, 4097, 12345, 768, 100003]


def bits(t):
    return t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


class Twin:
    """A set of tensors on the GPU and the same on the host, stepped by the specification."""

    def __init__(self, sizes, kinds, fmt, rest, seed=0, offset=0, std=0.02):
        rng = np.random.default_rng(seed)
        self.kinds, self.fmt = kinds, fmt
        self.state = gws.AdamWState(sizes, fmt, rest=rest)
        self.params, self.w, self.rest = [], [], []
        for n, kind in zip(sizes, kinds):
            w = (rng.standard_normal(n) * std).astype(np.float32)
            dtype = torch.bfloat16 if kind == "bf16" else torch.float32
            room = torch.zeros(n + offset, dtype=dtype, device=DEV)
            if kind == "bf16":
                w = (ref.round_bf16(w).astype(np.uint32) << 16).view(np.float32)
            room[offset:] = torch.from_numpy(w).to(DEV).to(dtype)
            self.params.append(room[offset:])
            self.w.append(w)
        self.offset, self.rng = offset, rng
        self.groups = [-(-n // 256) for n in sizes]
        self.m = [np.zeros(256 * k, np.float32) for k in self.groups]
        self.v = [np.zeros(256 * k, np.float32) for k in self.groups]
        self.r = [np.zeros(256 * k, np.float32) for k in self.groups]

    def grads(self, std=1e-3):
        out = []
        for p, kind in zip(self.params, self.kinds):
            g = torch.from_numpy((self.rng.standard_normal(p.numel()) * std * np.exp(self.rng.standard_normal(p.numel()))).astype(np.float32))
            g = g.to(DEV).to(p.dtype)
            room = torch.empty(p.numel() + self.offset, dtype=p.dtype, device=DEV)
            room[self.offset:] = g
            out.append(room[self.offset:])
        return out

    def step(self, grads, step, decays, scale=None, **over):
        hyper = {**HYPER, **over}
        for i, g in enumerate(grads):
            if g is None:
                continue
            n = len(self.w[i])
            pad = lambda t: np.concatenate([t, np.zeros(256 * self.groups[i] - n, np.float32)])
            gh = pad(g.float().cpu().numpy())
            p, m, v, r = ref.adamw32(pad(self.w[i]), gh, self.m[i], self.v[i], hyper["lr"], *hyper["betas"], hyper["eps"], decays[i], step, scale)
            if self.fmt == gws.ADAMW_8BIT:
                cm, um = ref.encode_m(m)
                cr, ur = ref.encode_r(r)
                self.check_codes(i, cm, um, cr, ur)
                m = ref.decode_m(cm, um).ravel()
                r = ref.decode_r(cr, ur).ravel()
                v = r * r
            self.m[i], self.v[i] = m, v
            p = p[:n].astype(np.float32)
            if self.kinds[i] == "bf16" and self.state.rest is None:
                p = (ref.round_bf16(p).astype(np.uint32) << 16).view(np.float32)
            self.w[i] = p

    def check_codes(self, i, cm, um, cr, ur):
        self.codes = getattr(self, "codes", {})
        self.codes[i] = (cm, um, cr, ur)

    def compare(self):
        st = self.state
        values = [t.cpu().numpy() for t in st.values()]
        for i, w in enumerate(self.w):
            n, at = len(w), st.starts[i]
            span = slice(at, at + 256 * self.groups[i])
            assert np.array_equal(values[0][span], self.m[i], equal_nan=True), "m of tensor %d" % i
            assert np.array_equal(values[1][span], self.v[i], equal_nan=True), "v of tensor %d" % i
            if self.kinds[i] == "f32":
                assert np.array_equal(self.params[i].cpu().numpy(), w, equal_nan=True)
            elif st.rest is None:
                assert np.array_equal(bits(self.params[i]), ref.round_bf16(w))
            else:
                high, low = ref.split(w)
                assert np.array_equal(bits(self.params[i]), high), "weight of tensor %d" % i
                assert np.array_equal(st.rest[at:at + n].cpu().numpy(), low), "rest of tensor %d" % i
                assert np.array_equal(st.weight(i, self.params[i]).cpu().numpy(), w)
                assert not bool(st.rest[at + n:at + 256 * self.groups[i]].any())
            if self.fmt == gws.ADAMW_8BIT and i in getattr(self, "codes", {}):
                cm, um, cr, ur = self.codes[i]
                got = st.moments[:, span].cpu().numpy()
                assert np.array_equal(got[1], cr.ravel())
                assert np.array_equal(got[0] & (0x7F | (got[0] << 1 != 0) * 0x80), cm.ravel() & (0x7F | (cm.ravel() << 1 != 0) * 0x80))      # up to the sign of zero
                units = st.units[:, at // 256:at // 256 + self.groups[i]].cpu().numpy()
                assert np.array_equal(units[0], um, equal_nan=True) and np.array_equal(units[1], ur, equal_nan=True)


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("fmt", [gws.ADAMW_F32, gws.ADAMW_8BIT])
def test_steps_are_the_specified_bits(fmt, rest, offset):
    kinds = ["bf16", "f32", "bf16", "bf16", "bf16", "bf16", "f32", "bf16", "f32", "bf16"]
    twin = Twin(SIZES, kinds, fmt, rest, seed=offset, offset=offset)
    decays = [0.1 if i % 2 else 0.0 for i in range(len(SIZES))]
    clip = torch.full((1,), 0.7, device=DEV)
    for step in range(1, 6):
        grads = twin.grads()
        if step == 2:
            grads[0] = grads[3] = grads[7] = None                  # left alone, state and all
        scale = 0.7 if step % 2 else None
        gws.adamw_step(twin.params, grads, twin.state, weight_decay=decays, step=step, grad_scale=clip if scale else None, **HYPER)
        twin.step(grads, step, decays, scale)
        twin.compare()


@pytest.mark.parametrize("fmt", [gws.ADAMW_F32, gws.ADAMW_8BIT])
def test_one_step_against_the_formula_in_64_bits(fmt):
    n = 5000
    twin = Twin([n], ["bf16"], fmt, True, seed=4)
    grads = twin.grads()
    gws.adamw_step(twin.params, grads, twin.state, weight_decay=0.1, step=1, **HYPER)
    zero = np.zeros(n)
    p, m, v = ref.adamw64(twin.w[0], grads[0].float().cpu().numpy(), zero, zero, HYPER["lr"], *HYPER["betas"], HYPER["eps"], 0.1, 1)
    got = twin.state.weight(0, twin.params[0]).cpu().numpy().astype(np.float64)
    # five roundings of the step (itself of the size of lr) and of its factors, two of the weight
    assert np.all(np.abs(got - p) <= ref.U32 * (3 * np.abs(twin.w[0]) + 12 * np.abs(p - twin.w[0]) + 1e-12))
    gm, gv = (t.cpu().numpy()[:n] for t in twin.state.values())
    if fmt == gws.ADAMW_F32:
        assert np.all(np.abs(gm - m) <= 3 * ref.U32 * np.abs(m)) and np.all(np.abs(gv - v) <= 5 * ref.U32 * v)
    else:
        pad = np.zeros(5120 - n)
        top_m = np.abs(np.concatenate([m, pad])).reshape(-1, 256).max(1).repeat(256)[:n]
        top_r = np.sqrt(np.concatenate([v, pad])).reshape(-1, 256).max(1).repeat(256)[:n]
        # half a step of E4M3 (2^-4 of the value, 2^-10 of the unit below 2^-6), and of four bits of mantissa; a root that would be zero is kept above it
        assert np.all(np.abs(gm - m) <= 1.0001 * np.maximum(2.0 ** -4 * np.abs(m), 2.0 ** -10 * top_m / 448))
        root = np.sqrt(v)
        assert np.all(np.abs(np.sqrt(gv) - root) <= 1.0001 * np.maximum(2.0 ** -5 * root, 2.0 ** -15 * 1.0625 * top_r / 1.9375))


@pytest.mark.parametrize("fmt", [gws.ADAMW_F32, gws.ADAMW_8BIT])
@pytest.mark.parametrize("eps", [1e-8, 1e-15, 0.0])
def test_zeros_and_sizes_far_apart(fmt, eps):
    """Lanes that leave the fast arithmetic (a zero, tiny or huge second moment, a small eps) beside ones that do not: the same bits."""
    n = 20000
    twin = Twin([n, n], ["bf16", "f32"], fmt, True, seed=11)
    for step in range(1, 4):
        grads = twin.grads()
        for g in grads:
            r = torch.rand(n, generator=torch.Generator().manual_seed(step)).to(DEV)
            g[r < 0.02] = 0.0
            g[(r > 0.02) & (r < 0.03)] *= 1e-12
            g[(r > 0.03) & (r < 0.04)] *= 1e17
            g[:2048] = 0.0
        if eps == 0.0:                                         # 0 / 0 only where nothing has moved yet: keep to what has a gradient
            grads = [torch.where(g == 0, torch.full_like(g, 1e-6), g) for g in grads]
        gws.adamw_step(twin.params, grads, twin.state, weight_decay=0.1, step=step, lr=1e-3, betas=(0.9, 0.95), eps=eps)
        twin.step(grads, step, [0.1, 0.1], lr=1e-3, eps=eps)
        twin.compare()


def test_many_tensors_take_several_launches():
    sizes = [5 + 37 * (i % 40) for i in range(900)]
    twin = Twin(sizes, ["bf16" if i % 3 else "f32" for i in range(900)], gws.ADAMW_8BIT, True, seed=2)
    before = gws.launch_count()
    grads = twin.grads()
    gws.adamw_step(twin.params, grads, twin.state, weight_decay=0.1, step=1, **HYPER)
    assert gws.launch_count() - before == 3
    twin.step(grads, 1, [0.1] * 900)
    twin.compare()


def test_step_and_rate_on_the_device_and_a_captured_step():
    mine, other = (Twin([300, 5000], ["bf16", "f32"], gws.ADAMW_8BIT, True, seed=8) for _ in range(2))
    step, lr = torch.ones(1, dtype=torch.int64, device=DEV), torch.full((1,), 1e-3, device=DEV)
    grads = mine.grads()
    gws.adamw_step(mine.params, grads, mine.state, lr=lr, betas=(0.9, 0.95), weight_decay=0.1, step=step)        # warm-up: step 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        gws.adamw_step(mine.params, grads, mine.state, lr=lr, betas=(0.9, 0.95), weight_decay=0.1, step=step)
    rates = [1e-3, 2e-3, 5e-4]
    for k, rate in enumerate(rates):
        if k:
            lr.fill_(rate)
            graph.replay()
        gws.adamw_step(other.params, grads, other.state, lr=float(np.float32(rate)), betas=(0.9, 0.95), weight_decay=float(np.float32(0.1)), step=k + 1)
    torch.cuda.synchronize()
    assert int(step) == 3
    for a, b in zip(mine.params + [mine.state.moments, mine.state.units, mine.state.rest], other.params + [other.state.moments, other.state.units, other.state.rest]):
        assert torch.equal(a, b)


def test_values_that_are_not_finite_stay_in_their_elements_and_groups():
    for fmt in (gws.ADAMW_F32, gws.ADAMW_8BIT):
        twin = Twin([1000, 600], ["bf16", "f32"], fmt, True, seed=3)
        grads = twin.grads()
        grads[0][300] = float("inf")
        grads[1][10] = float("nan")
        gws.adamw_step(twin.params, grads, twin.state, weight_decay=0.0, step=1, **HYPER)
        for p, at in zip(twin.params, (300, 10)):
            bad = torch.zeros_like(p, dtype=torch.bool)
            bad[at] = True
            assert bool(p[bad].isnan().all()) and bool(p[~bad].isfinite().all())
        m, v = twin.state.values()
        for i, at in enumerate((300, 10)):
            start = twin.state.starts[i]
            lo, hi = (at // 256 * 256, at // 256 * 256 + 256) if fmt == gws.ADAMW_8BIT else (at, at + 1)
            for t in (m, v):
                t = t[start:start + twin.state.sizes[i]]
                assert not bool(t[lo:hi].isfinite().any()) and bool(t[:lo].isfinite().all()) and bool(t[hi:].isfinite().all())


def test_small_and_zero_moments():
    """Groups without a gradient keep units of zero; gradients of 2^-110 are stored as zeros; a root above zero keeps a code above zero."""
    state = gws.AdamWState([768], gws.ADAMW_8BIT)
    p = torch.zeros(768, device=DEV)
    g = torch.zeros(768, device=DEV)
    g[256:512] = 2.0 ** -110
    g[512] = 1.0
    g[513:] = 1e-7
    gws.adamw_step([p], [g], state, lr=1e-3, betas=(0.9, 0.95), weight_decay=0.0, step=1)
    assert state.units[:, :1].abs().sum() == 0 and state.units[0, 1] == 0 and bool((state.units[:, 2] > 0).all())
    assert not bool(state.moments[:, :512].any()) and bool((state.moments[1, 512:] > 0).all())
    assert not bool(p[:256].any()) and bool((p[512:] < 0).all()) and bool(p.isfinite().all())
    m, v = state.values()
    assert bool((v[513:] > 0).all()) and not bool(m[513:].any())


def test_a_weight_moves_by_less_than_half_its_spacing_only_with_the_rest():
    p = torch.ones(300, dtype=torch.bfloat16, device=DEV)
    q = p.clone()
    g = torch.ones_like(p)
    plain, keeps = gws.AdamWState([300]), gws.AdamWState([300], rest=True)
    for step in range(1, 11):
        gws.adamw_step([p], [g], plain, lr=1e-4, weight_decay=0.0, step=step)
        gws.adamw_step([q], [g], keeps, lr=1e-4, weight_decay=0.0, step=step)
    assert bool((p == 1).all()) and bool((keeps.weight(0, q) < 1 - 9e-4).all()) and bool((q == 1).all())


def test_parameters_set_to_zero_from_outside():
    p = torch.randn(1000, device=DEV).to(torch.bfloat16)
    state = gws.AdamWState([1000], rest=True)
    g = torch.full_like(p, 1e-3)
    for step in (1, 2):
        gws.adamw_step([p], [g], state, lr=1e-3, weight_decay=0.0, step=step)
    assert bool((state.rest < 0).any())
    rest = state.rest[:1000].clone()
    p[::3] = 0
    weight = state.weight(0, p)
    want = torch.where((p == 0) & (rest < 0), 0.0, weight)
    gws.adamw_step([p], [g], state, lr=1e-3, weight_decay=0.0, step=3)
    after = state.weight(0, p)
    assert bool(p.isfinite().all()) and bool(((want - after) - 1e-3).abs().max() < 1e-4)          # each moved by lr


def test_version_counters_see_the_step():
    p = torch.nn.Parameter(torch.ones(300, dtype=torch.bfloat16, device=DEV))
    loss = (p * p).sum()
    gws.adamw_step([p], [torch.ones_like(p)], gws.AdamWState([300]), lr=1e-2, step=1)
    with pytest.raises(RuntimeError):
        loss.backward()


def test_another_stream():
    twins = [Twin([3000], ["bf16"], gws.ADAMW_F32, True, seed=1) for _ in range(2)]
    grads = twins[0].grads()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    gws.adamw_step(twins[0].params, grads, twins[0].state, lr=1e-3, step=3, stream=side)
    gws.adamw_step(twins[1].params, grads, twins[1].state, lr=1e-3, step=3)
    torch.cuda.synchronize()
    assert torch.equal(twins[0].params[0], twins[1].params[0]) and torch.equal(twins[0].state.moments, twins[1].state.moments)


def test_gradients_of_any_strides_and_shapes():
    p, q = torch.ones(40, 30, device=DEV), torch.ones(40, 30, device=DEV)
    g = torch.randn(30, 40, device=DEV).t()
    a, b = gws.AdamWState([1200]), gws.AdamWState([1200])
    gws.adamw_step([p], [g], a, lr=1e-3, step=1)
    gws.adamw_step([q], [g.contiguous()], b, lr=1e-3, step=1)
    assert torch.equal(p, q) and torch.equal(a.moments, b.moments)
    empty = gws.AdamWState([0, 5])
    gws.adamw_step([torch.empty(0, device=DEV), torch.ones(5, device=DEV)], [torch.empty(0, device=DEV), None], empty, lr=1e-3)
    gws.adamw_step([], [], gws.AdamWState([]), lr=1e-3)


def test_offsets_that_pass_32_bits():
    big, few = (1 << 31) + 300, 1000
    p, g = (torch.empty(big, dtype=torch.bfloat16, device=DEV).normal_(0, std) for std in (0.02, 1e-3))
    q, h = (torch.empty(few, dtype=torch.bfloat16, device=DEV).normal_(0, std) for std in (0.02, 1e-3))
    whole, ends = gws.AdamWState([big, few], gws.ADAMW_8BIT, rest=True), gws.AdamWState([300, few], gws.ADAMW_8BIT, rest=True)
    p_ends, g_ends = [p[1 << 31:].clone(), q.clone()], [g[1 << 31:].clone(), h]
    for step in (1, 2):
        gws.adamw_step([p, q], [g, h], whole, step=step, **HYPER)
        gws.adamw_step(p_ends, g_ends, ends, step=step, **HYPER)
    assert torch.equal(p[1 << 31:], p_ends[0]) and torch.equal(q, p_ends[1])
    assert torch.equal(whole.moments[:, 1 << 31:], ends.moments) and torch.equal(whole.units[:, 1 << 23:], ends.units) and torch.equal(whole.rest[1 << 31:], ends.rest)
    assert bool(whole.rest[(1 << 31) - 256:1 << 31].any()) and not bool((p[(1 << 31) - 256:1 << 31] == 0).all())


def test_refusals():
    p, g = torch.ones(300, device=DEV), torch.ones(300, device=DEV)
    st = gws.AdamWState([300])
    wrong = [lambda: gws.adamw_step([p], [g, g], st, lr=1e-3), lambda: gws.adamw_step([p[:299]], [g[:299]], st, lr=1e-3),
             lambda: gws.adamw_step([p], [g.bfloat16()], st, lr=1e-3), lambda: gws.adamw_step([p.half()], [g.half()], st, lr=1e-3),
             lambda: gws.adamw_step([p.cpu()], [g], st, lr=1e-3), lambda: gws.adamw_step([torch.ones(600, device=DEV)[::2]], [g], st, lr=1e-3),
             lambda: gws.adamw_step([p], [g], st, lr=1e-3, weight_decay=[0.1, 0.1]), lambda: gws.adamw_step([p], [g], st, lr=1e-3, grad_scale=0.5),
             lambda: gws.adamw_step([p], [g], st, lr=torch.ones(1), step=1), lambda: gws.adamw_step([p], [g], st, lr=1e-3, step=torch.ones(1, device=DEV)),
             lambda: gws.AdamWState([300], 2), lambda: gws.AdamWState([300], moments=torch.zeros(2, 300, device=DEV)),
             lambda: gws.AdamWState([300], gws.ADAMW_8BIT, moments=torch.zeros(2, 512, dtype=torch.uint8, device=DEV)),
             lambda: gws.AdamWState([300], units=torch.zeros(2, 2, device=DEV)), lambda: gws.AdamWState([300], rest=torch.zeros(300, dtype=torch.int16, device=DEV)),
             lambda: gws.AdamWState([-1])]
    for call in wrong:
        with pytest.raises(ValueError):
            call()
    two = gws.AdamWState([300, 300])
    before = p.clone()
    for call in (lambda: gws.adamw_step([p], [g], st, lr=1e-3, step=0), lambda: gws.adamw_step([p, p], [g, g], two, lr=1e-3),
                 lambda: gws.adamw_step([p], [p], st, lr=1e-3), lambda: gws.adamw_step([p], [g], st, lr=1e-3, betas=(1.0, 0.9)),
                 lambda: gws.adamw_step([p], [g], st, lr=1e-3, eps=-1.0)):
        with pytest.raises(gws.GwsError):
            call()
    assert torch.equal(p, before)
