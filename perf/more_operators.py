"""Measured cases of the operators of a plain transformer block's training step: layer norm, linear layer with epilogue, AdamW.

Three operators, each with a plain form in 32-bit torch operations and, where ``own`` is true, the package's kernels:

* ``norm``    layer norm of s = x + residual over the rows: s (rounded to BF16, the residual stream) and y; with ``train`` the
              backward pass too: the gradient of x (and of the residual, which is the same), of the weight and of the bias
* ``linear``  y = act(x W^T + bias) + residual; with ``train`` x and z = x W^T + bias are kept as 8-bit checkpoints and the backward
              pass gives dx, dW, dbias and act(z) again, which the next layer's weight gradient needs
* ``adamw``   one step over all tensors of some blocks: parameters in BF16 with the low 16 bits of their 32-bit form in a tensor of their own,
              or in FP32; moments in 32 or in 8 bits

The 8-bit checkpoints of ``linear``: groups of 32 elements along a row with one power-of-two scale 2^(s - 127), s = max(E - emax, 0), E the
biased exponent of the group's largest magnitude.  "int8": codes c in [-127, 127], value c / 64 * scale, emax 0.  "e4m3": value
e4m3 * scale, clamped to +-448, emax 8.

State of ``adamw``: every tensor's elements start at a multiple of 256 of arrays that all tensors share.  FP32: m and v.  8 bits: groups of 256
elements.  m: codes E4M3, unit = max|m| * (1 / 448), value code * unit.  v is held as its root r: codes c = 16 e + f stand for
(1 + f / 16) 2^(e - 15), 0 for zero, unit = max r * (1 / 1.9375), and a root above zero has a code of at least 1.  A group whose maximum
is below 2^-100 has unit 0.  Codes are rounded to nearest even from value * (1 / unit), in FP32.  A BF16 parameter p and its rest l (int16) stand
for the 32-bit number whose bits are (bits of p) * 2^16 + l; p is the nearest BF16 number, the larger one of two as near.
"""
import math

import torch

own = False

GROUP = 32
BLOCK = 256
DEVICE = "cuda"
BETA1, BETA2, EPS, LR, STEP = 0.9, 0.95, 1e-8, 3e-4, 1000


def listed():
    return [
        # one decoded or streamed token of a 2048-wide model: residual stream and norm, nothing but latency
        dict(name="norm_one_token", op="norm", m=1, n=2048, pad=0, residual=True, weights="bf16", bias=True, train=False),
        # training on a ragged batch of an odd width, rows of a wider activation, no bias, 32-bit weights
        dict(name="norm_odd_train", op="norm", m=1531, n=1365, pad=11, residual=False, weights="f32", bias=False, train=True),
        # a micro-batch (8 x 2048 tokens) of a 2048-wide model
        dict(name="norm_train_16k", op="norm", m=16384, n=2048, pad=0, residual=True, weights="bf16", bias=True, train=True),
        # one token through an up projection: reading the weights once
        dict(name="linear_one_token", op="linear", m=1, k=2048, n=5632, act="gelu_tanh", residual=False, fmt="int8", train=False),
        # evaluation of a short ragged batch: a projection back onto the residual stream
        dict(name="linear_ragged_residual", op="linear", m=517, k=2730, n=768, act="none", residual=True, fmt="int8", train=False),
        # training step of a small layer on a handful of tokens: latency of the whole chain of calls
        dict(name="linear_train_33", op="linear", m=33, k=768, n=2048, act="gelu_tanh", residual=False, fmt="e4m3", train=True),
        # every size odd, all parts of the epilogue
        dict(name="linear_train_odd", op="linear", m=2047, k=1023, n=2729, act="silu", residual=True, fmt="int8", train=True),
        # up projection with GELU of a plain feed-forward block on a whole micro-batch
        dict(name="linear_train_16k", op="linear", m=16384, k=2048, n=5632, act="gelu_tanh", residual=False, fmt="int8", train=True),
        # the norms and biases of two blocks, or the bit-widths of a few layers: small FP32 tensors, latency
        dict(name="adamw_vectors", op="adamw", blocks=2, k=768, n=2048, matrices=False, param="f32", states="f32", tight=False),
        # odd widths, tensors one after the other in one buffer (no alignment), 8-bit moments
        dict(name="adamw_odd_8bit", op="adamw", blocks=3, k=1023, n=2729, matrices=True, param="bf16", states="8bit", tight=True),
        # eight blocks of a 2048-wide model, 32-bit moments
        dict(name="adamw_blocks_f32", op="adamw", blocks=8, k=2048, n=5632, matrices=True, param="bf16", states="f32", tight=False),
        # the same with moments in 8 bits
        dict(name="adamw_blocks_8bit", op="adamw", blocks=8, k=2048, n=5632, matrices=True, param="bf16", states="8bit", tight=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A layer width: a multiple of 8 three times out of four, any number otherwise."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.25 else max(8, w // 8 * 8)


def draw(rng):
    op = rng.choice(["norm", "linear", "adamw"])
    if op == "norm":
        n = _width(rng, 64, 8192)
        return dict(op=op, m=_log_int(rng, 1, min(16384, 2048 * 16384 // n)), n=n, pad=rng.choice([0, 0, 8, 13]), residual=rng.random() < 0.5,
                    weights=rng.choice(["bf16", "f32"]), bias=rng.random() < 0.75, train=rng.random() < 0.7)
    if op == "linear":
        return dict(op=op, m=_log_int(rng, 1, 16384), k=_width(rng, 256, 2048), n=_width(rng, 256, 5632),
                    act=rng.choice(["none", "silu", "gelu_tanh", "relu"]), residual=rng.random() < 0.5, fmt=rng.choice(["int8", "e4m3"]),
                    train=rng.random() < 0.6)
    return dict(op=op, blocks=rng.randint(1, 8), k=_width(rng, 64, 2048), n=_width(rng, 256, 5632), matrices=rng.random() < 0.8,
                param=rng.choice(["bf16", "bf16", "f32"]), states=rng.choice(["f32", "8bit"]), tight=rng.random() < 0.25)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _generator(seed, stream):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed * 16 + stream)
    return g


def _normal(seed, stream, shape, std, mean=0.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=_generator(seed, stream), device=DEVICE) * std + mean).to(dtype)


def _activation(seed, stream, rows, cols, pad=0):
    """Activations: unit variance, one channel in 256 eight times larger, every 61st token a padded one (zeros)."""
    g = _generator(seed, stream)
    x = torch.randn((rows, cols + pad), generator=g, device=DEVICE)
    channel = torch.rand((cols + pad,), generator=g, device=DEVICE)
    x *= torch.where(channel < 1 / 256, 8.0, 1.0)
    x[60::61] = 0
    return x.to(torch.bfloat16)[:, :cols]


def _shapes(case):
    """Tensors of the blocks: norm weight and bias, up projection and bias, down projection and bias."""
    k, n = case["k"], case["n"]
    block = [(k,), (k,), (n, k), (n,), (k, n), (k,)] if case["matrices"] else [(k,), (k,), (n,), (k,)]
    return block * case["blocks"]


def _round_up(v, to):
    return -(-v // to) * to


def prepare(case, seed):
    op = case["op"]
    state = dict(case)
    if op == "norm":
        m, n = case["m"], case["n"]
        weights = torch.bfloat16 if case["weights"] == "bf16" else torch.float32
        state["x"] = _activation(seed, 0, m, n, case["pad"])
        state["residual"] = _activation(seed, 1, m, n) if case["residual"] else None
        state["weight"] = _normal(seed, 2, (n,), 0.1, 1.0, weights)
        state["bias"] = _normal(seed, 3, (n,), 0.1, 0.0, weights) if case["bias"] else None
        if case["train"]:
            state["grad_y"] = _normal(seed, 4, (m, n), 1e-3)
            state["grad_s"] = _normal(seed, 5, (m, n), 1e-3) if case["residual"] else None
        return state
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        state["x"] = _activation(seed, 0, m, k)
        state["w"] = _normal(seed, 2, (n, k), 0.02)
        state["bias"] = _normal(seed, 3, (n,), 0.1)
        state["residual"] = _activation(seed, 1, m, n) if case["residual"] else None
        if case["train"]:
            state["grad_y"] = _normal(seed, 4, (m, n), 1e-3)
        return state
    shapes = _shapes(case)
    sizes = [math.prod(s) for s in shapes]
    starts, total = [], 0                               # of the tensors in the arrays of the state
    for s in sizes:
        starts.append(total)
        total += _round_up(s, BLOCK)
    places, length = (starts, total)                    # of the parameters and gradients in their buffers
    if case["tight"]:
        places, length = [sum(sizes[:i]) for i in range(len(sizes))], sum(sizes)
    dtype = torch.bfloat16 if case["param"] == "bf16" else torch.float32
    real = torch.zeros(total, dtype=torch.bool, device=DEVICE)
    decay = torch.zeros(total // BLOCK, device=DEVICE)  # decay for matrices, none for vectors
    for s, at, shape in zip(sizes, starts, shapes):
        real[at:at + s] = True
        decay[at // BLOCK:(at + s + BLOCK - 1) // BLOCK] = 0.1 if len(shape) > 1 else 0.0
    state["index"] = real.nonzero().squeeze(1) if case["tight"] else None
    state["decay"] = decay
    weights = (torch.randn(total, generator=_generator(seed, 0), device=DEVICE) * 0.02) * real
    grads = (torch.randn(total, generator=_generator(seed, 1), device=DEVICE) * 1e-3 * real).to(dtype)
    m = torch.randn(total, generator=_generator(seed, 2), device=DEVICE) * 3e-4 * real
    v = torch.rand(total, generator=_generator(seed, 3), device=DEVICE).square_().mul_(2e-6) * real
    if case["param"] == "bf16":
        p, rest = _split(weights)
        state["rest"] = rest
    else:
        p, state["rest"] = weights, None
    if case["states"] == "8bit":
        m_codes, m_unit = _encode_m(m.view(-1, BLOCK))
        r_codes, r_unit = _encode_r(torch.sqrt(v).view(-1, BLOCK))
        state["moments"] = torch.stack([m_codes.flatten(), r_codes.flatten()])
        state["units"] = torch.stack([m_unit, r_unit])
    else:
        state["moments"], state["units"] = torch.stack([m, v]), None
    if case["tight"]:
        p, grads = p[real], grads[real]
    assert p.numel() == length
    state["p"], state["g"] = p, grads
    state["params"] = [p[at:at + s].view(shape) for s, at, shape in zip(sizes, places, shapes)]
    state["grads"] = [grads[at:at + s].view(shape) for s, at, shape in zip(sizes, places, shapes)]
    state["decays"] = [0.1 if len(shape) > 1 else 0.0 for shape in shapes]
    state["clip"] = torch.full((1,), 0.75, device=DEVICE)       # the factor of a clipped gradient norm
    return state


# ---- plain form -----------------------------------------------------------------------------------------------------

def _quantize(x, fmt):
    """(element values, scale bytes) of 32-bit x: [rows, groups, 32] floats on the element grid, [rows, groups] integers."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % GROUP)).view(rows, -1, GROUP)
    top = x.abs().amax(-1)
    exponent = torch.frexp(top).exponent + 126                       # biased exponent of a normal number
    byte = torch.where(top > 0, (exponent - (8 if fmt == "e4m3" else 0)).clamp(min=0), 0)
    y = torch.ldexp(x, torch.where(top > 0, 127 - byte, 0).unsqueeze(-1))
    if fmt == "e4m3":
        return y.clamp(-448, 448).to(torch.float8_e4m3fn).to(y.dtype), byte
    return torch.round(y * 64).clamp(-127, 127) / 64, byte


def _restored(x, fmt):
    element, byte = _quantize(x, fmt)
    return torch.ldexp(element, (byte - 127).unsqueeze(-1)).flatten(1)[:, :x.shape[1]]


def _act(z, kind):
    """act(z) and its derivative."""
    if kind == "none":
        return z, torch.ones_like(z)
    if kind == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if kind == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def _plain_norm(s):
    b16 = torch.bfloat16
    total = s["x"]
    if s["residual"] is not None:
        total = (s["x"].float() + s["residual"].float()).to(b16)
    x, w = total.float(), s["weight"].float()
    centred = x - x.mean(1, keepdim=True)
    rstd = torch.rsqrt((centred * centred).mean(1, keepdim=True) + 1e-5)
    xh = centred * rstd
    y = xh * w
    if s["bias"] is not None:
        y = y + s["bias"].float()
    out = dict(y=y.to(b16))
    if s["residual"] is not None:
        out["sum"] = total
    if s["train"]:
        dy = s["grad_y"].float()
        a = dy * w
        dx = rstd * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
        if s["grad_s"] is not None:
            dx = dx + s["grad_s"].float()
        out["grad_x"] = dx.to(b16)
        out["grad_weight"] = (dy * xh).sum(0).to(s["weight"].dtype)
        if s["bias"] is not None:
            out["grad_bias"] = dy.sum(0).to(s["weight"].dtype)
    return out


def _plain_linear(s):
    b16 = torch.bfloat16
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.T + s["bias"].float()
    y = _act(z, s["act"])[0]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if not s["train"]:
        return y.to(b16)
    a, slope = _act(_restored(z, s["fmt"]), s["act"])
    dz = s["grad_y"].float() * slope
    return dict(y=y.to(b16), grad_x=(dz @ w).to(b16), grad_w=(dz.T @ _restored(x, s["fmt"])).to(b16), grad_bias=dz.sum(0).to(b16), act_again=a.to(b16))


def _split(weights):
    """(BF16, rest) of 32-bit numbers."""
    bits = weights.view(torch.int32)
    high = (bits + 0x8000) >> 16
    return high.to(torch.int16).view(torch.bfloat16), (bits - (high << 16)).to(torch.int16)


def _joined(p, rest):
    return ((p.view(torch.int16).to(torch.int32) << 16) + rest.to(torch.int32)).view(torch.float32)


def _unit(top, step):
    return torch.where(top >= 2.0 ** -100, top * step, 0.0)


def _encode_m(m):
    unit = _unit(m.abs().amax(1), 1 / 448)
    inverse = torch.where(unit > 0, torch.reciprocal(unit), 0.0)
    return (m * inverse.unsqueeze(1)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), unit


def _decode_m(codes, unit):
    return codes.view(torch.float8_e4m3fn).to(unit.dtype) * unit.unsqueeze(1)


def _encode_r(r):
    unit = _unit(r.amax(1), 1 / 1.9375)
    inverse = torch.where(unit > 0, torch.reciprocal(unit), 0.0)
    bits = (r * inverse.unsqueeze(1)).view(torch.int32)
    code = ((bits + 0x3FFFF + ((bits >> 19) & 1)) >> 19) - (112 << 4)
    return torch.where((r > 0) & (unit > 0).unsqueeze(1), code.clamp(1, 255), 0).to(torch.uint8), unit


def _decode_r(codes, unit):
    grid = ((codes.to(torch.int32) + (112 << 4)) << 19).view(torch.float32).to(unit.dtype)
    return torch.where(codes > 0, grid, 0.0) * unit.unsqueeze(1)


def _plain_adamw(s):
    index, states8 = s["index"], s["states"] == "8bit"
    total = s["moments"].shape[1]

    def spread(t):                                       # a buffer in the order of the state's arrays
        if index is None:
            return t.view(-1, BLOCK)
        return t.new_zeros(total).index_copy(0, index, t).view(-1, BLOCK)

    def packed(t):
        return t.flatten() if index is None else t.flatten()[index]

    bf16 = s["rest"] is not None
    p = _joined(spread(s["p"]), s["rest"].view(-1, BLOCK)) if bf16 else spread(s["p"])
    g = spread(s["g"]).float() * s["clip"]
    if states8:
        m = _decode_m(s["moments"][0].view(-1, BLOCK), s["units"][0])
        r = _decode_r(s["moments"][1].view(-1, BLOCK), s["units"][1])
        v = r * r
    else:
        m, v = s["moments"][0].view(-1, BLOCK), s["moments"][1].view(-1, BLOCK)
    keep = 1 - LR * s["decay"].double()
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * (1 - BETA2)) * g
    r = torch.sqrt(v)
    p = p * keep.float().unsqueeze(1) - (m * (LR / (1 - BETA1 ** STEP))) / (r * (1 / math.sqrt(1 - BETA2 ** STEP)) + EPS)
    if states8:
        m_codes, m_unit = _encode_m(m)
        r_codes, r_unit = _encode_r(r)
        s["moments"][0], s["moments"][1] = m_codes.flatten(), r_codes.flatten()
        s["units"][0], s["units"][1] = m_unit, r_unit
        r = _decode_r(r_codes, r_unit)
        out = dict(m=_decode_m(m_codes, m_unit).flatten(), v=(r * r).flatten())
    else:
        s["moments"][0], s["moments"][1] = m.flatten(), v.flatten()
        out = dict(m=s["moments"][0], v=s["moments"][1])
    if bf16:
        high, rest = _split(p)
        s["p"].copy_(packed(high))
        s["rest"].copy_(rest.flatten())
        out["rest"] = s["rest"]
    else:
        s["p"].copy_(packed(p))
    out["p"] = s["p"]
    return out


# ---- the package's kernels -----------------------------------------------------------------------------------------------

def _own_norm(s, gws):
    y, total, stats = gws.layernorm_fwd(s["x"], s["weight"], s["bias"], residual=s["residual"])
    out = dict(y=y)
    if s["residual"] is not None:
        out["sum"] = total
    if s["train"]:
        out["grad_x"], out["grad_weight"], grad_bias = gws.layernorm_bwd(s["grad_y"], total, s["weight"], stats, grad_sum=s["grad_s"],
                                                                       want_grad_bias=s["bias"] is not None)
        if s["bias"] is not None:
            out["grad_bias"] = grad_bias
    return out


def _own_linear(s, gws):
    act = {"none": gws.ACT_NONE, "silu": gws.GATED_SILU, "gelu_tanh": gws.GATED_GELU_TANH, "relu": gws.GATED_RELU}[s["act"]]
    if not s["train"]:
        return gws.linear_fwd(s["x"], s["w"], s["bias"], residual=s["residual"], activation=act)[0]
    fmt = {"int8": gws.ACT8_INT8, "e4m3": gws.ACT8_E4M3}[s["fmt"]]
    x8 = gws.act8_save(s["x"], fmt)
    y, saved = gws.linear_fwd(s["x"], s["w"], s["bias"], residual=s["residual"], activation=act, save=fmt)
    grad_x, grad_w, grad_bias, again = gws.linear_bwd(s["grad_y"], x8, s["w"], saved, act, want_grad_bias=True, want_act=True)
    return dict(y=y, grad_x=grad_x, grad_w=grad_w, grad_bias=grad_bias, act_again=again)


def _own_adamw(s, gws):
    fmt = gws.ADAMW_8BIT if s["states"] == "8bit" else gws.ADAMW_F32
    state = gws.AdamWState([p.numel() for p in s["params"]], fmt, moments=s["moments"], units=s["units"], rest=s["rest"])
    gws.adamw_step(s["params"], s["grads"], state, lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=s["decays"], step=STEP, grad_scale=s["clip"])
    m, v = state.values() if s["states"] == "8bit" else s["moments"]
    out = dict(m=m, v=v, p=s["p"])
    if s["rest"] is not None:
        out["rest"] = s["rest"]
    return out


def run(state):
    op = state["op"]
    if own:
        import paper_2505_11170_b200 as gws
        return (_own_norm if op == "norm" else _own_linear if op == "linear" else _own_adamw)(state, gws)
    return (_plain_norm if op == "norm" else _plain_linear if op == "linear" else _plain_adamw)(state)


# ---- least work and exact results ------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "norm":
        m, n = case["m"], case["n"]
        each = 2 + 2 * case["residual"] + case["train"] * (2 + case["residual"])      # x, y, both residuals; grad_y, grad_x, grad_s
        weights = (2 if case["weights"] == "bf16" else 4) * n * (1 + case["bias"]) * (1 + case["train"])
        return dict(bytes=2 * m * n * each + weights, flops=0)
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        moved = m * k + n * k + n + m * n * (1 + case["residual"])
        if case["train"]:                                                              # grad_y in; grad_x, grad_w, grad_bias and act(z) out
            moved += m * n + m * k + n * k + n + m * n
        return dict(bytes=2 * moved, flops=(6 if case["train"] else 2) * m * n * k)
    elements = sum(math.prod(s) for s in _shapes(case))
    weights = 10 if case["param"] == "bf16" else 12                                    # p and its rest in and out, g in
    moments = 16 if case["states"] == "f32" else 4 * (1 + 4 / BLOCK) + 8               # in and out; the values that 8-bit ones stand for out
    return dict(bytes=elements * (weights + moments), flops=0)


def _exact_restored(x, fmt):
    """The checkpoint's values in 64 bits, by the spacing of the element grid at each magnitude."""
    rows, cols = x.shape
    pad = -cols % GROUP
    x = torch.cat([x, x.new_zeros(rows, pad)], 1).reshape(rows, -1, GROUP)
    top = x.abs().max(-1, keepdim=True).values
    shared = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
    shared = torch.where(torch.exp2(shared) > top, shared - 1, shared)            # log2 of a value just under a power of two
    shared = torch.where(torch.exp2(shared + 1) <= top, shared + 1, shared)
    scale = torch.exp2((shared - (8 if fmt == "e4m3" else 0)).clamp(min=-127))
    if fmt == "int8":
        step, most = scale / 64, scale * 127 / 64
    else:
        most = 448 * scale
        own_exponent = (torch.frexp(x / scale).exponent - 1).clamp(min=-6)
        step = torch.exp2((own_exponent - 3).double()) * scale
    y = torch.minimum(torch.maximum(torch.round(x / step) * step, -most), most)
    return torch.where(top > 0, y, 0.0).reshape(rows, -1)[:, :cols]


def _exact_act(z, kind):
    if kind == "none":
        return z
    if kind == "silu":
        return z * torch.special.expit(z)
    if kind == "relu":
        return torch.where(z > 0, z, 0.0)
    return z * torch.special.expit(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))      # (1 + tanh u) / 2 = sigmoid(2 u)


def exact(case, seed):
    s = prepare(case, seed)
    wide = lambda name: s[name].double()
    if case["op"] == "norm":
        x = wide("x")
        if s["residual"] is not None:                                  # the stream is BF16: the norm is of the rounded sum (64-bit sums of BF16 are exact)
            x = (x + wide("residual")).float().to(torch.bfloat16).double()
        out = dict(y=None)
        if s["residual"] is not None:
            out["sum"] = x
        leaves = [x.detach().requires_grad_(), wide("weight").requires_grad_()] + ([wide("bias").requires_grad_()] if s["bias"] is not None else [])
        with torch.enable_grad():                                      # gradients by differentiation
            var, mean = torch.var_mean(leaves[0], 1, correction=0, keepdim=True)
            y = (leaves[0] - mean) / torch.sqrt(var + 1e-5) * leaves[1]
            if s["bias"] is not None:
                y = y + leaves[2]
            out["y"] = y.detach()
            if s["train"]:
                grads = torch.autograd.grad(y, leaves, wide("grad_y"))
                out["grad_x"] = grads[0] if s["grad_s"] is None else grads[0] + wide("grad_s")
                out["grad_weight"] = grads[1]
                if s["bias"] is not None:
                    out["grad_bias"] = grads[2]
        return out
    if case["op"] == "linear":
        x, w = wide("x"), wide("w")
        z = torch.addmm(wide("bias"), x, w.T)
        y = _exact_act(z, s["act"])
        if s["residual"] is not None:
            y = y + wide("residual")
        if not s["train"]:
            return y
        z, x = _exact_restored(z, s["fmt"]), _exact_restored(x, s["fmt"])
        with torch.enable_grad():                                      # the slope by differentiation
            leaf = z.requires_grad_()
            a = _exact_act(leaf, s["act"])
            dz, = torch.autograd.grad(a, leaf, wide("grad_y"))
        return dict(y=y, grad_x=dz @ w, grad_w=dz.T @ x, grad_bias=dz.sum(0), act_again=a.detach())
    total = s["moments"].shape[1]
    at = torch.arange(total, device=DEVICE) if s["index"] is None else s["index"]
    if s["units"] is not None:                                         # E4M3 values, and (1 + f / 16) 2^(e - 15), times their units
        unit = s["units"].double().repeat_interleave(BLOCK, 1)
        m = s["moments"][0].view(torch.float8_e4m3fn).double() * unit[0]
        code = s["moments"][1].long()
        v = (torch.where(code > 0, (1 + (code % 16).double() / 16) * torch.exp2((code // 16 - 15).double()), 0.0) * unit[1]) ** 2
    else:
        m, v = s["moments"].double()
    g = torch.zeros_like(m)
    g[at] = wide("g") * float(s["clip"])
    p = torch.zeros_like(m)
    p[at] = wide("p")
    if s["rest"] is not None:                                          # the rest counts units of the 32-bit number's last place
        low = s["rest"].double()
        inside = torch.frexp(p).exponent - 24
        step = torch.exp2(inside.double())
        # below a power of two the numbers are twice as dense
        p = p + torch.where((torch.frexp(p).mantissa.abs() == 0.5) & (low < 0), step / 2, step) * low * torch.where(p < 0, -1.0, 1.0)
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    root = torch.sqrt(v)
    decay = s["decay"].double().repeat_interleave(BLOCK)
    p = p - LR * decay * p - LR / (1 - BETA1 ** STEP) * m / (root / math.sqrt(1 - BETA2 ** STEP) + EPS)
    out = dict(m=m, v=v, p=p[at])
    if s["units"] is not None:                                         # which code a value next to a border gets is a matter of the 32-bit steps
        out["m"] = out["v"] = None
    if s["rest"] is not None:
        out["rest"] = None
    return out
