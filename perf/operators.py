"""Measured cases of the activation operators: 8-bit activation checkpoints and the gated feed-forward block.

Four operators, each with a plain form in 32-bit torch operations and, where ``own`` is true, the package's kernels:

* ``act8``         an activation written as an 8-bit checkpoint in the forward pass and read back for the backward pass
* ``wgrad_act8``   the weight gradient of a linear layer, dW = dY^T X, with X held as such a checkpoint
* ``gated``        forward pass of the gated feed-forward block, h = act(x Wg^T) * (x Wu^T)
* ``gated_train``  its forward pass with x, the gate and the up projection kept as 8-bit checkpoints, then its backward
                   pass: dx, dWg, dWu and the h that the next layer's weight gradient needs

A checkpoint holds groups of 32 elements along a row with one power-of-two scale 2^(s - 127), s = max(E - emax, 0) with E the
biased exponent of the group's largest magnitude.  "int8": codes c in [-127, 127], value c / 64 * scale, emax 0.  "e4m3":
value e4m3 * scale, clamped to +-448, emax 8.  Rounding is to nearest even.  The buffer is rows x ld codes (ld: cols rounded
up to 32, the rest zero), then from the next multiple of 256 bytes rows x ld / 32 scale bytes.
"""
import math

import torch

own = False

GROUP = 32
DEVICE = "cuda"


def listed():
    return [
        # one decoded or streamed token of a 2048-wide model: nothing but the latency of the two calls
        dict(name="act8_one_token", op="act8", m=1, k=2048, pad=0, fmt="int8"),
        # a slice of a wider activation with an odd width (8/3 * 512 = 1365): strided rows, ragged last group
        dict(name="act8_odd_strided", op="act8", m=1531, k=1365, pad=11, fmt="e4m3"),
        # the hidden activation of one micro-batch (8 x 2048 tokens) of the 1B-parameter Llama-style model
        dict(name="act8_hidden_16k", op="act8", m=16384, k=5632, pad=0, fmt="int8"),
        # attention projection of the 124M-parameter GPT-2 model on a short ragged batch
        dict(name="wgrad_gpt2_proj", op="wgrad_act8", m=515, n=768, k=768, fmt="int8"),
        # odd widths throughout, wide-range codes
        dict(name="wgrad_odd_e4m3", op="wgrad_act8", m=3001, n=1023, k=2730, fmt="e4m3"),
        # down projection of the Llama-style model, whole micro-batch, its 5632-wide input kept in 8 bits
        dict(name="wgrad_llama_down", op="wgrad_act8", m=16384, n=2048, k=5632, fmt="int8"),
        # one token through the Llama-style block: reading the two weights once
        dict(name="gated_one_token", op="gated", m=1, k=2048, n=5632, act="silu"),
        # evaluation of a short ragged batch with a GELU gate and an even, 16-byte-unfriendly width
        dict(name="gated_ragged_gelu", op="gated", m=517, k=768, n=2730, act="gelu_tanh"),
        # evaluation of a whole micro-batch of the Llama-style model
        dict(name="gated_llama_16k", op="gated", m=16384, k=2048, n=5632, act="silu"),
        # training step of a small block on a handful of tokens: latency of the whole chain of calls
        dict(name="train_33_tokens", op="gated_train", m=33, k=768, n=2048, act="silu", fmt="e4m3"),
        # training step with every size odd
        dict(name="train_odd_gelu", op="gated_train", m=2047, k=1023, n=2729, act="gelu_tanh", fmt="int8"),
        # training step of the Llama-style block on a whole micro-batch
        dict(name="train_llama_16k", op="gated_train", m=16384, k=2048, n=5632, act="silu", fmt="int8"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A layer width: a multiple of 8 three times out of four, any number otherwise."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.25 else max(8, w // 8 * 8)


def draw(rng):
    op = rng.choice(["act8", "wgrad_act8", "gated", "gated_train"])
    m = _log_int(rng, 1, 16384)
    fmt = rng.choice(["int8", "e4m3"])
    act = rng.choice(["silu", "gelu_tanh", "relu"])
    if op == "act8":
        return dict(op=op, m=m, k=_width(rng, 64, 5632), pad=rng.choice([0, 0, 8, 13]), fmt=fmt)
    if op == "wgrad_act8":
        return dict(op=op, m=m, n=_width(rng, 256, 5632), k=_width(rng, 256, 2048), fmt=fmt)
    if op == "gated":
        return dict(op=op, m=m, k=_width(rng, 256, 2048), n=_width(rng, 512, 5632), act=act)
    return dict(op=op, m=m, k=_width(rng, 256, 2048), n=_width(rng, 512, 5632), act=act, fmt=fmt)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _generator(seed, stream):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed * 16 + stream)
    return g


def _normal(seed, stream, rows, cols, std):
    return (torch.randn((rows, cols), generator=_generator(seed, stream), device=DEVICE) * std).to(torch.bfloat16)


def _activation(seed, stream, rows, cols, pad=0):
    """Normed activations: unit variance, one channel in 256 eight times larger, every 61st token a padded one (zeros)."""
    g = _generator(seed, stream)
    x = torch.randn((rows, cols + pad), generator=g, device=DEVICE)
    channel = torch.rand((cols + pad,), generator=g, device=DEVICE)
    x *= torch.where(channel < 1 / 256, 8.0, 1.0)
    x[60::61] = 0
    return x.to(torch.bfloat16)[:, :cols]


def prepare(case, seed):
    op, m, k = case["op"], case["m"], case["k"]
    state = dict(case)
    if op == "act8":
        state["x"] = _activation(seed, 0, m, k, case["pad"])
    elif op == "wgrad_act8":
        state["grad_y"] = _normal(seed, 1, m, case["n"], 1e-3)
        state["x8"] = _pack(*_quantize(_activation(seed, 0, m, k).float(), case["fmt"]), case["fmt"])
    else:
        n = case["n"]
        state["x"] = _activation(seed, 0, m, k)
        state["w_gate"] = _normal(seed, 2, n, k, 0.02)
        state["w_up"] = _normal(seed, 3, n, k, 0.02)
        if op == "gated_train":
            state["grad_h"] = _normal(seed, 4, m, n, 1e-3)
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


def _values(element, byte, cols):
    return torch.ldexp(element, (byte - 127).unsqueeze(-1)).flatten(1)[:, :cols]


def _restored(x, fmt):
    return _values(*_quantize(x, fmt), x.shape[1])


def _pack(element, byte, fmt):
    """One buffer in the layout of a checkpoint."""
    if fmt == "e4m3":
        codes = element.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        codes = (element * 64).to(torch.int8).view(torch.uint8)
    codes = codes.flatten()
    buffer = torch.zeros(-(-codes.numel() // 256) * 256 + byte.numel(), dtype=torch.uint8, device=codes.device)
    buffer[:codes.numel()] = codes
    buffer[buffer.numel() - byte.numel():] = byte.flatten().to(torch.uint8)
    return buffer


def _unpack(buffer, rows, cols, fmt, dtype):
    groups = -(-cols // GROUP)
    codes = buffer[:rows * groups * GROUP].view(rows, groups, GROUP)
    byte = buffer[buffer.numel() - rows * groups:].view(rows, groups).to(torch.int32)
    if fmt == "e4m3":
        element = codes.view(torch.float8_e4m3fn).to(dtype)
    else:
        element = codes.view(torch.int8).to(dtype) / 64
    return _values(element, byte, cols)


def _act(g, kind):
    """act(g) and its derivative."""
    if kind == "relu":
        return g.clamp(min=0), (g > 0).to(g.dtype)
    if kind == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _run_plain(s):
    op = s["op"]
    b16 = torch.bfloat16
    if op == "act8":
        return _restored(s["x"].float(), s["fmt"]).to(b16)
    if op == "wgrad_act8":
        x = _unpack(s["x8"], s["m"], s["k"], s["fmt"], torch.float32)
        return (s["grad_y"].float().T @ x).to(b16)
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    gate, up = x @ wg.T, x @ wu.T
    h = (_act(gate, s["act"])[0] * up).to(b16)
    if op == "gated":
        return h
    gate, up, x = (_restored(t, s["fmt"]) for t in (gate, up, x))
    a, slope = _act(gate, s["act"])
    grad_h = s["grad_h"].float()
    grad_gate, grad_up = grad_h * up * slope, grad_h * a
    return dict(h=h, grad_x=(grad_gate @ wg + grad_up @ wu).to(b16), grad_w_gate=(grad_gate.T @ x).to(b16), grad_w_up=(grad_up.T @ x).to(b16),
                h_again=(a * up).to(b16))


# ---- the package's kernels -----------------------------------------------------------------------------------------------

def _run_own(s):
    import paper_2505_11170_b200 as gws

    op = s["op"]
    if op != "gated":
        fmt = {"int8": gws.ACT8_INT8, "e4m3": gws.ACT8_E4M3}[s["fmt"]]
    if op == "act8":
        return gws.act8_load(gws.act8_save(s["x"], fmt))
    if op == "wgrad_act8":
        return gws.wgrad_act8(s["grad_y"], gws.Act8(s["x8"], s["m"], s["k"], fmt))
    act = {"silu": gws.GATED_SILU, "gelu_tanh": gws.GATED_GELU_TANH, "relu": gws.GATED_RELU}[s["act"]]
    if op == "gated":
        return gws.gated_fwd(s["x"], s["w_gate"], s["w_up"], act)[0]
    x8 = gws.act8_save(s["x"], fmt)
    h, saved = gws.gated_fwd(s["x"], s["w_gate"], s["w_up"], act, save=fmt)
    grad_x, grad_w_gate, grad_w_up, h_again = gws.gated_bwd(s["grad_h"], x8, s["w_gate"], s["w_up"], saved, act, want_h=True)
    return dict(h=h, grad_x=grad_x, grad_w_gate=grad_w_gate, grad_w_up=grad_w_up, h_again=h_again)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- least work and exact results ------------------------------------------------------------------------------------

def work(case):
    op, m, k = case["op"], case["m"], case["k"]
    packed = lambda cols: m * -(-cols // GROUP) * (GROUP + 1)
    if op == "act8":                                  # x in, checkpoint out; checkpoint in, x out
        return dict(bytes=4 * m * k + 2 * packed(k), flops=0)
    n = case["n"]
    if op == "wgrad_act8":
        return dict(bytes=2 * m * n + packed(k) + 2 * n * k, flops=2 * m * n * k)
    if op == "gated":
        return dict(bytes=2 * (m * k + 2 * n * k + m * n), flops=4 * m * n * k)
    # x, both weights and grad_h in; h, grad_x, both weight gradients and h again out
    return dict(bytes=2 * (2 * m * k + 4 * n * k + 3 * m * n), flops=12 * m * n * k)


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


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    wide = lambda name: s[name].double()
    if op == "act8":
        return _exact_restored(wide("x"), s["fmt"])
    if op == "wgrad_act8":
        return wide("grad_y").T.contiguous() @ _unpack(s["x8"], s["m"], s["k"], s["fmt"], torch.float64)
    x, wg, wu = wide("x"), wide("w_gate"), wide("w_up")
    gate, up = x @ wg.T, x @ wu.T

    def act(g):
        if s["act"] == "silu":
            return g * torch.special.expit(g)
        if s["act"] == "relu":
            return torch.where(g > 0, g, 0.0)
        return g * torch.special.expit(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))    # (1 + tanh u) / 2 = sigmoid(2 u)

    h = act(gate) * up
    if op == "gated":
        return h
    gate, up, x = _exact_restored(gate, s["fmt"]), _exact_restored(up, s["fmt"]), _exact_restored(x, s["fmt"])
    grad_h = wide("grad_h")
    with torch.enable_grad():                                                                   # the slope by differentiation
        leaf = gate.detach().requires_grad_()
        a = act(leaf)
        grad_gate, = torch.autograd.grad(a, leaf, grad_h * up)
    a = a.detach()
    grad_up = grad_h * a
    return dict(h=h, grad_x=grad_gate @ wg + grad_up @ wu, grad_w_gate=grad_gate.T @ x, grad_w_up=grad_up.T @ x, h_again=a * up)
