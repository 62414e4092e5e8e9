"""Plain forms of the norm and of the optimizer for the tests (no code of the package): the norm in 64 bits, AdamW in 64 bits and, where the bits are
specified, operation by operation in numpy's 32."""
import numpy as np
import torch

GROUP = 256
U32 = 2.0 ** -24          # half a step of FP32, relative
U16 = 2.0 ** -8           # of BF16


# ---- layer norm --------------------------------------------------------------------------------------------------------
def norm(s, weight, bias, eps):
    """(y, xh, mean, rstd) in 64 bits."""
    s = s.double()
    mean = s.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((s - mean).square().mean(1, keepdim=True) + eps)
    xh = (s - mean) * rstd
    y = xh if weight is None else xh * weight.double()
    return (y if bias is None else y + bias.double()), xh, mean, rstd


def norm_depth(n):
    """Additions in a row on the way of an element into a sum over a row: 64 of a thread (n / 1024 where a block reads the row in turns), 5 of a warp, 32 of a block."""
    return max(64, n // 1024 + 1) + 37


def norm_errors(s, eps):
    """Bounds of what FP32 leaves in (mean, rstd relative to itself, xh)."""
    s = s.double()
    n = s.shape[1]
    d = (norm_depth(n) + 2) * U32
    mean = s.mean(1, keepdim=True)
    e_mean = d * s.abs().mean(1, keepdim=True)
    centred = (s - mean).abs()
    var = centred.square().mean(1, keepdim=True)
    # an error of the mean adds e^2 to the variance (its first order is a sum of zero) and 2 e times the centring's own rounding
    e_c = U32 * (centred + e_mean) + e_mean
    e_var = (d + 3 * U32) * var + e_mean.square() + 2 * (U32 * centred * centred).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    # the reciprocal root has two ulp, the sum with eps half of one; rstd falls by half of the variance's relative error
    e_rstd = 0.5 * e_var / (var + eps) * 1.01 + 6 * U32
    e_xh = e_c * rstd * (1 + e_rstd) + centred * rstd * (e_rstd + 2 * U32)
    return e_mean, e_rstd, e_xh


def norm_forward_bound(s, weight, bias, eps):
    y, xh, _, _ = norm(s, weight, bias, eps)
    _, _, e_xh = norm_errors(s, eps)
    w = 1.0 if weight is None else weight.double().abs()
    b = 0.0 if bias is None else bias.double().abs()
    err = w * e_xh + 2 * U32 * (w * xh.abs() + b)
    return err + U16 * (y.abs() + err)


def norm_backward(dy, s, weight, eps, grad_sum=None):
    """((dx, dweight, dbias), their bounds) in 64 bits; the bounds of the sums are without the rounding to their own type."""
    dy = dy.double()
    m, n = dy.shape
    _, xh, _, rstd = norm(s, None, None, eps)
    _, e_rstd, e_xh = norm_errors(s, eps)
    a = dy if weight is None else dy * weight.double()
    c1, c2 = a.mean(1, keepdim=True), (a * xh).mean(1, keepdim=True)
    inner = a - c1 - xh * c2
    dx = rstd * inner
    d = (norm_depth(n) + 3) * U32
    e1 = d * a.abs().mean(1, keepdim=True)
    e2 = d * (a * xh).abs().mean(1, keepdim=True) + (a.abs() * e_xh).mean(1, keepdim=True)
    size = a.abs() + c1.abs() + (xh * c2).abs()
    err = rstd * (e1 + (xh.abs() + e_xh) * e2 + e_xh * c2.abs() + 4 * U32 * size) + (e_rstd + U32) * dx.abs()
    if grad_sum is not None:
        dx = dx + grad_sum.double()
    err = err + U16 * (dx.abs() + err) + U32 * dx.abs()
    deep = (m + 300) * U32
    dw, db = (dy * xh).sum(0), dy.sum(0)
    return (dx, dw, db), (err, deep * (dy * xh).abs().sum(0) + (dy.abs() * e_xh).sum(0), deep * dy.abs().sum(0))


# ---- AdamW ---------------------------------------------------------------------------------------------------------------
f32 = np.float32


def split(w):
    """FP32 weights -> (BF16 bits as uint16, rest as int16)."""
    bits = w.view(np.uint32)
    high = ((bits.astype(np.uint64) + 0x8000) >> 16).astype(np.uint32)
    return high.astype(np.uint16), ((bits - (high << np.uint32(16))) & np.uint32(0xFFFF)).astype(np.uint16).view(np.int16)


def join(p_bits, rest):
    return ((p_bits.astype(np.uint32) << np.uint32(16)) + rest.astype(np.int32).view(np.uint32)).view(f32)


def round_bf16(w):
    """Nearest even, as uint16 bits."""
    bits = w.view(np.uint32).astype(np.uint64)
    return ((bits + 0x7FFF + ((bits >> 16) & 1)) >> 16).astype(np.uint16)


def _unit(top, step):
    unit = np.where(top >= f32(2.0 ** -100), top * f32(step), f32(0)).astype(f32)
    return np.where(np.isfinite(top), unit, f32(np.nan)).astype(f32)


def _inverse(unit):
    with np.errstate(all="ignore"):
        return np.where(unit > 0, f32(1) / unit, f32(0)).astype(f32)


E4M3 = np.array([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127], dtype=np.float64)
ROOTS = np.array([0.0] + [(1 + (c & 15) / 16) * 2.0 ** ((c >> 4) - 15) for c in range(1, 256)], dtype=np.float64)


def _nearest(grid, x):
    """Index of the nearest grid value, ties to the even index (even mantissa)."""
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo = hi - 1
    a, b = x - grid[lo], grid[hi] - x
    return np.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi)


def encode_m(m):
    """[groups, 256] FP32 -> (codes, units), by search in the grid."""
    m = m.reshape(-1, GROUP)
    unit = _unit(np.abs(m).max(1), 1 / 448)
    y = (m * _inverse(unit)[:, None]).astype(f32)
    code = _nearest(E4M3, np.minimum(np.abs(np.nan_to_num(y)).astype(np.float64), 448.0)).astype(np.uint8) | (np.signbit(y).astype(np.uint8) << 7)
    return np.where((unit > 0)[:, None], code, 0).astype(np.uint8), unit


def encode_r(r):
    r = r.reshape(-1, GROUP)
    unit = _unit(r.max(1), 1 / 1.9375)
    y = (r * _inverse(unit)[:, None]).astype(f32).astype(np.float64)
    code = np.maximum(_nearest(ROOTS, np.minimum(np.nan_to_num(y), 1.9375)), 1)
    return np.where((r > 0) & (unit > 0)[:, None], code, 0).astype(np.uint8), unit


def decode_m(codes, unit):
    codes = codes.reshape(-1, GROUP)
    value = E4M3[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    return (value.astype(f32) * unit.reshape(-1, 1)).astype(f32)


def decode_r(codes, unit):
    return (ROOTS[codes.reshape(-1, GROUP)].astype(f32) * unit.reshape(-1, 1)).astype(f32)


def adamw32(p, g, m, v, lr, b1, b2, eps, wd, step, scale=None):
    """One step in FP32, each operation rounded once.  Returns (p, m, v, r)."""
    alpha, rho, keep = f32(lr / (1 - b1 ** step)), f32(1 / np.sqrt(1 - b2 ** step)), f32(1 - lr * wd)
    with np.errstate(all="ignore"):
        g = g if scale is None else g * f32(scale)
        m = m * f32(b1) + g * f32(1 - b1)
        v = v * f32(b2) + (g * f32(1 - b2)) * g
        r = np.sqrt(v)
        return p * keep - (m * alpha) / (r * rho + f32(eps)), m, v, r


def adamw64(p, g, m, v, lr, b1, b2, eps, wd, step, scale=1.0):
    p, g, m, v = (np.asarray(t, dtype=np.float64) for t in (p, g, m, v))
    g = g * scale
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    return p * (1 - lr * wd) - lr / (1 - b1 ** step) * m / (np.sqrt(v) / np.sqrt(1 - b2 ** step) + eps), m, v
