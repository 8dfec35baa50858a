"""Plain forms of the 8-bit linear layers and of the fused residual / norm step, on the host: integers in 32-bit
arithmetic as the header defines them, everything else in 64 bits.  And the error that a kernel may have."""
import numpy as np
import torch

U32 = 2.0 ** -24      # one rounding to fp32, relative
U16 = 2.0 ** -8       # one rounding to bf16, relative: torch.finfo(torch.bfloat16).eps / 2
FLT_MIN = np.float32(1.1754943508222875e-38)

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.detach().double().cpu().numpy()


def quantize(x, axis):
    """(integers, scales) of rows (axis 1) or columns (axis 0), every step rounded to fp32 once."""
    x = np.asarray(x, np.float32)
    top = np.abs(x).max(axis)
    with np.errstate(all="ignore"):
        scale = np.maximum(top * np.float32(1.0 / 127.0), FLT_MIN).astype(np.float32)
        inv = (np.float32(1.0) / scale).astype(np.float32)
        q = np.rint(x * np.expand_dims(inv, axis)).astype(np.float32)
    bad = ~np.isfinite(top)
    q = np.where(np.expand_dims(bad, axis), np.float32(0), q)
    return q.astype(np.int8), np.where(bad, np.float32(np.nan), scale)


def gelu(x):
    return torch.nn.functional.gelu(torch.from_numpy(np.ascontiguousarray(x))).numpy()


def linear_i8(a, a_scale, w, w_scale, bias, res, epi):
    """(out, size) in 64 bits; size: the sum of the magnitudes of what is added, for the bound on roundings."""
    acc = torch.from_numpy(np.ascontiguousarray(a, np.int8)).double() @ torch.from_numpy(np.ascontiguousarray(w, np.int8)).double()
    p = acc.numpy() * np.outer(np.asarray(a_scale, np.float64), np.asarray(w_scale, np.float64))
    b = 0.0 if bias is None else np.asarray(bias, np.float64)
    out, size = p + b, np.abs(p) + np.abs(b)
    if epi == "gelu":
        out = gelu(out)
    if epi == "res":
        out, size = out + res, size + np.abs(res)
    return out, size


def linear_bound(out, size, epi, dtype):
    """fp32: the sum's conversion, the product of the scales, the fused product and sum, the residual: 4 roundings of values up to
    `size`, 5 allowed.  GELU has a slope of at most 1.13 and takes a handful of roundings of its own (erff, two products, a sum):
    8 more; in bf16 a fitted form that is 2.5e-5 off at most (3e-5 allowed: its own roundings).  One rounding to the type."""
    tol = 5 * U32 * size
    if epi == "gelu":
        tol = 1.13 * tol + (8 * U32 * size if dtype == "f32" else 3e-5)
    return tol + (U16 * (np.abs(out) + tol) if dtype == "bf16" else U32 * np.abs(out))


def _norm(v, err, kind, eps, g, b):
    """Norm of rows and a bound on what fp32 makes of it, for values that are `err` off.  Sums over a row go through chains of at most
    64 terms and a tree: 96 roundings of the terms' magnitudes cover mean and variance with what is done to each value."""
    c = 96 * U32
    D = v.shape[-1]
    if kind == "none":
        return v, err
    mean = v.mean(-1, keepdims=True) if kind == "layer" else np.zeros_like(v[..., :1])
    err_mean = (err.mean(-1, keepdims=True) + c * np.abs(v).mean(-1, keepdims=True)) if kind == "layer" else 0.0
    d = v - mean
    r = 1.0 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    err_d = err + err_mean + 2 * U32 * (np.abs(v) + np.abs(mean))
    # r moves by r^3 mean(d err_d) and by the roundings of the sum of squares, half of which it feels
    err_r = r ** 3 * (np.abs(d) * err_d).mean(-1, keepdims=True) + r * c
    n = d * r
    err_n = err_d * r + np.abs(d) * err_r + 2 * U32 * np.abs(n)
    g = np.ones(D) if g is None else g
    b = np.zeros(D) if b is None else b
    return n * g + b, err_n * np.abs(g) + 2 * U32 * (np.abs(n * g) + np.abs(b))


def residual_norm(x, f, post, pre, post_eps, pre_eps, x_scale, f_scale, v):
    """x, f: [B, N, D] in 64 bits; v: the vectors (or None), gate and mod_* as [B or 1, 1, D].
    Returns y, u and the bounds on what fp32 makes of them before they are rounded for memory."""
    if f is None:
        y, ey = x * x_scale, U32 * np.abs(x * x_scale)
    else:
        p, ep = _norm(f, np.zeros_like(f), post, post_eps, v.get("post_g"), v.get("post_b"))
        gate = 1.0 if v.get("gate") is None else v["gate"]
        t, et = f_scale * gate * p, np.abs(f_scale * gate) * ep
        y = x * x_scale + t
        ey = et + 4 * U32 * (np.abs(x * x_scale) + np.abs(t))
    u, eu = _norm(y, ey, pre, pre_eps, v.get("pre_g"), v.get("pre_b"))
    ms = 0.0 if v.get("mod_scale") is None else v["mod_scale"]
    mt = 0.0 if v.get("mod_shift") is None else v["mod_shift"]
    u2 = u * (1 + ms) + mt
    return y, u2, ey, eu * (1 + np.abs(ms)) + 3 * U32 * (np.abs(u) * (1 + np.abs(ms)) + np.abs(mt))
