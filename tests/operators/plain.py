"""The operators around the compressed layer in 64 bits, straight from their formulas (include/qmoe.h), for the tests.

Next to a result stands the sum of the absolute terms that an fp32 evaluation adds up: a bound on its error is a
number of roundings (2^-24 each) of that sum."""
import numpy as np

U32, U_BF16 = 2.0 ** -24, 2.0 ** -8  # half a step, relative to the value: fp32, bf16


def bf16(a):
    """float array -> nearest bf16 (ties to even), as float64"""
    f = np.ascontiguousarray(np.asarray(a, dtype=np.float64).astype(np.float32))
    u = f.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    return np.where(np.isfinite(f), r.view(np.float32), f).astype(np.float64)


def bf16_bits(a):
    return (bf16(a).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def of_bits(b):
    return (np.asarray(b, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


# ---------------------------------------------------------------- residual stream and norm

def norm(v, kind, weight, bias, eps, err):
    """-> (normed v, bound on its error); err: bound on v's.  A row's sums run over d values, at most 8 * 4 in a lane, then 6 + 16
    more additions: under 64 roundings."""
    d = v.shape[1]
    w = np.ones(d) if weight is None else weight.astype(np.float64)
    b = np.zeros(d) if bias is None else bias.astype(np.float64)
    mean = v.mean(axis=1, keepdims=True) if kind == "layer" else np.zeros((v.shape[0], 1))
    size = np.abs(v) + (np.abs(v).mean(axis=1, keepdims=True) if kind == "layer" else 0.0)
    c, c_err = v - mean, err + err.mean(axis=1, keepdims=True) * (kind == "layer") + 64 * U32 * size
    q = (c * c).mean(axis=1, keepdims=True) + eps
    r = 1.0 / np.sqrt(q)
    # relative error of r: half that of q, and a few roundings of root and quotient
    r_rel = (np.abs(c) * c_err).mean(axis=1, keepdims=True) / q + 36 * U32
    out = c * r * w + b
    return out, (c_err * r + np.abs(c) * r * (r_rel + 3 * U32)) * np.abs(w) + 2 * U32 * (np.abs(c * r * w) + np.abs(b))


def residual_norm(h, y, k, gate, post, alpha, channel, pre, copies):
    """post, pre: None or (kind, weight, bias, eps).  -> h' before its rounding, its error bound, x before its rounding [n * copies, d], its bound"""
    n, d = h.shape
    v, err = h.astype(np.float64), np.zeros((n, d))
    if y is not None:
        g = np.ones(n * k) if gate is None else gate.astype(np.float64)
        terms = (y.astype(np.float64) * g[:, None]).reshape(n, k, d)
        b, b_err = terms.sum(axis=1), (k + 1) * U32 * np.abs(terms).sum(axis=1)
        if post is not None:
            b, b_err = norm(b, *post, err=b_err)
        c = np.ones(d) if channel is None else channel.astype(np.float64)
        a = float(np.float32(alpha))
        err = np.abs(a * c) * b_err + 3 * U32 * (np.abs(a * c * b) + np.abs(v))
        v = v + a * c * b
    x, x_err = (v, err) if pre is None else norm(v, *pre, err=err)
    return v, err, np.repeat(x, copies, axis=0), np.repeat(x_err, copies, axis=0)


# ---------------------------------------------------------------- the router's choice

def route(logits, bias, mask, k, chosen):
    """logits: float32 values.  -> idx int32 [n, k], gates float64, relative bound on the gates' error"""
    l = np.asarray(logits, dtype=np.float32)
    n, e = l.shape
    big = np.float32(np.finfo(np.float32).max)
    with np.errstate(over="ignore", invalid="ignore"):
        l = np.where(np.isnan(l), np.float32(-np.inf), np.minimum(l, big))
        key = l if bias is None else l + np.asarray(bias, dtype=np.float32)[None, :]
        key = np.where(np.isnan(key) | (l == -np.inf), np.float32(-np.inf), np.minimum(key, big))
    idx, gate, rel = np.full((n, k), -1, np.int32), np.zeros((n, k)), np.zeros((n, k))
    for t in range(n):
        if mask is not None and not mask[t]:
            continue
        order = sorted(range(e), key=lambda i: (-float(key[t, i]), i))[:k]
        order = [i for i in order if key[t, i] > -np.inf]
        over = [float(l[t, i]) for i in (order if chosen else range(e)) if l[t, i] > -np.inf]
        if not order:
            continue
        top = max(over)
        s = sum(np.exp(v - top) for v in over)
        for j, i in enumerate(order):
            idx[t, j], gate[t, j] = i, np.exp(float(l[t, i]) - top) / s
            # the difference of two logits is rounded once, exp and quotient to a few steps; sums of at most 32 + 8 (wide: 64 + 8) terms
            rel[t, j] = (min(abs(float(l[t, i]) - top), 120.0) + 100) * U32
    return idx, gate, rel


# ---------------------------------------------------------------- four-bit weights

def int4_place(c):
    """The byte of a row and the shift inside it where column c stands: word 4 i + s of a block, bits 4 j (even) or 16 + 4 j."""
    block, within = c // 128, c % 128
    s, i, e = within // 32, within % 32 // 8, within % 8
    bit = 32 * (4 * i + s) + (4 * (e // 2) if e % 2 == 0 else 16 + 4 * (e // 2))
    return 64 * block + bit // 8, bit % 8


def int4_pack(values):
    rows, cols = values.shape
    out = np.zeros((rows, 64 * ((cols + 127) // 128)), dtype=np.uint8)
    for c in range(cols):
        byte, shift = int4_place(c)
        out[:, byte] |= (values[:, c] << shift).astype(np.uint8)
    return out


def int4_matrix(values, scale_bits, zero, group):
    """-> W float64 [rows, cols], and |s| (16 + q + 16 + z), what a kernel that adds and takes off 16 + z adds up"""
    rows, cols = values.shape
    g = np.arange(cols) // group
    s = np.asarray(scale_bits, dtype=np.uint16).view(np.float16).astype(np.float64)[:, g]
    z = 8.0 if zero is None else zero.astype(np.float64)[:, g]
    return s * (values - z), np.abs(s) * (32.0 + values + z)


def int4_steps(cols, group):
    """Roundings on the way of a term: at most 128 products of its group, a scale and a difference, the groups, eight parts."""
    return 128 + 4 + 8 + (cols + min(group, 128) - 1) // min(group, 128)


def activate(v, err, act):
    """v, err: [tokens, rows] -> the same after the activation; derivatives of relu, silu and gelu are below 1.13"""
    if act == "none":
        return v, err
    if act == "relu":
        return np.maximum(v, 0.0), err
    half = v.shape[1] // 2
    g, u, ge, ue = v[:, :half], v[:, half:], err[:, :half], err[:, half:]
    with np.errstate(over="ignore"):
        a = g / (1.0 + np.exp(-g)) if act == "silu" else 0.5 * g * (1.0 + np.tanh(np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)))
    # exp's argument is rounded (|g| steps of the result); 1 + tanh loses what it cancels: an absolute error of |g| / 2 times a few steps
    a_err = 1.13 * ge + U32 * (8 + np.minimum(np.abs(g), 90.0)) * (np.abs(a) if act == "silu" else np.abs(g))
    return a * u, a_err * np.abs(u) + (np.abs(a) + a_err) * ue + 4 * U32 * np.abs(a * u)


def int4_product(x, values, scale_bits, zero, group, act):
    """x [tokens, cols] -> result float64 and a bound on an fp32 evaluation's error"""
    w, size = int4_matrix(values, scale_bits, zero, group)
    return activate(x @ w.T, int4_steps(values.shape[1], group) * U32 * (np.abs(x) @ size.T), act)
