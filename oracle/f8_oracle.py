"""CPU oracle of the 8-bit products and the routing in 64 bits, from the definitions (numpy only; shares no code with the kernels).

e4m3: sign, 4 exponent bits with bias 7, 3 fraction bits, largest value 448, steps of 2^-9 below 2^-6.  A block's scale is the least
power of two 2^e, e >= -126, with max |v| <= 448 * 2^e; values are v / 2^e, rounded to the nearest e4m3 number, ties to even."""
import numpy as np

BLOCK = 128


def exponent(amax):
    """e for a block's largest magnitude"""
    m, e = np.frexp(np.asarray(amax, np.float64) / 448)   # in [0.5, 1) * 2^e, exact: 24 bits over a power of two times 7
    return np.maximum(np.where(m == 0, -126, np.where(m == 0.5, e - 1, e)), -126)


def round_e4m3(v):
    """the nearest e4m3 number, ties to even, for |v| <= 448"""
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(v / step) * step


def quantise_rows(x):
    """x [rows, in] -> (values that x stands for in 8 bits, exponents [rows, blocks])"""
    x = np.asarray(x, np.float64)
    n, width = x.shape
    kb = -(-width // BLOCK)
    pad = np.zeros((n, kb * BLOCK))
    pad[:, :width] = x
    pad = pad.reshape(n, kb, BLOCK)
    bad = ~np.isfinite(pad).all(axis=2)
    e = exponent(np.abs(np.where(bad[:, :, None], 0, pad)).max(axis=2))
    s = np.ldexp(1.0, e)[:, :, None]
    v = round_e4m3(np.where(bad[:, :, None], 0, pad) / s) * s
    v[bad] = np.nan
    return v.reshape(n, -1)[:, :width], e


def quantise_weight(w):
    """w [out, in] -> (values, exponents [row blocks, column blocks])"""
    w = np.asarray(w, np.float64)
    out, inn = w.shape
    nb, kb = -(-out // BLOCK), -(-inn // BLOCK)
    pad = np.zeros((nb * BLOCK, kb * BLOCK))
    pad[:out, :inn] = w
    pad = pad.reshape(nb, BLOCK, kb, BLOCK)
    e = exponent(np.abs(pad).max(axis=(1, 3)))
    s = np.ldexp(1.0, e)[:, None, :, None]
    return (round_e4m3(pad / s) * s).reshape(nb * BLOCK, -1)[:out, :inn], e


def weight_values(q, s):
    """e4m3 numbers [out, in] and scales [row blocks, column blocks] -> the weight"""
    q, s = np.asarray(q, np.float64), np.asarray(s, np.float64)
    return q * np.repeat(np.repeat(s, BLOCK, 0)[: q.shape[0]], BLOCK, 1)[:, : q.shape[1]]


def gated(x):
    g, u = np.split(np.asarray(x, np.float64), 2, axis=1)
    return g / (1 + np.exp(-g)) * u


def route(logits, top_k, renormalise):
    """(experts, weights, slots, rows, offsets), token by token"""
    l = np.asarray(logits, np.float64)
    n, e = l.shape
    l = np.where(np.isnan(l), -np.inf, np.minimum(l, np.finfo(np.float32).max))
    experts, weights = np.full((n, top_k), -1, np.int32), np.zeros((n, top_k))
    for t in range(n):
        order = [i for i in sorted(range(e), key=lambda i: (-l[t, i], i)) if l[t, i] > -np.inf]
        if not order:
            continue
        p = np.exp(l[t] - l[t, order[0]])
        top = order[:top_k]
        total = p[top].sum() if renormalise else p[l[t] > -np.inf].sum()
        experts[t, : len(top)] = top
        weights[t, : len(top)] = p[top] / total
    slots, rows = np.full((n, top_k), -1, np.int32), np.full(n * top_k, -1, np.int32)
    offsets, at = [0], 0
    for i in range(e):
        for t, j in zip(*np.nonzero(experts == i)):   # in the order of (token, j)
            slots[t, j], rows[at] = at, t
            at += 1
        offsets.append(at)
    return experts, weights, slots, rows, np.asarray(offsets, np.int32)
