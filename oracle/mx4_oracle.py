"""Oracle of the microscaled 4-bit operators, the balance loss and the router's gradient: plain numpy in 64 bits, written from the formulas.

Test infrastructure only.  Arrays of bf16, fp16 or fp32 values arrive widened to float64 (exact).
"""
import math

import numpy as np

NUMBERS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
MIDDLES = (NUMBERS[1:] + NUMBERS[:-1]) / 2
BLOCK = 32


def up(n, m):
    return -(-n // m) * m


def to_code(m):
    """Codes 0 .. 7 of magnitudes: the nearest number, ties to the even code."""
    at = np.searchsorted(MIDDLES, m)                                  # numbers whose upper middle lies below m
    tie = (at < 7) & (MIDDLES[np.minimum(at, 6)] == m)
    return np.where(tie & (at % 2 == 1), at + 1, at).astype(np.uint8)


def exponent(peak):
    """The byte of blocks with these largest magnitudes."""
    good = np.isfinite(peak)
    e = np.frexp(np.where(good & (peak > 0), peak, 1.0))[1] - 1       # floor(log2)
    return np.where(good, np.where(peak > 0, np.clip(e - 2 + 127, 0, 254), 0), 255).astype(np.uint8)


def quantize(x):
    """x [rows, K] -> codes [rows, Kp] (one a byte) and exponent bytes [rows, Kp / 32], Kp = K up to a multiple of 256."""
    rows, K = x.shape
    b = np.zeros((rows, up(K, 256)))
    b[:, :K] = x
    b = b.reshape(rows, -1, BLOCK)
    with np.errstate(invalid="ignore"):
        byte = exponent(np.abs(b).max(axis=2))
    unit = np.ldexp(1.0, byte.astype(int) - 127)
    number = (byte != 255)[..., None]
    m = np.abs(np.where(number & np.isfinite(b), b, 0.0)) / unit[..., None]
    codes = to_code(m) | np.where(np.signbit(b), 8, 0).astype(np.uint8)
    return np.where(number, codes, 0).astype(np.uint8).reshape(rows, -1), byte


def values(codes, byte):
    """What the codes stand for."""
    rows = codes.shape[0]
    unit = np.where(byte == 255, np.nan, np.ldexp(1.0, byte.astype(int) - 127))
    v = NUMBERS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return (v.reshape(rows, -1, BLOCK) * unit[..., None]).reshape(rows, -1)


def packed(codes):
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def tiles(codes, byte):
    """The tile layout, zeros behind the rows' end."""
    N, Kp = codes.shape
    n = up(N, 32)
    q = np.zeros((n, Kp // 2), np.uint8)
    q[:N] = packed(codes)
    s = np.zeros((n, Kp // BLOCK), np.uint8)
    s[:N] = byte
    q = q.reshape(n // 32, 32, Kp // 256, 2, 4, 16).transpose(0, 2, 4, 3, 1, 5)
    s = s.reshape(n // 32, 32, Kp // 256, 2, 4).transpose(0, 2, 3, 1, 4)
    return np.ascontiguousarray(q).reshape(n, Kp // 2), np.ascontiguousarray(s).reshape(n, Kp // BLOCK)


def matmul(xv, wv):
    """The product of two matrices of values, and a bound on what fp32 sums of its blocks may be off: a matrix instruction adds two blocks'
    exact sums to what is there, which is two roundings at most, each of 2^-24 of a number no larger than the sum of the blocks'
    magnitudes; and the parts that a shape splits K into meet in at most 16 additions.  (For blocks of like sizes.  Beside a block whose products are much
    larger than its sum the instruction cuts what is there: tests/test_gpu_mx4_bits.py has the bound for those.)"""
    T, K = xv.shape
    y = xv @ wv.T
    mag = np.zeros_like(y)
    for b in range(0, K, BLOCK):
        mag += np.abs(xv[:, b:b + BLOCK] @ wv[:, b:b + BLOCK].T)
    return y, (2 * (up(K, 256) // BLOCK) + 16) * 2.0 ** -24 * mag


def _range(h, dh):
    """The least and the largest value that rows known to dh may be converted to, [rows, F]."""
    rows, F = h.shape
    b, d = (np.zeros((rows, up(F, BLOCK))) for _ in range(2))
    b[:, :F], d[:, :F] = h, dh
    b, d = b.reshape(rows, -1, BLOCK), d.reshape(rows, -1, BLOCK)
    least = np.maximum(np.abs(b) - d, 0.0).max(axis=2)
    most = (np.abs(b) + d).max(axis=2)
    lo, hi = np.full(b.shape, math.inf), np.full(b.shape, -math.inf)
    e0, e1 = exponent(least).astype(int), exponent(most).astype(int)
    for e in (e0, e1):
        unit = np.ldexp(1.0, e - 127)[..., None]
        for v in (b - d, b + d):
            q = NUMBERS[to_code(np.abs(v) / unit)] * unit * np.sign(v)
            lo, hi = np.minimum(lo, q), np.maximum(hi, q)
    assert (e1 - e0 <= 1).all() or (most[e1 - e0 > 1] < 1e-30).all()
    return lo.reshape(rows, -1)[:, :F], hi.reshape(rows, -1)[:, :F]


def moe_ffn(xv, idx, gate, experts):
    """xv [T, H]: values of converted tokens; experts: per expert None or three matrices of values.  Returns y [T, H] and a bound on what a
    kernel with fp32 sums may be off: wherever the error of the intermediate reaches the middle of two codes, or that of a block's
    largest value a power of two, either value is allowed; elsewhere the codes are the same, and what they stand for exact."""
    T, H = xv.shape
    y, bound = np.zeros((T, H)), np.zeros((T, H))
    for e, mats in enumerate(experts):
        token, slot = np.nonzero(idx == e)
        if not len(token) or mats is None:
            continue
        w1, w3, w2 = mats
        x = xv[token]
        (a, da), (u, du) = matmul(x, w1), matmul(x, w3)
        with np.errstate(over="ignore"):
            s = a / (1.0 + np.exp(-a))
        h = s * u
        # |silu'| <= 1.1; silu and the product round by 9 steps of 2^-24 together
        dh = 1.1 * da * (np.abs(u) + du) + np.abs(s) * du + 9 * 2.0 ** -24 * np.abs(h) + 2.0 ** -140
        lo, hi = _range(h, dh)
        hv = values(*quantize(h))[:, :h.shape[1]]
        o, do = matmul(hv, w2)
        do = do + np.maximum(hi - hv, hv - lo) @ np.abs(w2).T
        g = gate[token, slot][:, None]
        np.add.at(y, token, g * o)
        # each pair's product with its weight and its addition round once
        np.add.at(bound, token, np.abs(g) * do)
    k = idx.shape[1]
    for e, mats in enumerate(experts):
        token, slot = np.nonzero(idx == e)
        if len(token) and mats is not None:
            x = xv[token]
            a, u = x @ mats[0].T, x @ mats[1].T
            with np.errstate(over="ignore"):
                h = values(*quantize(a / (1.0 + np.exp(-a)) * u))[:, :a.shape[1]]
            np.add.at(bound, token, (k + 1) * 2.0 ** -24 * np.abs(gate[token, slot][:, None] * (h @ mats[2].T)))
    return y, bound


def _scores(logits, sigmoid, lowest):
    """(masked [T, E], log of the scores, whether a token is no number [T])."""
    nan = np.isnan(logits).any(axis=1)
    if not sigmoid:
        nan |= (logits == math.inf).any(axis=1)
    masked = np.isnan(logits) | (logits <= lowest)
    l = np.where(masked, 0.0, logits)
    logs = np.minimum(l, 0.0) - np.log1p(np.exp(-np.abs(l))) if sigmoid else l
    return masked, np.where(masked, -math.inf, logs), nan


def _shares(logs):
    """e^logs over their sums, row by row; rows of zeros where there is nothing to divide."""
    top = np.max(logs, axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        z = np.where(np.isfinite(top) & (logs > -math.inf), np.exp(logs - top), 0.0)
    sums = z.sum(axis=1, keepdims=True)
    return z / np.where(sums > 0, sums, 1.0)


def balance(logits, idx, coef, sigmoid, keep=None, lowest=-math.inf):
    """(counts [E + 1], mean [E], loss)."""
    T, E = logits.shape
    k = idx.shape[1]
    part = np.ones(T, bool) if keep is None else np.asarray(keep) != 0
    chosen = idx[part]
    counts = np.append(np.bincount(chosen[(chosen >= 0) & (chosen < E)].reshape(-1), minlength=E), part.sum()).astype(np.int64)
    _, logs, nan = _scores(logits, sigmoid, lowest)
    p = np.where(nan[:, None], math.nan, _shares(logs))[part]
    M = int(counts[E])
    mean = np.array([math.fsum(c) if np.isfinite(c).all() else math.nan for c in p.T]) / M if M else np.zeros(E)
    loss = coef * E * float((counts[:E] / (M * k) * mean).sum()) if M else 0.0
    return counts, mean, loss


def backward(logits, idx, dw, sigmoid, renorm=True, factor=1.0, counts=None, coef=0.0, dloss=1.0, keep=None, lowest=-math.inf):
    """(gradient [T, E], size of the terms that meet in each of its values)."""
    T, E = logits.shape
    k = idx.shape[1]
    grad, size = np.zeros((T, E)), np.zeros((T, E))
    masked, logs, nan = _scores(logits, sigmoid, lowest)
    p = _shares(logs)
    l = np.where(masked, 0.0, logits)
    e = np.exp(-np.abs(l))
    rest = np.where(masked, 0.0, np.where(l > 0, e, 1.0) / (1.0 + e) if sigmoid else 1.0)
    part = np.zeros(T, bool) if counts is None else np.ones(T, bool) if keep is None else np.asarray(keep) != 0
    if counts is not None:
        M = float(counts[E])
        g = dloss * coef * E * counts[:E] / (M * M * k) if M else np.zeros(E)
        on = part[:, None] * rest * p
        grad += on * (g - (p * g).sum(axis=1, keepdims=True))
        size += on * (np.abs(g) + (p * np.abs(g)).sum(axis=1, keepdims=True))
    if dw is not None:
        rows = np.arange(T)[:, None].repeat(k, 1)
        inside = (idx >= 0) & (idx < E)
        to = np.where(inside, idx, 0)
        inside &= ~masked[rows, to]
        d = np.where(inside, dw, 0.0)
        lg = np.where(inside, logs[rows, to], -math.inf)

        def slots(v, s):
            np.add.at(grad, (rows[inside], to[inside]), v[inside])
            np.add.at(size, (rows[inside], to[inside]), s[inside])

        r = rest[rows, to]
        if renorm:
            q = _shares(lg)
            slots(factor * r * q * (d - (q * d).sum(axis=1, keepdims=True)), factor * r * q * (np.abs(d) + (q * np.abs(d)).sum(axis=1, keepdims=True)))
        elif sigmoid:
            slots(factor * np.exp(lg) * r * d, factor * np.exp(lg) * r * np.abs(d))
        else:
            q = np.where(inside, p[rows, to], 0.0)
            slots(factor * q * d, factor * q * np.abs(d))
            grad -= factor * p * (q * d).sum(axis=1, keepdims=True)
            size += factor * p * (q * np.abs(d)).sum(axis=1, keepdims=True)
    hit = nan & (part | (dw is not None))
    grad[hit] = math.nan
    return np.where((nan & ~hit)[:, None], 0.0, grad), size
