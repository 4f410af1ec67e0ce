"""Oracle of the routing by scores and of the products in 8-bit integers: plain numpy in 64 bits, written from the formulas.

Test infrastructure only.  Arrays of bf16 values arrive widened to float64 (exact), masks as -inf or as the type's lowest value.
"""
import math

import numpy as np


def route_scored(logits, k, bias=None, sigmoid=True, groups=1, top_groups=1, group_best=1, renorm=True, factor=1.0, lowest=-math.inf):
    """logits [T, E] float64; lowest: the value up to which a logit is a mask.  Returns idx [T, k], w [T, k], scores [T, E]."""
    T, E = logits.shape
    per = E // groups
    idx, w, scores = np.zeros((T, k), np.int32), np.zeros((T, k)), np.zeros((T, E))
    for t in range(T):
        nan = any(math.isnan(v) for v in logits[t]) or (not sigmoid and any(v == math.inf for v in logits[t]))
        masked = [math.isnan(v) or v <= lowest for v in logits[t]]
        s = [0.0] * E
        if sigmoid:
            for e in range(E):
                if not masked[e]:
                    v = float(logits[t, e])
                    s[e] = 1.0 / (1.0 + math.exp(-v)) if v > -700.0 else 0.0
        elif not nan and not all(masked):
            top = max(float(logits[t, e]) for e in range(E) if not masked[e])
            z = [0.0 if masked[e] else math.exp(float(logits[t, e]) - top) for e in range(E)]
            s = [v / math.fsum(z) for v in z]
        c = []
        for e in range(E):
            v = -math.inf if masked[e] else float(logits[t, e]) if bias is None else s[e] + float(bias[e])
            c.append(-math.inf if math.isnan(v) else v)
        allowed = list(range(E))
        if groups > 1:
            value = []
            for g in range(groups):
                inside = range(g * per, (g + 1) * per)
                v = [c[e] for e in inside] if bias is not None or group_best == 1 else [-math.inf if masked[e] else s[e] for e in inside]
                v = sorted(v, reverse=True)
                value.append(v[0] + v[1] if group_best == 2 and per > 1 and v[1] > -math.inf else v[0])
            best = sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups]
            allowed = [e for e in range(E) if e // per in best]
        chosen = sorted(allowed, key=lambda e: (-c[e], e))[:k]
        idx[t] = chosen
        total = math.fsum(s[e] for e in chosen)
        for j, e in enumerate(chosen):
            w[t, j] = math.nan if nan else factor * ((s[e] / total if total > 0 else 0.0) if renorm else s[e])
        scores[t] = math.nan if nan else s
    return idx, w, scores


def quantize_rows(x):
    """x [rows, K] float64 (values of a 16- or 32-bit type) -> codes [rows, K] int8, scale [rows] float32."""
    a = np.abs(x).max(axis=1) if x.shape[1] else np.zeros(x.shape[0])
    good = np.isfinite(a)
    div = np.where(good & (a > 0), a, 1.0)
    q = np.where((good & (a > 0))[:, None], 127.0 * np.where(np.isfinite(x), x, 0.0) / div[:, None], 0.0)
    scale = np.where(good, a.astype(np.float32) / np.float32(127.0), np.float32(np.nan)).astype(np.float32)
    return np.rint(q).astype(np.int8), scale


def tiles(codes):
    """Row-major int8 codes -> the library's tile layout, zeros behind both ends."""
    N, K = codes.shape
    n, k = -(-N // 32) * 32, -(-K // 128) * 128
    p = np.zeros((n, k), np.int8)
    p[:N, :K] = codes
    return np.ascontiguousarray(p.reshape(n // 32, 32, k // 128, 2, 4, 16).transpose(0, 2, 4, 3, 1, 5)).reshape(n, k)


def matmul(xq, xs, wq, ws):
    """The product without its bias, float64."""
    return (xq.astype(np.float64) @ wq.astype(np.float64).T) * xs.astype(np.float64)[:, None] * ws.astype(np.float64)[None, :]


def moe_ffn(x, idx, gate, experts, eps_h):
    """experts: per expert None or three (codes, scale) pairs, row-major.  Returns y [T, H]; a bound on what a kernel may be off
    where the intermediate carries a relative error of eps_h, that a chance of 2e-9 an output exceeds; its mean square; and what a
    kernel might be off beside that that rounded the pairs' outputs to fp16 (the library's does not).  tests/test_gpu_int8.py derives them."""
    T, H = x.shape
    xq, xs = quantize_rows(x)
    y, var, drift, half, most = (np.zeros((T, H)) for _ in range(5))
    for t in range(T):
        for j, e in enumerate(idx[t]):
            if not 0 <= e < len(experts) or experts[e] is None:
                continue
            (q1, s1), (q3, s3), (q2, s2) = experts[e]
            a, u = (matmul(xq[t:t + 1], xs[t:t + 1], q, s)[0] for q, s in ((q1, s1), (q3, s3)))
            h = a / (1.0 + np.exp(-a)) * u
            peak = np.abs(h).max()
            step = peak / 127.0
            hv = np.rint(h / step) * step if peak > 0 else h * 0.0
            w2 = q2.astype(np.float64) * s2.astype(np.float64)[:, None]
            g = float(gate[t, j])
            o = w2 @ hv
            y[t] += g * o
            drift[t] += abs(g) * np.abs(o) * eps_h
            half[t] += abs(g) * (np.abs(o) * 2.0 ** -11 + 2.0 ** -40 * 127 * 127 * h.size * step * float(s2.max()))
            var[t] += g * g * (w2 ** 2 @ (2.0 * eps_h * np.abs(h) * step))
            most[t] = np.maximum(most[t], abs(g) * step * np.abs(w2).max(axis=1))
    rare = math.log(2.0 / 2e-9)
    bound = most * rare / 3.0 + np.sqrt((most * rare / 3.0) ** 2 + 2.0 * var * rare)
    return y, bound * (eps_h > 0) + drift, var + drift ** 2, half
