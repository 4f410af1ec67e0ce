"""GPU parity of the balance loss and of the router's gradient against their oracle (64 bits).

Tolerances: a share p is a quotient of exponentials.  An exponent's argument is a difference of two fp32 numbers, rounded by 2^-24 of
itself (d, which moves p by |d| 2^-24); the exponential by 2^-22 (the instruction's ulp, its argument's correction and its product), a sum over up
to 1024 experts by 2^-24 for each of its at most 22 additions (16 in a lane, 6 across lanes), quotient and sigmoid's sum and product
by 4 of 2^-24.  With |d| <= 40: EPS = 80 * 2^-24 in all for a score divided by a sum; p smaller than e^-40 of the largest is held to (1 + |d|) 2^-23 more.
* counts are equal; a mean is a sum in 64 bits of such p, rounded once; the loss is one of those means.
* a gradient is a sum of products of at most two such numbers and 1 - s (8 of 2^-24), with fp32 sums: 3 EPS of the terms that meet in it
  (the oracle's second result), and half a step of its type.
"""
import math

import numpy as np
import pytest
import torch

from oracle import mx4_oracle as Q
from paper_2603_19172_amd import binding as B
from gpu_helpers import DEV

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LOWEST = {t: torch.finfo(t).min for t in HALF}
OUT = {torch.bfloat16: B.OUT_BF16, torch.float16: B.OUT_F16, torch.float32: B.OUT_F32}
SCORES = [B.SCORE_SIGMOID, B.SCORE_SOFTMAX]
EPS = 80 * 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    c.close()


def f64(t):
    return t.detach().double().cpu().numpy()


def randn(seed, *shape, dtype=torch.float32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).to(DEV)


def choose(seed, T, E, k):
    g = torch.Generator().manual_seed(seed)
    return torch.rand((T, E), generator=g).topk(k, dim=-1).indices.to(torch.int32).to(DEV)


def keep_some(seed, T, share):
    return (torch.rand(T, generator=torch.Generator().manual_seed(seed)) < share).to(torch.uint8).to(DEV)


def check_balance(ctx, logits, idx, coef, score, keep=None):
    counts, mean, loss = ctx.route_balance(logits, idx, coef, score=score, keep=keep)
    c, m, l = Q.balance(f64(logits), idx.cpu().numpy(), float(np.float32(coef)), score == B.SCORE_SIGMOID,
                        None if keep is None else keep.cpu().numpy(), LOWEST[logits.dtype])
    assert np.array_equal(counts.cpu().numpy(), c)
    assert np.array_equal(np.isnan(f64(mean)), np.isnan(m)) and math.isnan(float(loss)) == math.isnan(l)
    ok = ~np.isnan(m)
    assert (np.abs(f64(mean) - m)[ok] <= EPS * np.abs(m)[ok] + 2.0 ** -126).all()
    if not math.isnan(l):
        assert abs(float(loss) - l) <= EPS * abs(l) + 2.0 ** -126
    return counts


def check_backward(ctx, logits, idx, score, dw=None, renorm=True, factor=1.0, counts=None, coef=0.0, dloss=None, keep=None, out=None):
    grad = ctx.route_scored_backward(logits, idx, dw=dw, score=score, renorm=renorm, factor=factor, counts=counts, coef=coef, dloss=dloss,
                                     keep=keep, grad_dtype=None if out is None else OUT[out])
    t = logits.dtype if out is None else out
    assert grad.dtype == t
    ref, size = Q.backward(f64(logits), idx.cpu().numpy(), None if dw is None else f64(dw), score == B.SCORE_SIGMOID, renorm,
                           float(np.float32(factor)), None if counts is None else counts.cpu().numpy(), float(np.float32(coef)),
                           1.0 if dloss is None else float(dloss), None if keep is None else keep.cpu().numpy(), LOWEST[logits.dtype])
    got = f64(grad)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    ok = ~np.isnan(ref)
    tiny = 2.0 ** -25 if t == torch.float16 else 2.0 ** -126
    off = np.abs(got - ref)[ok] - (3 * EPS * size[ok] + HALF[t] * np.abs(ref)[ok] + tiny)
    assert (off <= 0).all(), off.max()
    return grad


SIZES = [(1, 1, 1), (1, 256, 8), (2, 7, 7), (24, 128, 8), (32, 64, 6), (33, 65, 3), (130, 60, 4), (257, 300, 10), (9, 1000, 12), (70, 1024, 64), (515, 513, 2),
         (2300, 16, 2)]


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("score", SCORES)
def test_balance_and_gradient(ctx, T, E, k, dtype, score):
    logits, idx = randn(E + k, T, E, dtype=dtype, std=2.0), choose(T, T, E, k)
    dw, dloss = randn(T, T, k), torch.tensor([0.7], device=DEV)
    for keep in (None, keep_some(T, T, 0.6)):
        counts = check_balance(ctx, logits, idx, 0.01, score, keep)
        # the loss weighs as much as the gate weights: a gradient in which both parts can be seen
        coef = 0.1 * T
        for renorm, factor in ((True, 1.0), (False, 2.5)):
            check_backward(ctx, logits, idx, score, dw, renorm, factor, counts, coef, dloss, keep)
            check_backward(ctx, logits, idx, score, dw, renorm, factor)
        check_backward(ctx, logits, idx, score, counts=counts, coef=coef, keep=keep)
    for out in OUT:
        check_backward(ctx, logits, idx, score, dw, counts=counts, coef=coef, out=out)


@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_masks_and_what_is_no_number(ctx, score, dtype):
    E, k = 80, 6
    low = LOWEST[dtype]
    one = torch.randn(E, generator=torch.Generator().manual_seed(1))
    few = torch.full((E,), -math.inf)
    few[[3, 41, 42]] = torch.tensor([0.5, -2.0, 1.0])
    rows = [torch.zeros(E), torch.full((E,), -math.inf), torch.full((E,), low), few, torch.where(few > -math.inf, few, torch.tensor(low)),
            torch.full((E,), -300.0), torch.linspace(-39, 1, E), torch.linspace(-1, 39, E), one * 0 - 60.0 + one]
    idx = choose(2, len(rows), E, k)
    idx[3:5, :4] = torch.tensor([3, 41, 7, 42], dtype=torch.int32)
    logits = torch.stack(rows).to(dtype).to(DEV)
    dw = randn(3, len(rows), k)
    counts = check_balance(ctx, logits, idx, 0.5, score)
    for renorm in (True, False):
        g = check_backward(ctx, logits, idx, score, dw, renorm, 1.3, counts, 0.5)
        assert (g[1:3] == 0).all() and (g[3][torch.isinf(few).to(DEV)] == 0).all()
    # NaN and infinities: their token alone, and in the means only where it takes part
    bad = []
    for v in (math.nan, math.inf, -math.inf):
        r = one.clone()
        r[[5, 60]] = v
        bad.append(r)
    logits = torch.stack([one, *bad, one]).to(dtype).to(DEV)
    idx, dw = choose(4, 5, E, k), randn(5, 5, k)
    keep = torch.tensor([1, 0, 0, 1, 1], dtype=torch.uint8, device=DEV)
    check_balance(ctx, logits, idx, 0.5, score)
    counts = check_balance(ctx, logits, idx, 0.5, score, keep)
    for renorm in (True, False):
        check_backward(ctx, logits, idx, score, dw, renorm, 1.0, counts, 0.5, keep=keep)
        check_backward(ctx, logits, idx, score, dw, renorm, 1.0)
    check_backward(ctx, logits, idx, score, counts=counts, coef=0.5, keep=keep)


@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("T", [5, 200])
def test_indices_outside_and_twice(ctx, score, T):
    E, k = 20, 4
    logits, idx, dw = randn(1, T, E), choose(1, T, E, k), randn(2, T, k)
    idx[0] = torch.tensor([-1, 20, 1 << 30, -(1 << 31)], dtype=torch.int32)
    idx[1] = 7
    idx[2, 1:3] = torch.tensor([-5, 0], dtype=torch.int32)
    counts = check_balance(ctx, logits, idx, 0.3, score)
    for renorm in (True, False):
        check_backward(ctx, logits, idx, score, dw, renorm, 1.0, counts, 3.0)


@pytest.mark.parametrize("T", [0, 1, 20, 90])
@pytest.mark.parametrize("score", SCORES)
def test_no_tokens_take_part(ctx, T, score):
    E, k = 70, 3
    logits, idx = randn(1, T, E), choose(1, T, E, k)
    keep = torch.zeros((T,), dtype=torch.uint8, device=DEV)
    counts, mean, loss = ctx.route_balance(logits, idx, 1.0, score=score, keep=keep)
    assert (counts == 0).all() and (mean == 0).all() and float(loss) == 0
    g = ctx.route_scored_backward(logits, idx, score=score, counts=counts, coef=1.0, keep=keep)
    assert g.shape == (T, E) and (g == 0).all()


def test_gradient_against_differences_of_the_forward_calls(ctx):
    """Through route_scored and route_balance themselves: fp32 outputs of two calls, so differences are good to 2^-22 / d."""
    T, E, k, d = 6, 12, 3, 2.0 ** -6
    for score in SCORES:
        for renorm in (True, False):
            logits = randn(9, T, E)
            idx, w = ctx.route_scored(logits, k, score=score, renorm=renorm, factor=2.0)
            dw, coef = randn(10, T, k), 5.0
            counts, _, _ = ctx.route_balance(logits, idx, coef, score=score)
            grad = f64(ctx.route_scored_backward(logits, idx, dw=dw, score=score, renorm=renorm, factor=2.0, counts=counts, coef=coef))

            def total(l):
                # the choices are held: an expert that has moved keeps its slot
                s = torch.empty((T, E), device=DEV)
                ctx.route_scored(l, k, score=score, scores=s)
                v = s.double().gather(1, idx.long())
                v = 2.0 * (v / v.sum(1, keepdim=True) if renorm else v)
                _, _, loss = ctx.route_balance(l, idx, coef, score=score)
                return float((v * dw.double()).sum()) + float(loss)
            for t in range(T):
                for e in range(E):
                    hi, lo = logits.clone(), logits.clone()
                    hi[t, e] += d
                    lo[t, e] -= d
                    got = (total(hi) - total(lo)) / (2 * d)
                    # third derivatives of a few (|dw| up to 3, factor 2): d^2 / 6 of them; fp32 totals of up to 8
                    assert abs(got - grad[t, e]) <= 6 * d * d / 6 * 4 + 8 * 2.0 ** -22 / d


def test_long_batches_and_every_run_alike(ctx):
    T, E, k = 40000, 96, 4
    logits, idx = randn(1, T, E, dtype=torch.bfloat16), choose(2, T, E, k)
    for score in SCORES:
        first = ctx.route_balance(logits, idx, 0.1, score=score)
        p = logits.double().sigmoid() if score == B.SCORE_SIGMOID else logits.double().softmax(-1)
        mean = (p / p.sum(-1, keepdim=True)).mean(0)
        assert (torch.abs(first[1].double() - mean) <= EPS * mean).all()
        assert torch.equal(first[0][:E], torch.bincount(idx.reshape(-1).long(), minlength=E).to(torch.int32)) and int(first[0][E]) == T
        loss = 0.1 * E * float((first[0][:E].double() / (T * k) * mean).sum())
        assert abs(float(first[2]) - loss) <= 2 * EPS * loss
        dw = randn(3, T, k)
        grad = ctx.route_scored_backward(logits, idx, dw=dw, score=score, counts=first[0], coef=0.1)
        for _ in range(3):
            again = ctx.route_balance(logits, idx, 0.1, score=score)
            assert all(torch.equal(a, b) for a, b in zip(first, again))
            assert torch.equal(grad, ctx.route_scored_backward(logits, idx, dw=dw, score=score, counts=first[0], coef=0.1))
        check_backward(ctx, logits[-300:], idx[-300:], score, dw[-300:])
        # rows do not depend on their company where the counts are the same
        assert torch.equal(grad[-300:], ctx.route_scored_backward(logits[-300:], idx[-300:], dw=dw[-300:], score=score, counts=first[0], coef=0.1))


@pytest.mark.parametrize("T", [20, 600])
def test_another_stream_a_graph_and_any_workspace(ctx, T):
    E, k = 130, 5
    sets = [(randn(s, T, E), choose(s, T, E, k)) for s in range(3)]
    want = [ctx.route_balance(*s, 0.2) for s in sets]
    grads = [ctx.route_scored_backward(*s, counts=w[0], coef=0.2, dloss=w[2]) for s, w in zip(sets, want)]
    nb = B.route_balance_workspace_bytes(T, E)
    buf = torch.full((nb + 256,), 255, dtype=torch.uint8, device=DEV)
    got = ctx.route_balance(*sets[0], 0.2, workspace=buf[:nb])
    assert all(torch.equal(a, b) for a, b in zip(got, want[0])) and (buf[nb:] == 255).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [ctx.route_balance(*s, 0.2, stream=side) for s in sets]
    back = [ctx.route_scored_backward(*s, counts=w[0], coef=0.2, dloss=w[2], stream=side) for s, w in zip(sets, got)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w)) and all(torch.equal(a, b) for a, b in zip(back, grads))
    logits, idx = (t.clone() for t in sets[0])
    out = tuple(torch.empty_like(t) for t in want[0])
    grad = torch.empty_like(grads[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.route_balance(logits, idx, 0.2, counts=out[0], mean=out[1], loss=out[2], workspace=buf)
        ctx.route_scored_backward(logits, idx, counts=out[0], coef=0.2, dloss=out[2], out=grad)
    for s, w, g in zip(sets, want, grads):
        logits.copy_(s[0])
        idx.copy_(s[1])
        buf.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, w)) and torch.equal(grad, g)


def test_rows_behind_the_last_are_left(ctx):
    T, E, k = 9, 50, 3
    logits, idx = randn(1, T, E), choose(1, T, E, k)
    grad = torch.full((T + 2, E), 7.0, device=DEV)
    ctx.route_scored_backward(logits, idx, dw=randn(2, T, k), out=grad[:T])
    counts = torch.full((E + 3,), 7, dtype=torch.int32, device=DEV)
    ctx.route_balance(logits, idx, 0.1, counts=counts[:E + 1])
    assert (grad[T:] == 7).all() and (counts[E + 1:] == 7).all()


def test_as_many_tokens_as_the_calls_take(ctx):
    T, E = (1 << 25) - 1, 2
    logits = torch.zeros((T, E), dtype=torch.bfloat16, device=DEV)
    logits[::4, 1] = 1.0
    idx = (torch.arange(T, device=DEV) % 4 == 0).to(torch.int32)[:, None].contiguous()
    counts, mean, loss = ctx.route_balance(logits, idx, 1.0, score=B.SCORE_SOFTMAX)
    many = -(-T // 4)
    assert counts.tolist() == [T - many, many, T]
    p = math.e / (1.0 + math.e)
    want = [((T - many) * 0.5 + many * (1 - p)) / T, ((T - many) * 0.5 + many * p) / T]
    assert all(abs(float(m) - w) <= EPS * w for m, w in zip(mean, want))
    assert abs(float(loss) - 2 * ((T - many) / T * want[0] + many / T * want[1])) <= 2 * EPS
    dw = torch.ones((T, 1), device=DEV)
    grad = ctx.route_scored_backward(logits, idx, dw=dw, score=B.SCORE_SOFTMAX, renorm=False)
    for i in (0, 1, T // 2 // 4 * 4, T - 1):
        q = p if i % 4 == 0 else 0.5
        g = q * (1 - q)
        w = [-g, g] if i % 4 == 0 else [g, -g]
        assert all(abs(float(a) - b) <= (3 * EPS + 2.0 ** -8) * g for a, b in zip(grad[i], w))
    for r in (0, 1, 2, 3):
        assert (grad[r::4] == grad[r]).all()
