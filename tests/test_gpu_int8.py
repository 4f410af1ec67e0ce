"""GPU parity of the routing by scores and of the products in 8-bit integers against their oracle (64 bits).

Tolerances, from the formulas:
* indices and codes are equal.  A weight or score is one rounding to fp32 of a number of 64 bits: 2^-24 of it, and 1e-12 for the
  64-bit arithmetic (a few operations of 2^-53, a sum of at most 1024 of them).
* matmul: the sum is exact; its conversion, two products and the bias's addition are four roundings of 2^-24 each of what they round, and
  the output's type adds half a step: 2^-8 (bf16), 2^-11 (fp16), 2^-24 (fp32) of the result, below 2^-14 half of 2^-24 for fp16.
* moe_ffn: beside those, the intermediate h reaches the quantiser with a relative error eps of 2^-16:
  fp32 sums, scales and the sigmoid (an exponential of arguments up to 64: 2^-18, the rest an order less).  Its scale moves by as
  much, so h / scale moves by up to 2 eps |h| / scale of a step: a code flips with that probability, by one step, and
  what it stands for drifts by eps of itself.  Codes flip independently of each other: an output's deviation is the drift, eps of
  each pair's output, and a sum over the F codes of independent terms, each 0 or one step times a weight.  Often there are
  none or a few flips in a row, so the sum is no Gaussian one; Bernstein's inequality holds for any number of them: beyond
  M L / 3 + sqrt((M L / 3)^2 + 2 L V) with a chance of 2 exp(-L) at most, V the sum of the variances, M the largest term.
  L = ln(1e9), a chance of 2e-9 an output.  And over the outputs of a hundred tokens or more, hundreds of flips, the mean square of
  the deviations is what the variances say: at most four times it.
  With bf16 outputs a call of many pairs rounds each pair's output to fp16 before the sum over the slots, scaled so that the
  largest sum there can be, 127 * 127 * F steps of the intermediate times the largest channel scale, is 2^15: half a step is 2^-11
  of the pair's output, or, below 2^-14, 2^-25 on that scale, 2^-40 of the largest sum (int8_oracle.moe_ffn's last result).
"""
import math

import numpy as np
import pytest
import torch

from oracle import int8_oracle as Q
from paper_2603_19172_amd import binding as B
from paper_2603_19172_amd.layer import Int8Experts, Int8MoELayer
from gpu_helpers import DEV

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LOWEST = {t: torch.finfo(t).min for t in HALF}
OUT = {torch.bfloat16: B.OUT_BF16, torch.float16: B.OUT_F16, torch.float32: B.OUT_F32}
EPS_H = 2.0 ** -16


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    c.close()


def f64(t):
    return t.detach().double().cpu().numpy()


def randn(seed, *shape, dtype=torch.bfloat16, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).to(DEV)


# ------------------------------------------------------------------------------------------------------------------ routing

def check_route(ctx, logits, k, bias=None, **kw):
    T, E = logits.shape
    scores = torch.full((T, E), 7.0, device=DEV)
    idx, w = ctx.route_scored(logits, k, bias=bias, scores=scores, **kw)
    torch.cuda.synchronize()
    score = kw.pop("score", B.SCORE_SIGMOID)
    ridx, rw, rs = Q.route_scored(f64(logits), k, None if bias is None else f64(bias), sigmoid=score == B.SCORE_SIGMOID,
                                  lowest=LOWEST[logits.dtype], **kw)
    number = ~np.isnan(rw[:, 0])                   # (a token whose weights are NaN has k different indices, any)
    assert np.array_equal(idx.cpu().numpy()[number], ridx[number])
    for got, ref in ((f64(w), rw), (f64(scores), rs)):
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        ok = ~np.isnan(ref)
        assert (np.abs(got - ref)[ok] <= (2.0 ** -24 + 1e-12) * np.abs(ref)[ok] + 2.0 ** -149).all()
    return idx, w


@pytest.mark.parametrize("T,E,k,groups,top,best", [(1, 1, 1, 1, 1, 1), (1, 256, 8, 8, 4, 2), (5, 7, 7, 1, 1, 1), (67, 64, 6, 1, 1, 1),
                                                   (33, 65, 3, 13, 5, 1), (130, 128, 8, 4, 2, 2), (9, 440, 10, 8, 7, 2),
                                                   (4, 1024, 64, 64, 9, 2), (3, 512, 2, 2, 1, 1), (6, 24, 3, 24, 5, 2), (2, 1000, 12, 1, 1, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("score", [B.SCORE_SIGMOID, B.SCORE_SOFTMAX])
def test_route_matches_the_oracle(ctx, T, E, k, groups, top, best, dtype, score):
    logits = randn(E + k, T, E, dtype=dtype, std=2.0)
    bias = randn(E, E, dtype=torch.float32, std=0.1)
    for b in (bias, None):
        for renorm, factor in ((True, 1.0), (False, 2.5)):
            check_route(ctx, logits, k, b, score=score, groups=groups, top_groups=top, group_best=best, renorm=renorm, factor=factor)


@pytest.mark.parametrize("groups,top,best", [(1, 1, 1), (4, 2, 1), (4, 2, 2), (4, 4, 2)])
@pytest.mark.parametrize("score", [B.SCORE_SIGMOID, B.SCORE_SOFTMAX])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_route_ties_masks_and_what_is_no_number(ctx, groups, top, best, score, dtype):
    E, k = 80, 6
    rows = [torch.zeros(E), torch.zeros(E).index_fill(0, torch.arange(0, E, 2), -0.0), torch.full((E,), -math.inf), torch.full((E,), LOWEST[dtype]),
            torch.arange(E) % 3 * 1.0, torch.full((E,), -300.0), torch.linspace(-400, 400, E)]
    few = torch.full((E,), -math.inf)
    few[[3, 41, 42]] = torch.tensor([0.5, -2.0, 1.0])
    rows += [few, torch.where(few > -math.inf, few, torch.tensor(LOWEST[dtype]))]
    one = torch.randn(E, generator=torch.Generator().manual_seed(1))
    for v in (math.nan, math.inf, -math.inf):
        r = one.clone()
        r[[5, 60]] = v
        rows.append(r)
    rows.append(torch.full((E,), math.nan))
    logits = torch.stack(rows).to(dtype).to(DEV)
    near = torch.zeros(E)
    near[::7] = 2.0 ** -40                       # apart by less than 32 bits tell
    for bias in (None, torch.zeros(E, device=DEV), near.to(DEV), randn(3, E, dtype=torch.float32, std=0.01)):
        for renorm in (True, False):
            idx, _ = check_route(ctx, logits, k, bias, score=score, groups=groups, top_groups=top, group_best=best, renorm=renorm)
            i = idx.cpu().numpy()
            assert ((i >= 0) & (i < E)).all() and all(len(set(r)) == k for r in i.tolist())


def test_route_order_below_32_bits(ctx):
    """Biases that 64 bits tell apart and 32 do not, against scores of one value."""
    E = 256
    logits = torch.zeros((3, E), device=DEV)
    bias = (torch.randperm(E, generator=torch.Generator().manual_seed(0)).float() * 2.0 ** -60).to(DEV) + 0.0
    check_route(ctx, logits + 40.0, 9, bias)     # 1 - 4e-18 rounds to 1: all alike, lowest indices
    check_route(ctx, logits, 9, bias * 2.0 ** 12)
    check_route(ctx, logits, 9, bias * 2.0 ** 12, groups=8, top_groups=3, group_best=2)


def test_route_leaves_rows_behind_the_last(ctx):
    T, E, k = 5, 60, 4
    logits = randn(1, T, E, dtype=torch.float32)
    idx = torch.full((T + 3, k), 99, dtype=torch.int32, device=DEV)
    w = torch.full((T + 3, k), 99.0, device=DEV)
    ctx.route_scored(logits, k, idx=idx[:T], w=w[:T])
    ctx.route_scored(logits[:0], k, idx=idx[:0], w=w[:0])
    assert (idx[T:] == 99).all() and (w[T:] == 99).all() and (idx[:T] < E).all()


# ------------------------------------------------------------------------------------------------------------------ rows

def row_inputs(seed, rows, K, dtype):
    x = randn(seed, rows, K, dtype=torch.float32)
    if rows > 1:
        x[1] = 0
    if rows > 2:
        x[2] *= 2.0 ** -20
    if rows > 4:
        x[3, K // 2] = math.inf
        x[4, 0] = math.nan
    if rows > 6:
        # every code and every tie: whole and half steps of a largest value of 127
        x[5] = (torch.arange(K) % 509 - 254).to(DEV) / 2.0
        x[5, 0] = 127.0
        x[6] = torch.arange(K).to(DEV) % 2 * 2.0 - 1.0
    return x.to(dtype)


@pytest.mark.parametrize("rows,K", [(1, 1), (7, 3), (5, 64), (33, 127), (8, 128), (9, 129), (7, 513), (70, 1000), (7, 2050), (11, 4096),
                                    (9, 4097), (7, 8200), (3, 14336), (2, 16390), (7, 40000), (1, 70001), (8, 131072), (4100, 130), (4100, 700), (4100, 1500), (4100, 2500)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_codes_are_those_of_the_oracle(ctx, rows, K, dtype):
    x = row_inputs(rows + K, rows, K, dtype)
    codes, scale = ctx.quantize_rows(x)
    tiled, scale2 = ctx.quantize_rows(x, layout=B.LAYOUT_TILE)
    c, s = Q.quantize_rows(f64(x))
    got = codes.cpu().numpy()
    assert np.array_equal(got[:, :K], c) and (got[:, K:] == 0).all()
    assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True) and np.array_equal(scale2.cpu().numpy(), s, equal_nan=True)
    assert np.array_equal(tiled.cpu().numpy(), Q.tiles(c))


def test_rows_of_32_bits(ctx):
    x = row_inputs(5, 40, 3001, torch.float32)
    x[7] *= 1e38
    x[8] *= 1e-38
    x[9] *= 1e-44
    codes, scale = ctx.quantize_rows(x)
    c, s = Q.quantize_rows(f64(x))
    got = codes.cpu().numpy()[:, :3001]
    assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True)
    # a quotient right to its last bit is within 2^-23 of itself (127 x and its quotient round once each): another code only there
    v = f64(x)
    peak = np.abs(v).max(axis=1, keepdims=True)
    with np.errstate(all="ignore"):
        q = 127.0 * v / peak
    near = np.abs(np.abs(q - np.trunc(q)) - 0.5) <= 127 * 2.0 ** -23
    assert ((got == c) | (near & (np.abs(got.astype(int) - c) == 1)))[np.isfinite(peak[:, 0]) & (peak[:, 0] > 0)].all()
    assert (got[~np.isfinite(peak[:, 0])] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_at_the_ends_of_the_types_range(ctx, dtype):
    """Every value of the type beside a largest one of its range's two ends and its middle."""
    bits = torch.arange(-(1 << 15), 1 << 15, dtype=torch.int32).to(torch.int16).view(dtype)
    v = bits[torch.isfinite(bits)]
    fi = torch.finfo(dtype)
    rows = []
    for peak in (fi.max, 1.0, 1.9921875, fi.tiny, fi.smallest_normal * 3, float(v[v > 0].min()), float(v[v > 0].min()) * 5):
        p = torch.tensor(peak).to(dtype)
        r = torch.where(v.abs().float() <= p.float(), v, torch.zeros((), dtype=dtype))
        r[0] = p
        rows.append(r)
    x = torch.stack(rows).to(DEV)
    codes, scale = ctx.quantize_rows(x)
    c, s = Q.quantize_rows(f64(x))
    assert np.array_equal(codes.cpu().numpy()[:, :x.shape[1]], c) and np.array_equal(scale.cpu().numpy(), s)


@pytest.mark.parametrize("K,pitch,off", [(100, 101, 1), (257, 300, 3), (1024, 1031, 5), (64, 64, 1)])
def test_rows_apart_and_unaligned(ctx, K, pitch, off):
    rows = 6
    flat = randn(K, rows * pitch + off)
    x = flat[off:off + rows * pitch].view(rows, pitch)[:, :K]
    out = (torch.full((rows + 2, -(-K // 128) * 128), 55, dtype=torch.int8, device=DEV), torch.full((rows + 2,), 5.0, device=DEV))
    ctx.quantize_rows(x, out=(out[0][:rows], out[1][:rows]))
    c, s = Q.quantize_rows(f64(x))
    assert np.array_equal(out[0].cpu().numpy()[:rows, :K], c) and np.array_equal(out[1].cpu().numpy()[:rows], s)
    assert (out[0][rows:] == 55).all() and (out[1][rows:] == 5).all()


# ------------------------------------------------------------------------------------------------------------------ product

@pytest.mark.parametrize("layout", [B.LAYOUT_ROWMAJOR, B.LAYOUT_TILE])
def test_rows_of_more_than_one_launch(ctx, layout):
    rows, K = (1 << 21) + 37, 5
    x = randn(8, rows, K)
    codes, scale = ctx.quantize_rows(x, layout=layout)
    cut = (1 << 21) - 64                             # both sides of the launches' border
    want, ws = Q.quantize_rows(f64(x[cut:]))
    if layout == B.LAYOUT_TILE:
        want = Q.tiles(want)
    else:
        want = np.pad(want, ((0, 0), (0, 128 - K)))
    assert np.array_equal(codes[cut:].cpu().numpy().reshape(want.shape), want)
    assert np.array_equal(scale[cut:].cpu().numpy(), ws.astype(np.float32))
    peak = x.double().abs().amax(1) / 127.0          # (scale: that, rounded once)
    assert ((scale.double() - peak).abs() <= 2.0 ** -24 * peak).all() and torch.equal(codes[:64], ctx.quantize_rows(x[:64], layout=layout)[0])


def matmul_bound(prod, y, dtype):
    return 4 * 2.0 ** -24 * np.abs(prod) + (HALF[dtype] + 2 * 2.0 ** -24) * np.abs(y) + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def weight(ctx, seed, N, K):
    w = randn(seed, N, K, std=0.05)
    return ctx.quantize_rows(w, layout=B.LAYOUT_TILE), Q.quantize_rows(f64(w))


SIZES = [(1, 1, 1), (1, 64, 128), (1, 4096, 4096), (1, 100, 14336), (2, 33, 129), (3, 200, 1000), (5, 31, 300), (8, 512, 640), (16, 1000, 257),
         (17, 96, 2048), (31, 65, 77), (32, 64, 4224), (33, 160, 384), (61, 1536, 2048), (64, 520, 128), (65, 130, 1100), (127, 300, 640),
         (128, 256, 256), (129, 257, 1408), (200, 1030, 520), (256, 512, 1024), (300, 700, 2000), (513, 770, 900), (1030, 300, 450)]


@pytest.mark.parametrize("T,N,K", SIZES)
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32, torch.float16])
def test_matmul_matches_the_oracle(ctx, T, N, K, out):
    wt, (wq, ws) = weight(ctx, N, N, K)
    x = randn(T + K, T, K, dtype=torch.float16 if out == torch.float16 else torch.bfloat16)
    bias = randn(7, N, dtype=torch.float32)
    xq, xs = Q.quantize_rows(f64(x))
    prod = Q.matmul(xq, xs, wq, ws)
    for b in (None, bias):
        y = ctx.matmul_int8(x, wt, bias=b, out_dtype=OUT[out])
        ref = prod if b is None else prod + f64(b)
        assert y.dtype == out
        assert (np.abs(f64(y) - ref) <= matmul_bound(prod, ref, out)).all()
    # codes made beforehand give the same bits
    assert torch.equal(y, ctx.matmul_int8(*ctx.quantize_rows(x)[:1], wt, x_scale=ctx.quantize_rows(x)[1], bias=bias, out_dtype=OUT[out]))


@pytest.mark.parametrize("T", [1, 3, 40, 150, 600])
def test_matmul_extreme_sums_are_exact(ctx, T):
    """All codes at their ends: the largest sums there are, and their cancellation."""
    N, K = 70, 131072 if T < 100 else 8192
    x = torch.ones((T, K), dtype=torch.bfloat16, device=DEV)
    x[:, 1::2] *= -1 if T == 3 else 1
    w = torch.ones((N, K), dtype=torch.bfloat16, device=DEV)
    w[1] = -1
    wt = ctx.quantize_rows(w, layout=B.LAYOUT_TILE)
    y = ctx.matmul_int8(x, wt, out_dtype=B.OUT_F32)
    whole = 0 if T == 3 else 127 * 127 * K
    ref = np.full((T, N), float(whole)) * np.float64(np.float32(1) / np.float32(127)) ** 2
    ref[:, 1] *= -1
    assert (np.abs(f64(y) - ref) <= 3 * 2.0 ** -24 * np.abs(ref)).all()


@pytest.mark.parametrize("T,N,K", [(1, 100, 300), (5, 100, 300), (40, 77, 200), (140, 300, 260), (300, 290, 500)])
def test_matmul_strided_rows_and_what_lies_between(ctx, T, N, K):
    wt, (wq, ws) = weight(ctx, N, N, K)
    flat = randn(T, T * (K + 5) + 3)
    x = flat[3:].view(T, K + 5)[:, :K]
    for out, gap in ((torch.bfloat16, 3), (torch.bfloat16, 8), (torch.float32, 1), (torch.float16, 7)):
        y = torch.full((T + 2, N + gap), 77.0, dtype=out, device=DEV)
        ctx.matmul_int8(x, wt, y=y[:T, :N])
        xq, xs = Q.quantize_rows(f64(x))
        prod = Q.matmul(xq, xs, wq, ws)
        assert (np.abs(f64(y[:T, :N]) - prod) <= matmul_bound(prod, prod, out)).all()
        assert (y[T:] == 77).all() and (y[:, N:] == 77).all()


@pytest.mark.parametrize("T", [1, 4, 16, 20, 64, 130, 260])
def test_matmul_row_that_is_no_number_stays_alone(ctx, T):
    wt, _ = weight(ctx, 3, 300, 500)
    x = randn(T, T, 500)
    clean = ctx.matmul_int8(x, wt)
    x2 = x.clone()
    x2[T // 2, 7] = math.nan
    x2[T - 1, 3] = math.inf
    y = ctx.matmul_int8(x2, wt)
    hit = torch.zeros(T, dtype=torch.bool, device=DEV)
    hit[[T // 2, T - 1]] = True
    assert torch.isnan(y[hit]).all() and torch.equal(y[~hit], clean[~hit])


def test_matmul_rows_do_not_depend_on_their_company(ctx):
    wt, _ = weight(ctx, 5, 520, 1200)
    x = randn(5, 700, 1200)
    y = ctx.matmul_int8(x, wt)
    for lo, hi in ((0, 1), (3, 8), (100, 117), (200, 260), (0, 130), (1, 400)):
        assert torch.equal(ctx.matmul_int8(x[lo:hi], wt), y[lo:hi])


@pytest.mark.parametrize("N,K", [(520, 1200), (4100, 2100)])
def test_matmul_rows_with_a_bias_do_not_depend_on_their_company(ctx, N, K):
    """The bias's addition is rounded alike in every shape the product is computed in."""
    T = 2500
    wt, _ = weight(ctx, 6, N, K)
    x, bias = randn(6, T, K), randn(7, N, dtype=torch.float32)
    y = ctx.matmul_int8(x, wt, bias=bias, out_dtype=B.OUT_F32)
    for lo, hi in ((0, 1), (3, 8), (100, 117), (200, 260), (0, 130), (1, 400), (300, 1700)):
        assert torch.equal(ctx.matmul_int8(x[lo:hi], wt, bias=bias, out_dtype=B.OUT_F32), y[lo:hi])


@pytest.mark.parametrize("T", [1, 8, 12, 16, 40])
def test_matmul_many_outputs(ctx, T):
    """Wider matrices than the shapes of a few rows are for from nine rows on."""
    N, K = 90001, 130
    wt, (wq, ws) = weight(ctx, T, N, K)
    x, bias = randn(T, T, K), randn(T + 1, N, dtype=torch.float32)
    y = f64(ctx.matmul_int8(x, wt, bias=bias, out_dtype=B.OUT_F32))
    xq, xs = Q.quantize_rows(f64(x))
    prod = Q.matmul(xq, xs, wq, ws)
    want = prod + f64(bias)
    assert (np.abs(y - want) <= matmul_bound(prod, want, torch.float32)).all()


# ------------------------------------------------------------------------------------------------------------------ experts

def make_experts(ctx, seed, E, H, F, absent=()):
    dev, host = [], []
    for e in range(E):
        if e in absent:
            dev.append(None)
            host.append(None)
            continue
        mats = [randn(seed * 1000 + 3 * e + i, *s, std=0.05) for i, s in enumerate(((F, H), (F, H), (H, F)))]
        dev.append([ctx.quantize_rows(m, layout=B.LAYOUT_TILE) for m in mats])
        host.append([Q.quantize_rows(f64(m)) for m in mats])
    return dev, host


def routing(seed, T, E, k, popular=0.0):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn((T, E), generator=g) - popular * torch.log(torch.arange(E) + 1.0)
    top = l.softmax(-1).topk(k, dim=-1)
    return top.indices.to(torch.int32).to(DEV), (top.values / top.values.sum(-1, keepdim=True)).to(DEV)


def check_ffn(ctx, x, idx, gate, dev, host, F, out=torch.bfloat16, table=None):
    T, H = x.shape
    table = B.make_int8_table(dev, DEV) if table is None else table
    ws = torch.full((B.moe_ffn_int8_workspace_bytes(T, H, F, len(dev), idx.shape[1]),), 0xFF, dtype=torch.uint8, device=DEV)
    y = torch.full((T + 2, H), 77.0, dtype=out, device=DEV)
    ctx.moe_ffn_int8(x, idx, gate, table, F, y=y[:T], workspace=ws)
    torch.cuda.synchronize()
    ref, dev_tol, square, half = Q.moe_ffn(f64(x), idx.cpu().numpy(), f64(gate), host, EPS_H)
    if out == torch.bfloat16:
        dev_tol, square = dev_tol + half, square + half ** 2
    got = f64(y[:T])
    # sums over k slots of fp32 products, and the output's type
    k = idx.shape[1]
    tol = dev_tol + HALF[out] * (np.abs(ref) + dev_tol) + (k + 6) * 2.0 ** -24 * (np.abs(ref) + dev_tol) + 2.0 ** -24 * np.abs(ref).max() + (2.0 ** -25 if out == torch.float16 else 0)
    assert np.isfinite(got).all()
    worst = (np.abs(got - ref) / np.maximum(tol, 1e-300)).max() if got.size else 0.0
    print("T=%d H=%d F=%d: worst %.2f of the bound" % (T, H, F, worst), flush=True)
    assert worst <= 1.0
    if T >= 100:
        rounding = HALF[out] * np.abs(ref) + (k + 6) * 2.0 ** -24 * np.abs(ref) + 2.0 ** -24 * np.abs(ref).max()
        assert ((got - ref) ** 2).sum() <= 4.0 * (square + rounding ** 2).sum()
    assert (y[T:] == 77).all()
    return y[:T]


FFN = [(1, 256, 512, 8, 2), (1, 100, 60, 4, 1), (2, 200, 392, 8, 8), (3, 512, 1000, 16, 4), (4, 136, 72, 128, 8), (5, 300, 500, 8, 2), (8, 256, 640, 60, 6),
       (16, 256, 512, 8, 2), (16, 128, 128, 8, 8), (17, 640, 264, 8, 2), (33, 129, 131, 8, 3), (61, 256, 96, 128, 8), (64, 384, 512, 4, 2), (150, 200, 136, 8, 2),
       (300, 264, 520, 8, 2), (520, 136, 200, 2, 1), (700, 128, 257, 4, 4)]


@pytest.mark.parametrize("T,H,F,E,k", FFN)
def test_ffn_matches_the_oracle(ctx, T, H, F, E, k):
    dev, host = make_experts(ctx, T, E, H, F)
    idx, gate = routing(T, T, E, k)
    x = randn(T, T, H)
    a = check_ffn(ctx, x, idx, gate, dev, host, F)
    b = check_ffn(ctx, x, idx, gate, dev, host, F)
    assert torch.equal(a, b)                       # the same bits from call to call


@pytest.mark.parametrize("T", [1, 7, 40, 200])
@pytest.mark.parametrize("xt,out", [(torch.float16, torch.float16), (torch.float32, torch.float32), (torch.bfloat16, torch.float32)])
def test_ffn_types(ctx, T, xt, out):
    dev, host = make_experts(ctx, 11, 8, 200, 328)
    idx, gate = routing(T, T, 8, 2)
    check_ffn(ctx, randn(T, T, 200, dtype=xt), idx, gate, dev, host, 328, out=out)


@pytest.mark.parametrize("T", [1, 3, 12, 50, 400])
def test_ffn_all_tokens_on_one_expert_and_on_none(ctx, T):
    dev, host = make_experts(ctx, 12, 8, 256, 320)
    x = randn(T, T, 256)
    one = torch.full((T, 1), 5, dtype=torch.int32, device=DEV)
    g = torch.ones((T, 1), device=DEV)
    check_ffn(ctx, x, one, g, dev, host, 320)
    for bad in (-1, 8, 1 << 30, -(1 << 31)):
        y = check_ffn(ctx, x, torch.full((T, 1), bad, dtype=torch.int32, device=DEV), g, dev, host, 320)
        assert (y == 0).all()
    # the same expert in two slots of a token
    check_ffn(ctx, x, torch.full((T, 2), 3, dtype=torch.int32, device=DEV), torch.cat([g * 0.25, g * -2.0], 1), dev, host, 320)


@pytest.mark.parametrize("T", [1, 4, 16, 70, 300])
def test_ffn_left_out_pairs_and_absent_experts(ctx, T):
    assert ctx.device_flags() == 0
    dev, host = make_experts(ctx, 13, 9, 192, 256, absent=(2, 7))
    idx, gate = routing(T, T, 9, 3)
    idx[T // 2, 1] = -1
    idx[0, 0] = 9
    idx[T - 1, 2] = 7
    check_ffn(ctx, randn(T, T, 192), idx, gate, dev, host, 256)
    assert ctx.device_flags() == B.FLAG_FORMAT_MISSING and ctx.device_flags() == 0


@pytest.mark.parametrize("T", [2, 6, 16, 90, 300])
def test_ffn_token_that_is_no_number_stays_alone(ctx, T):
    dev, host = make_experts(ctx, 14, 4, 160, 224)
    table = B.make_int8_table(dev, DEV)
    idx, gate = routing(T, T, 4, 2)
    x = randn(T, T, 160)
    clean = ctx.moe_ffn_int8(x, idx, gate, table, 224)
    x[T // 2, 3] = math.nan
    y = ctx.moe_ffn_int8(x, idx, gate, table, 224)
    rest = torch.arange(T, device=DEV) != T // 2
    assert torch.isnan(y[T // 2]).all() and torch.equal(y[rest], clean[rest])


@pytest.mark.parametrize("T,k", [(1, 64), (2, 32), (1, 65), (2, 33), (3, 20), (40, 16)])
@pytest.mark.parametrize("same", [False, True])
def test_ffn_many_slots_and_the_same_expert_in_several(ctx, T, k, same):
    E, H, F = 70, 136, 72
    dev, host = make_experts(ctx, 31, E, H, F)
    g = torch.Generator().manual_seed(T + k)
    idx = torch.randint(0, 3, (T, k), generator=g) if same else torch.rand((T, E), generator=g).argsort(1)[:, :k]
    gate = torch.rand((T, k), generator=g).float().to(DEV) / k
    check_ffn(ctx, randn(T * k, T, H), idx.to(torch.int32).to(DEV), gate, dev, host, F)


def test_ffn_skewed_load(ctx):
    dev, host = make_experts(ctx, 15, 32, 128, 96)
    idx, gate = routing(1, 400, 32, 4, popular=1.5)
    check_ffn(ctx, randn(1, 400, 128), idx, gate, dev, host, 96)


def test_ffn_rows_longer_than_the_first_launch_takes(ctx):
    """Activations whose codes are a launch of their own."""
    dev, host = make_experts(ctx, 21, 2, 16500, 40)
    for T in (1, 20, 40):
        idx, gate = routing(T, T, 2, 1)
        check_ffn(ctx, randn(T, T, 16500), idx, gate, dev, host, 40)


@pytest.mark.parametrize("T,E,k,popular", [(2100, 8, 8, 0.0), (5000, 40, 4, 1.0)])
def test_ffn_more_pairs_than_a_plan_holds_in_lds(ctx, T, E, k, popular):
    dev, host = make_experts(ctx, 22, E, 64, 32)
    idx, gate = routing(3, T, E, k, popular)
    check_ffn(ctx, randn(4, T, 64), idx, gate, dev, host, 32)


def test_ffn_more_tiles_than_a_plan_holds_in_lds(ctx):
    """Rows are the same bits as in a call of their own size's kernels, whatever rows they stand among."""
    T, H, F, E, k, part = 66000, 40, 24, 8, 8, 8000
    dev, _ = make_experts(ctx, 23, E, H, F)
    table = B.make_int8_table(dev, DEV)
    idx, gate = routing(5, T, E, k)
    x = randn(6, T, H)
    whole = ctx.moe_ffn_int8(x, idx, gate, table, F)
    for lo in range(0, T, part):
        hi = min(T, lo + part)
        assert torch.equal(ctx.moe_ffn_int8(x[lo:hi], idx[lo:hi], gate[lo:hi], table, F), whole[lo:hi])


@pytest.mark.parametrize("T", [3, 40, 300])
def test_ffn_weights_at_the_ends_of_the_range(ctx, T):
    """Scales that are tiny, zero, and NaN: a channel of W2 that is no number is that output, and no other."""
    E, H, F = 2, 96, 64
    mats = [[randn(50 + 3 * e + i, *s, std=0.05) for i, s in enumerate(((F, H), (F, H), (H, F)))] for e in range(E)]
    mats[0][2][5] = 0
    mats[0][2][40:] *= 2.0 ** -126
    mats[1][2][64:] = 0
    dev = [[ctx.quantize_rows(m, layout=B.LAYOUT_TILE) for m in ex] for ex in mats]
    host = [[Q.quantize_rows(f64(m)) for m in ex] for ex in mats]
    idx, gate = routing(T, T, E, 2)
    x = randn(T, T, H)
    clean = check_ffn(ctx, x, idx, gate, dev, host, F).clone()
    mats[1][2][7, 3] = math.inf
    dev[1][2] = ctx.quantize_rows(mats[1][2], layout=B.LAYOUT_TILE)
    y = ctx.moe_ffn_int8(x, idx, gate, B.make_int8_table(dev, DEV), F)
    rest = torch.arange(H, device=DEV) != 7
    assert torch.isnan(y[:, 7]).all() and torch.equal(y[:, rest], clean[:, rest])


@pytest.mark.parametrize("T,spread", [(40, 40), (300, 9), (300, 40), (700, 100)])
def test_ffn_channels_far_apart(ctx, T, spread):
    """Neighbouring channels of W2 whose scales lie up to 2^spread apart: each is as exact as it would be alone.  The rounding of a pair's output to
    fp16 is half a step of 2^-11 of it, or half of the least step: of sums scaled so that 127 * 127 * F steps of the intermediate are 2^15,
    times a channel's share of its strip's largest scale where that is 2^-8 or more and one where it is less, 2^-25; so
    2^-25 * 127 * 127 * F * 2^-15 * 2^8 steps of the intermediate times the channel's own scale at most."""
    E, H, F, k = 2, 168, 264, 2
    g = torch.Generator().manual_seed(T + spread)
    mats = [[randn(90 + 3 * e + i, *s, std=0.05) for i, s in enumerate(((F, H), (F, H), (H, F)))] for e in range(E)]
    for e in range(E):
        down = torch.randint(0, spread + 1, (H, 1), generator=g)
        down[64:96] = 3                              # (a strip of equal channels beside the others)
        mats[e][2] = (mats[e][2].float() * (0.5 ** down.double()).float().to(DEV)).to(torch.bfloat16)
    mats[0][2][33] = 0
    dev = [[ctx.quantize_rows(m, layout=B.LAYOUT_TILE) for m in ex] for ex in mats]
    host = [[Q.quantize_rows(f64(m)) for m in ex] for ex in mats]
    idx, gate = routing(T, T, E, k)
    idx[: T // 8, 1] = -1
    x = randn(T, T, H)
    y = f64(ctx.moe_ffn_int8(x, idx, gate, B.make_int8_table(dev, DEV), F))
    ix = idx.cpu().numpy()
    ref, bound, _, _ = Q.moe_ffn(f64(x), ix, f64(gate), host, EPS_H)
    size = sum(np.abs(Q.moe_ffn(f64(x), ix[:, j:j + 1], f64(gate)[:, j:j + 1], host, 0.0)[0]) for j in range(k))
    least = np.zeros_like(ref)
    for t in range(T):
        for j in range(k):
            if ix[t, j] >= 0:
                (q1, s1), (q3, s3), (q2, s2) = host[ix[t, j]]
                xq, xs = Q.quantize_rows(f64(x[t:t + 1]))
                a, u = (Q.matmul(xq, xs, q, s)[0] for q, s in ((q1, s1), (q3, s3)))
                step = np.abs(a / (1.0 + np.exp(-a)) * u).max() / 127.0
                least[t] += abs(float(gate[t, j])) * 2.0 ** -32 * 127 * 127 * F * step * s2
    tol = bound + 2.0 ** -11 * size + least + HALF[torch.bfloat16] * (np.abs(ref) + bound) + (k + 6) * 2.0 ** -24 * (size + bound)
    assert (np.abs(y - ref) <= tol).all()
    assert (y[:, 64:96] != 0).all()


@pytest.mark.parametrize("T", [200, 400])
def test_ffn_tall_and_wide_tiles_side_by_side(ctx, T):
    """One expert with several tiles of 128 rows, others with a few pairs each; loads on both sides of where the kinds change."""
    E, H, F = 12, 200, 264
    dev, host = make_experts(ctx, 24, E, H, F)
    for n in (160, 161, 128, 129, 33, T):
        idx = torch.stack([torch.arange(T) % (E - 1) + 1, torch.where(torch.arange(T) < n, 0, -1)], 1).to(torch.int32).to(DEV)
        check_ffn(ctx, randn(T + n, T, H), idx, torch.full((T, 2), 0.5, device=DEV), dev, host, F)


# ------------------------------------------------------------------------------------------------------------------ as they are used

@pytest.mark.parametrize("T", [1, 9, 50, 300])
def test_router_and_experts_together_on_another_stream_and_in_a_graph(ctx, T):
    """Logits from an integer product, the selection, the experts: eager on a stream of its own, then captured once and replayed on
    changing inputs with eager work between the replays."""
    H, F, E, k = 256, 384, 16, 4
    dev, host = make_experts(ctx, 16, E, H, F)
    table = B.make_int8_table(dev, DEV)
    router, _ = weight(ctx, 99, E, H)
    bias = randn(98, E, dtype=torch.float32, std=0.05)
    x = randn(T, T, H)
    bufs = dict(l=torch.empty((T, E), device=DEV), i=torch.empty((T, k), dtype=torch.int32, device=DEV), w=torch.empty((T, k), device=DEV),
                y=torch.empty((T, H), dtype=torch.bfloat16, device=DEV),
                a=torch.empty((B.matmul_int8_workspace_bytes(T, E, H),), dtype=torch.uint8, device=DEV),
                b=torch.empty((B.moe_ffn_int8_workspace_bytes(T, H, F, E, k),), dtype=torch.uint8, device=DEV))

    def step(x, bufs):
        ctx.matmul_int8(x, router, y=bufs["l"], workspace=bufs["a"])
        ctx.route_scored(bufs["l"], k, bias=bias, groups=4, top_groups=2, group_best=2, idx=bufs["i"], w=bufs["w"])
        return ctx.moe_ffn_int8(x, bufs["i"], bufs["w"], table, F, y=bufs["y"], workspace=bufs["b"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = step(x, bufs).clone()
    torch.cuda.synchronize()
    ridx, rw, _ = Q.route_scored(f64(bufs["l"]), k, f64(bias), groups=4, top_groups=2, group_best=2)
    assert np.array_equal(bufs["i"].cpu().numpy(), ridx)
    check_ffn(ctx, x, bufs["i"], bufs["w"], dev, host, F, table=table)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(x, bufs)
    eager = {n: torch.empty_like(v) for n, v in bufs.items()}
    for r in range(4):
        x.copy_(randn(100 + r, T, H))
        bufs["b"].fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        got = bufs["y"].clone()
        assert torch.equal(got, step(x, eager))
        assert r > 0 or not torch.equal(got, first)


@pytest.mark.parametrize("T", [1, 33, 260])
def test_layer_class_is_its_calls(ctx, T):
    H, F, E, k = 192, 256, 16, 4
    mats = [[randn(700 + 3 * e + i, *s, std=0.05) for i, s in enumerate(((F, H), (F, H), (H, F)))] for e in range(E)]
    mats[3] = None
    experts = Int8Experts(ctx, mats, DEV)
    router = ctx.quantize_rows(randn(69, E, H, std=0.1), layout=B.LAYOUT_TILE)
    bias = randn(68, E, dtype=torch.float32, std=0.05)
    x = randn(T, T, H)
    layer = Int8MoELayer(ctx, T, H, F, E, k, groups=4, top_groups=2, group_best=2, factor=2.5)
    y = layer.step(x, experts, router=router, bias=bias)
    logits = ctx.matmul_int8(x, router, out_dtype=B.OUT_F32)
    idx, w = ctx.route_scored(logits, k, bias=bias, groups=4, top_groups=2, group_best=2, factor=2.5)
    assert torch.equal(layer.idx, idx) and torch.equal(layer.gate, w)
    assert torch.equal(y, ctx.moe_ffn_int8(x, idx, w, experts.table, F))
    assert torch.equal(layer.step(x, experts, logits=logits, bias=bias), y)
    assert ctx.device_flags() in (0, B.FLAG_FORMAT_MISSING)


def test_two_calls_at_once_on_two_streams(ctx):
    """Workspaces of their own: nothing else is shared."""
    H, F, E, k, T = 256, 512, 8, 2, 300
    dev, _ = make_experts(ctx, 25, E, H, F)
    table = B.make_int8_table(dev, DEV)
    wt, _ = weight(ctx, 26, 400, H)
    x = randn(27, T, H)
    idx, gate = routing(28, T, E, k)
    ref = ctx.moe_ffn_int8(x, idx, gate, table, F), ctx.matmul_int8(x, wt)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(5):
        with torch.cuda.stream(a):
            y = ctx.moe_ffn_int8(x, idx, gate, table, F)
        with torch.cuda.stream(b):
            z = ctx.matmul_int8(x, wt)
        got.append((y, z))
    torch.cuda.synchronize()
    for y, z in got:
        assert torch.equal(y, ref[0]) and torch.equal(z, ref[1])


@pytest.mark.parametrize("handle", [False, True])
def test_memory_of_a_call_belongs_to_its_stream(ctx, monkeypatch, handle):
    """What a call on another stream allocates is not given to the current stream's work before the call has run."""
    x = randn(3, 200, 512)
    wt, _ = weight(ctx, 9, 300, 512)
    dev, _ = make_experts(ctx, 9, 4, 512, 256)
    table = B.make_int8_table(dev, DEV)
    idx, gate = routing(9, 200, 4, 2)
    want = ctx.matmul_int8(x, wt), ctx.moe_ffn_int8(x, idx, gate, table, 256)
    taken, at = [], B._at
    monkeypatch.setattr(B, "_at", lambda t, *a: (taken.append((t.data_ptr(), t.numel())) if t is not None and t.dtype is torch.uint8 and t is not table else None) or at(t, *a))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    stream = s.cuda_stream if handle else s
    got = ctx.matmul_int8(x, wt, stream=stream), ctx.moe_ffn_int8(x, idx, gate, table, 256, stream=stream)
    assert len(taken) == 2
    for ptr, n in taken:
        mine = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(4)]
        assert all(t.data_ptr() != ptr for t in mine)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_scores_feed_the_importance_and_the_mixed_layer(ctx):
    """The router's outputs are what the precision steps take."""
    T, E, k = 3, 16, 4
    logits = randn(1, T, E, dtype=torch.float32)
    scores = torch.empty((T, E), device=DEV)
    idx, w = ctx.route_scored(logits, k, scores=scores)
    imp, load = ctx.expert_importance(B.PHASE_DECODE, idx, E, probs=scores)
    assert np.allclose(f64(imp), f64(scores).mean(axis=0), rtol=1e-6) and int(load.sum()) == T * k
