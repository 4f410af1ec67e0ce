"""GPU tests of the 8-bit integer experts and products across the shapes that a call is computed in: what a shape may not change, and
each shape against the oracle at sizes that reach its steady state.  The bounds are test_gpu_int8's unless a test derives its own."""
import numpy as np
import pytest
import torch

import test_gpu_int8 as G
from oracle import int8_oracle as Q
from paper_2603_19172_amd import binding as B
from paper_2603_19172_amd.layer import Int8Experts, Int8MoELayer
from gpu_helpers import DEV
from test_gpu_int8 import ctx  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 2, 40, 100, 300, 700])
def test_ffn_output_types_round_the_same_sums(ctx, T):  # noqa: F811
    """The sum over the slots is one of 32 bits whatever type it leaves in: 16-bit outputs are the fp32 ones rounded."""
    E, H, F, k = 8, 264, 392, 2
    dev, _ = G.make_experts(ctx, 41, E, H, F)
    table = B.make_int8_table(dev, DEV)
    idx, gate = G.routing(T, T, E, k)
    x = G.randn(T, T, H)
    y = ctx.moe_ffn_int8(x, idx, gate, table, F, out_dtype=B.OUT_F32)
    for t, code in ((torch.bfloat16, B.OUT_BF16), (torch.float16, B.OUT_F16)):
        assert torch.equal(ctx.moe_ffn_int8(x, idx, gate, table, F, out_dtype=code), y.to(t))


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_ffn_rows_do_not_depend_on_their_company(ctx, out):  # noqa: F811
    """Calls of one and two tokens, of few pairs an expert and of many, with tall tiles and with wide ones."""
    E, H, F, k, T = 8, 264, 520, 2, 900
    dev, _ = G.make_experts(ctx, 42, E, H, F)
    table = B.make_int8_table(dev, DEV)
    idx, gate = G.routing(7, T, E, k)
    assert torch.bincount(idx.flatten().long()).max() > 160
    x = G.randn(8, T, H)
    y = ctx.moe_ffn_int8(x, idx, gate, table, F, out_dtype=G.OUT[out])
    for lo, hi in ((0, 1), (5, 6), (3, 5), (10, 13), (20, 50), (100, 170), (0, 300), (200, 860)):
        assert torch.equal(ctx.moe_ffn_int8(x[lo:hi], idx[lo:hi], gate[lo:hi], table, F, out_dtype=G.OUT[out]), y[lo:hi])


@pytest.mark.parametrize("T", [1, 40, 300, 700])
def test_ffn_channel_scales_at_the_large_end(ctx, T):  # noqa: F811
    """Channels of W2 up to 2^127, intermediates of 2^-80: the outputs are ordinary numbers."""
    E, H, F, k = 2, 160, 1000, 2
    mats = [[G.randn(60 + 3 * e + i, *s, std=0.05) for i, s in enumerate(((F, H), (F, H), (H, F)))] for e in range(E)]
    for ex in mats:
        ex[2] = (ex[2].float() * 2.0 ** 64 * 2.0 ** 65).to(torch.bfloat16)
        assert torch.isfinite(ex[2]).all() and ex[2].abs().max() > 2.0 ** 126
    dev = [[ctx.quantize_rows(m, layout=B.LAYOUT_TILE) for m in ex] for ex in mats]
    host = [[Q.quantize_rows(G.f64(m)) for m in ex] for ex in mats]
    idx, gate = G.routing(T, T, E, k)
    G.check_ffn(ctx, G.randn(T, T, H, std=2.0 ** -40), idx, gate, dev, host, F)


SILU_T = [(1, 1), (2, 1), (2, 2), (20, 1), (64, 2), (200, 1), (300, 2), (700, 2)]


@pytest.mark.parametrize("T,E", SILU_T)
def test_ffn_swiglu_is_of_32_bits(ctx, T, E):  # noqa: F811
    """An expert of one feature shows its intermediate: its code is 127 or -127, its scale |h| / 127, and an output 127 |h| times powers
    of two.  Here scales are powers of two too, so a = W1 x and u = W3 x are exact.  In steps of 2^-24 of what they round: exp 2 (1 ulp) and
    its argument's correction 1, 1 + exp 1, the reciprocal 2, exp times it 1, the products with a and u 1 each, h / 127 and its product with
    the sum 1 each: 11 at most, and products of those; 12 allowed."""
    H, F = 128, 1
    for trial in range(1 if T > 8 else 24):
        c = (torch.arange(T) * 37 + 23 * trial) % 161 - 80
        x = torch.zeros((T, H))
        x[:, 0], x[:, 1] = 127, c.float()
        dev = []
        shift = [2.0 ** -(3 * e) for e in range(E)]                # expert e: a = c / 8^e
        for e in range(E):
            w1, w3, w2 = torch.zeros((F, H)), torch.zeros((F, H)), torch.full((H, F), 127 * 2.0 ** -3)
            w1[0, 1], w1[0, 2] = shift[e], 127 * shift[e]           # (x's column 2 is zero: there for the scale)
            w3[0, 0] = 127 * 2.0 ** -14                             # u = 127 * 127 * 2^-14
            w2[1::2] *= -1
            dev.append([ctx.quantize_rows(m.to(DEV), layout=B.LAYOUT_TILE) for m in (w1, w3, w2)])
        idx = (torch.arange(T) % E).to(torch.int32)[:, None]
        y = G.f64(ctx.moe_ffn_int8(x.to(torch.bfloat16).to(DEV), idx.to(DEV), torch.ones((T, 1), device=DEV), B.make_int8_table(dev, DEV), F,
                                   out_dtype=B.OUT_F32))
        a = c.double().numpy() * np.array(shift)[idx[:, 0].numpy()]
        want = 127 * 2.0 ** -3 * (a / (1.0 + np.exp(-a)) * (127 * 127 * 2.0 ** -14))
        want = want[:, None] * np.where(np.arange(H) % 2, -1.0, 1.0)
        off = np.abs(y - want) / np.maximum(np.abs(want), 1e-300)
        assert (np.abs(y - want) <= 12 * 2.0 ** -24 * np.abs(want)).all(), "%.1f steps" % (off.max() * 2 ** 24)


@pytest.mark.parametrize("T", [1, 2, 20, 200, 400])
def test_ffn_swiglu_beyond_the_exponentials_range(ctx, T):  # noqa: F811
    """a from 128 up to 2.5e38, where a log2 e is no number of 32 bits, is a itself times u, and up to -128 it is 0."""
    H, F = 128, 1
    for up in (2.0, 2.0 ** 121):
        c = ((torch.arange(T) * 7) % 31 + 64) * (1 - torch.arange(T) % 3 // 2 * 2)        # 64 .. 94, every third negative
        x = torch.zeros((T, H))
        x[:, 0], x[:, 1] = 127, c.float()
        w1, w3 = torch.zeros((F, H)), torch.zeros((F, H))
        w1[0, 1], w3[0, 0] = up, 127 * 2.0 ** -74
        if up < 4:
            w1[0, 2] = 127 * up                     # (x's column 2 is zero; where 127 up is no number, up itself has code 127)
        w2 = torch.full((H, F), 127 * 2.0 ** -3)
        dev = [[ctx.quantize_rows(m.to(DEV), layout=B.LAYOUT_TILE) for m in (w1, w3, w2)]]
        scale = float(dev[0][0][1][0])
        a = c.double().numpy() * (127.0 if up > 4 else 1.0) * scale
        assert np.abs(a).max() >= (2.36e38 if up > 4 and T > 2 else 128)
        y = G.f64(ctx.moe_ffn_int8(x.to(torch.bfloat16).to(DEV), torch.zeros((T, 1), dtype=torch.int32, device=DEV),
                                   torch.ones((T, 1), device=DEV), B.make_int8_table(dev, DEV), F, out_dtype=B.OUT_F32))
        want = np.where(a > 0, a, 0.0) * (127 * 127 * 2.0 ** -74) * 127 * 2.0 ** -3
        # roundings: a (its sum and scale) 2, the two products of the SwiGLU 2, the reciprocal of 1 is 1, h / 127 and its product 2
        assert (np.abs(y - want[:, None]) <= 8 * 2.0 ** -24 * np.abs(want)[:, None]).all()


@pytest.mark.parametrize("T", [(1 << 25) - 1, (1 << 25) + 5, (1 << 26) - 1])
def test_route_tokens_up_to_the_limit(ctx, T):  # noqa: F811
    """As many tokens as the call takes, a launch's and more than one's: each is written, and as it is among few."""
    E = 2
    logits = torch.empty((T, E), dtype=torch.bfloat16, device=DEV)
    logits[:, 0], logits[:, 1] = 0.0, 1.0
    logits[::3, 0] = 2.0
    scores = torch.full((T, E), 7.0, device=DEV)
    idx, w = ctx.route_scored(logits, 1, renorm=False, scores=scores)
    few = torch.zeros((6, E), device=DEV)
    fi, fw = ctx.route_scored(logits[:6], 1, renorm=False, scores=few)
    assert fi[:, 0].tolist() == [0, 1, 1, 0, 1, 1]
    for r in range(6):
        assert (idx[r::6] == fi[r]).all() and (w[r::6] == fw[r]).all() and (scores[r::6] == few[r]).all()


# (shape of csrc/int8_rule.hpp, tokens, outputs, columns): tiles of 128 columns odd and even in number, one more than a multiple of four for K split in
# four, fewer than its groups need; last tiles of rows of one, two and three fragments; the steady state of every loop
PRODUCTS = [("two", 2081, 8003, 2100), ("two", 2068, 8003, 2300), ("two", 2118, 8192, 2048), ("one", 1500, 4100, 2100), ("one", 2433, 9001, 700),
            ("split2", 1100, 3000, 700), ("split2", 1064, 4200, 2100), ("split4", 130, 4100, 2100), ("split4", 600, 3000, 1030),
            ("small64", 127, 4099, 2100), ("small32", 29, 8003, 2300), ("thin", 16, 4099, 2100), ("thin", 5, 8003, 14336)]


def big(seed, *shape, std=1.0, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def codes64(x):
    """The oracle's codes and scales of the rows of x, as tensors of 64 bits on the GPU."""
    c, s = Q.quantize_rows(G.f64(x))
    return torch.from_numpy(c.astype(np.float64)).to(DEV), torch.from_numpy(s.astype(np.float64)).to(DEV)


@pytest.mark.parametrize("shape,T,N,K", PRODUCTS)
def test_matmul_shapes_match_the_oracle(ctx, shape, T, N, K):  # noqa: F811
    """Every output of every shape, in each type, with a bias and without, rows of the output aligned for wide stores and not."""
    w, x = big(T, N, K, std=0.05), big(N, T, K)
    wt = ctx.quantize_rows(w, layout=B.LAYOUT_TILE)
    (wq, ws), (xq, xs) = codes64(w), codes64(x)
    prod = (xq @ wq.T) * xs[:, None] * ws[None, :]
    bias = big(3, N, dtype=torch.float32)
    xc, xsc = ctx.quantize_rows(x)
    for out in (torch.bfloat16, torch.float32, torch.float16):
        for b, gap in ((None, -N % 4), (bias, -N % 4 + 2)):
            y = torch.full((T + 1, N + gap), 77.0, dtype=out, device=DEV)
            ctx.matmul_int8(x, wt, bias=b, y=y[:T, :N])
            ref = prod if b is None else prod + b.double()
            tol = 4 * 2.0 ** -24 * prod.abs() + (G.HALF[out] + 2 * 2.0 ** -24) * ref.abs() + (2.0 ** -25 if out == torch.float16 else 0.0)
            assert ((y[:T, :N].double() - ref).abs() <= tol).all()
            assert (y[T] == 77).all() and (y[:, N:] == 77).all()
            z = torch.full((T + 1, N + gap), 77.0, dtype=out, device=DEV)
            ctx.matmul_int8(xc, wt, x_scale=xsc, bias=b, y=z[:T, :N])
            assert torch.equal(y, z)


# pairs of each expert: tall tiles from 161 on, wide ones up to 160, their last tiles of every number of fragments
LOADS = [276, 336, 161, 160, 129, 100, 70, 40, 20]
EXPERTS = [(700, 1100, 2200), (700, 2048, 1000), (700, 2100, 1920), (700, 1664, 2432)]          # tokens, H, F
LONG_ROWS = [(100, 16500, 40), (100, 40, 16500), (700, 16500, 264)]


def ffn_reference(x, idx, gate, host, eps):
    """int8_oracle.moe_ffn's y and bound for every expert's pairs at once, in 64 bits on the GPU; and the sum over the slots of what
    their outputs are in size.  host: an expert's three (codes, scales) of 64 bits."""
    T, H = x.shape
    xq, xs = codes64(x)
    y, var, drift, most, size = (torch.zeros((T, H), dtype=torch.float64, device=DEV) for _ in range(5))
    widest = 0.0
    for e, ((q1, s1), (q3, s3), (q2, s2)) in enumerate(host):
        t, j = (idx == e).nonzero(as_tuple=True)
        a, u = ((xq[t] @ q.T) * xs[t][:, None] * s for q, s in ((q1, s1), (q3, s3)))
        widest = max(widest, float(a.abs().max()))
        h = a / (1.0 + torch.exp(-a)) * u
        step = h.abs().amax(1, keepdim=True) / 127.0
        g, w2 = gate[t, j].double()[:, None], q2 * s2[:, None]
        o = (torch.round(h / step) * step) @ w2.T
        for i in range(idx.shape[1]):                            # (a token at most once for each slot: no two writers of a row)
            m = j == i
            r = t[m]
            y[r] += (g * o)[m]
            size[r] += (g.abs() * o.abs())[m]
            drift[r] += (g.abs() * o.abs() * eps)[m]
            var[r] += (g * g * ((2.0 * eps * h.abs() * step) @ (w2 ** 2).T))[m]
            most[r] = torch.maximum(most[r], (g.abs() * step * w2.abs().amax(1))[m])
    assert widest <= 16.0
    rare = float(np.log(2.0 / 2e-9))
    return y, most * rare / 3.0 + torch.sqrt((most * rare / 3.0) ** 2 + 2.0 * var * rare) + drift, size


@pytest.mark.parametrize("T,H,F", EXPERTS + LONG_ROWS)
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32, torch.float16])
def test_ffn_tiles_of_long_rows_match_the_oracle(ctx, T, H, F, out):  # noqa: F811
    """Experts' tiles in their loops' steady state.  The intermediate's relative error with |a| <= 16, in steps of 2^-24: a's own three roundings
    times 1 + |a|, 51; the sigmoid and its products 8.5; u's three: 63, so eps = 2^-18 in what test_gpu_int8 derives.  Beside it, of each
    pair's output: the scale of its codes, the sum's conversion and its two products 4, a slot's multiply-add one for each slot, the
    output's type."""
    k = 2
    loads = LOADS if T == 700 else [T, T // 2]
    E = len(loads)
    slots = torch.cat([torch.full((n,), e) for e, n in enumerate(loads)] + [torch.full((T * k - sum(loads),), -1)])
    idx = slots[torch.randperm(T * k, generator=torch.Generator().manual_seed(H))].view(T, k).to(torch.int32).to(DEV)
    gate = big(F, T, k, dtype=torch.float32).abs() + 0.1
    mats = [[big(700 + 3 * e + i, *s, std=0.5 * s[1] ** -0.5) for i, s in enumerate(((F, H), (F, H), (H, F)))] for e in range(E)]
    table = [[ctx.quantize_rows(m, layout=B.LAYOUT_TILE) for m in ex] for ex in mats]
    x = big(H + F, T, H)
    ref, bound, size = ffn_reference(x, idx, gate, [[codes64(m) for m in ex] for ex in mats], 2.0 ** -18)
    y = torch.full((T + 1, H), 77.0, dtype=out, device=DEV)
    ws = torch.full((B.moe_ffn_int8_workspace_bytes(T, H, F, E, k),), 0xFF, dtype=torch.uint8, device=DEV)
    ctx.moe_ffn_int8(x, idx, gate, B.make_int8_table(table, DEV), F, y=y[:T], workspace=ws)
    tol = bound + (k + 4) * 2.0 ** -24 * (size + bound) + G.HALF[out] * (ref.abs() + bound) + (2.0 ** -25 if out == torch.float16 else 0.0)
    off = (y[:T].double() - ref).abs()
    print("T=%d H=%d F=%d: worst %.2f of the bound" % (T, H, F, float((off / tol.clamp_min(1e-300)).max())), flush=True)
    assert (off <= tol).all() and (y[T] == 77).all()


@pytest.mark.parametrize("T", [1, 33, 260])
def test_layer_flags_an_absent_expert_where_it_is_chosen(ctx, T):  # noqa: F811
    H, F, E, k = 192, 256, 16, 4
    mats = [[G.randn(800 + 3 * e + i, *s, std=0.05) for i, s in enumerate(((F, H), (F, H), (H, F)))] for e in range(E)]
    mats[3] = None
    experts = Int8Experts(ctx, mats, DEV)
    layer = Int8MoELayer(ctx, T, H, F, E, k, groups=4, top_groups=2, group_best=2)
    logits, x = G.randn(70, T, E, dtype=torch.float32), G.randn(T, T, H)
    for push in (-5.0, 5.0, -5.0):
        bias = torch.zeros(E, device=DEV).index_fill(0, torch.tensor([3], device=DEV), push)
        ctx.device_flags()
        layer.step(x, experts, logits=logits, bias=bias)
        assert bool((layer.idx == 3).any()) == (push > 0)
        assert ctx.device_flags() == (B.FLAG_FORMAT_MISSING if push > 0 else 0)
