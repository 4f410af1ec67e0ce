"""GPU tests of what the microscaled 4-bit products owe bit for bit: rows converted in a call and codes made before it meet in the same sums, and
sums that 32 bits hold are exact whatever a row's length.

Tolerance of sums whose blocks are of sizes far apart, or cancel, in steps of 2^-24: a matrix instruction adds a block's exact sum to what is there and
rounds, half a step of a number no larger than the blocks' magnitudes, sum over blocks |sum|; and before that it cuts what is there, by less than a
step of the power of two of the block's largest product (0.5 counted as 1: at most 4 times the product; 16 - 16 leaves 2^-20 beside it and not 2^-21,
0.25 - 0.25 leaves 2^-24 and not 2^-25).  Largest products of all blocks add up to at most sum |x| |w|.  With another step for a block's
sum beside what is there, and 16 for the additions of the parts that K is dealt to: (2 K / 32 + 16) sum over blocks |sum| + 4 sum |x| |w|.
"""
import numpy as np
import pytest
import torch

import test_gpu_mx4 as G
from oracle import mx4_oracle as Q
from paper_2603_19172_amd import binding as B
from gpu_helpers import DEV
from test_gpu_mx4 import ctx  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def spread(seed, rows, K, dtype=torch.bfloat16, std=1.0):
    """Blocks of sizes far apart: their fp32 sum depends on its order."""
    g = torch.Generator().manual_seed(seed)
    size = torch.ldexp(torch.ones(()), torch.randint(-6, 7, (rows, -(-K // 32), 1), generator=g)).expand(-1, -1, 32).reshape(rows, -1)[:, :K]
    return (torch.randn((rows, K), generator=g) * std * size).to(dtype).to(DEV)


def product(xv, wv):
    """The product of two matrices of values, and the bound above."""
    T, K = xv.shape
    mag = np.zeros((T, len(wv)))
    for b in range(0, K, 32):
        mag += np.abs(xv[:, b:b + 32] @ wv[:, b:b + 32].T)
    return xv @ wv.T, ((2 * (Q.up(K, 256) // 32) + 16) * mag + 4 * (np.abs(xv) @ np.abs(wv).T)) * 2.0 ** -24


# both sides of the rule's lines: rows converted by every workgroup or in a launch of their own, K dealt to eight wavefronts or to four
@pytest.mark.parametrize("T,N,K", [(1, 12768, 4096), (1, 12769, 4096), (1, 14336, 4096), (4, 13001, 4096), (5, 13001, 4096), (16, 12900, 1000),
                                   (32, 12800, 512), (33, 12800, 512), (1, 12769, 300), (2, 33000, 2100)])
def test_rows_and_their_codes_give_the_same_bits(ctx, T, N, K):  # noqa: F811
    w = spread(N, N, K, std=0.05)
    wt = ctx.quantize_mx4(w, layout=B.LAYOUT_TILE)
    bias = G.randn(5, N, dtype=torch.float32)
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        x = spread(T + K, T, K, dtype=dtype)
        m = ctx.quantize_mx4(x)
        for b in (None, bias):
            y = ctx.matmul_mx4(x, wt, bias=b, out_dtype=B.OUT_F32)
            assert torch.equal(y, ctx.matmul_mx4(m, wt, bias=b, out_dtype=B.OUT_F32))
    prod, bound = product(Q.values(*Q.quantize(G.f64(x)))[:, :K], Q.values(*Q.quantize(G.f64(w)))[:, :K])
    G.close(ctx.matmul_mx4(x, wt, out_dtype=B.OUT_F32), prod, bound, torch.float32)


# the shapes by rows and outputs, as test_gpu_mx4_shapes.PRODUCTS names them
@pytest.mark.parametrize("T,N,K", [(1, 300, 14336), (3, 13001, 300), (40, 70, 9000), (130, 2600, 256), (222, 1295, 2300), (500, 2500, 520), (520, 2300, 200),
                                   (900, 5000, 300), (1950, 5000, 257), (2091, 4300, 520)])
def test_blocks_that_cancel_or_are_far_apart(ctx, T, N, K):  # noqa: F811
    x, w = spread(T, T, K), spread(N, N, K, std=0.05)
    x[:, 1::2], w[:, 1::2] = x[:, 0:K - K % 2:2], torch.where(torch.arange(K // 2, device=DEV) % 5 > 0, -w[:, 0:K - K % 2:2], w[:, 0:K - K % 2:2])
    prod, bound = product(Q.values(*Q.quantize(G.f64(x)))[:, :K], Q.values(*Q.quantize(G.f64(w)))[:, :K])
    y = ctx.matmul_mx4(x, ctx.quantize_mx4(w, layout=B.LAYOUT_TILE), out_dtype=B.OUT_F32)
    G.close(y, prod, bound, torch.float32)


def ones(seed, *shape):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randint(0, 2, shape, generator=g, device=DEV, dtype=torch.int8) * 2 - 1).half()


def exact(x, w):
    """Products of +-1, in 64 bits, a piece of K at a time."""
    return sum(x[:, c:c + 16384].double() @ w[:, c:c + 16384].double().T.contiguous() for c in range(0, x.shape[1], 16384))


# strips with one row and more, of eight wavefronts and of four, rows converted inside; tiles of 32, 64 and (64 x 256) rows: a block that is left out shows
@pytest.mark.parametrize("T,N,K", [(1, 40, 131072), (5, 300, 131071), (33, 40, 131072), (1, 12900, 16384), (1, 40, 16384), (1, 12900, 16500), (33, 12900, 9000),
                                   (2080, 128, 131072), (2080, 520, 40000), (935, 4500, 20000)])
def test_long_sums_that_32_bits_hold_are_exact(ctx, T, N, K):  # noqa: F811
    x, w = ones(T, T, K), ones(N, N, K)
    want = exact(x, w)
    wt = ctx.quantize_mx4(w, layout=B.LAYOUT_TILE)
    for a in (x, ctx.quantize_mx4(x)):
        assert torch.equal(ctx.matmul_mx4(a, wt, out_dtype=B.OUT_F32).double(), want)


# strips with K dealt to four wavefronts, tall tiles; K = H of the up projection, K = F of the down projection
@pytest.mark.parametrize("T,E", [(1, 2), (40, 2), (40, 8), (300, 2)])
def test_long_rows_of_experts(ctx, T, E):  # noqa: F811
    """Up: sums of +-1 over 131072 columns, a 2^-8 of each; the intermediate comes back through W2 = 1 on a diagonal.  A block that is left out moves
    a sum by 5 of 256 on average, and one code in twenty or so with it."""
    H, F = 131072, 64
    x, w1, w3, w2 = ones(1, T, H), ones(2, F, H) / 256, ones(3, F, H) / 256, torch.zeros((H, F), dtype=torch.half, device=DEV)
    w2[torch.arange(F), torch.arange(F)] = 1.0
    mats = [ctx.quantize_mx4(m, layout=B.LAYOUT_TILE) for m in (w1, w3, w2)]
    table = B.make_mx4_table([mats] * E, DEV)
    idx = (torch.arange(T, device=DEV) % E).int()[:, None].contiguous()
    y = ctx.moe_ffn_mx4(x, idx, torch.ones((T, 1), device=DEV), table, F, out_dtype=B.OUT_F32)
    a, u = exact(x, w1), exact(x, w3)
    h = a / (1.0 + torch.exp(-a)) * u
    # silu and its product are off by 9 steps of 2^-24; on either side of a border within 16
    lo, hi = (Q.values(*Q.quantize(G.f64(h * (1 + d)))) for d in (-16 * 2.0 ** -24, 16 * 2.0 ** -24))
    got = G.f64(y[:, :F])
    assert ((got == lo[:, :F]) | (got == hi[:, :F])).all() and (lo == hi).mean() > 0.99 and (y[:, F:] == 0).all()


@pytest.mark.parametrize("T,E", [(1, 2), (20, 2), (40, 8), (300, 2)])
def test_long_intermediates_of_experts(ctx, T, E):  # noqa: F811
    """Down: an intermediate of which every value is 1.5 (silu of 2^30 is 2^30), its signs those of W3, in a sum over 131072 of them."""
    H, F = 64, 131072
    sign, w2 = ones(4, F), ones(5, H, F)
    w1, w3 = torch.zeros((F, H), device=DEV), torch.zeros((F, H), device=DEV)
    w1[:, 0], w3[:, 32] = 1.0, sign.float()
    x = torch.zeros((T, H), device=DEV)
    x[:, 0], x[:, 32] = 2.0 ** 30, 1.5 * 2.0 ** -30 * (torch.arange(T, device=DEV) % 2 * 2 - 1)
    mats = [ctx.quantize_mx4(m, layout=B.LAYOUT_TILE) for m in (w1, w3, w2)]
    table = B.make_mx4_table([mats] * E, DEV)
    idx = (torch.arange(T, device=DEV) % E).int()[:, None].contiguous()
    y = ctx.moe_ffn_mx4(x, idx, torch.ones((T, 1), device=DEV), table, F, out_dtype=B.OUT_F32)
    want = 1.5 * (torch.arange(T, device=DEV) % 2 * 2 - 1)[:, None] * (w2.double() @ sign.double())[None]
    assert torch.equal(y.double(), want.expand(T, H))
