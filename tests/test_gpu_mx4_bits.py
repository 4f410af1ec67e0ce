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
