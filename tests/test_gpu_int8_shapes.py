"""GPU tests of the 8-bit integer experts and products across the shapes that a call is computed in: what a shape may not change, and
each shape against the oracle at sizes that reach its steady state.  The bounds are test_gpu_int8's unless a test derives its own."""
import numpy as np
import pytest
import torch

import test_gpu_int8 as G
from oracle import int8_oracle as Q
from paper_2603_19172_amd import binding as B
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
