"""GPU tests of the microscaled 4-bit calls at more tiles of 32 rows than a launch of those would take: what they run is tall tiles."""
import pytest
import torch

import test_gpu_mx4 as G
from oracle import mx4_oracle as Q
from paper_2603_19172_amd import binding as B
from paper_2603_19172_amd.layer import Mx4Experts
from gpu_helpers import DEV
from test_gpu_mx4 import ctx  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def test_a_product_of_2_to_the_33_outputs(ctx):  # noqa: F811
    """Rows and channels that repeat after 7 and 5: each output is one of 35, with the bits that a small call gives."""
    T, N, K = 65536, 131072, 64
    x, w = G.randn(1, 7, K), G.randn(2, 5, K, std=0.1)
    ref, bound = Q.matmul(*(Q.values(*Q.quantize(G.f64(t)))[:, :K] for t in (x, w)))
    many = lambda t, n: t.repeat(-(-n // len(t)), 1)[:n].contiguous()  # noqa: E731
    wt = ctx.quantize_mx4(many(w, N), layout=B.LAYOUT_TILE)
    y = torch.full((T + 1, N), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.matmul_mx4(many(x, T), wt, y=y[:T])
    G.close(y[:7, :5], ref, bound, torch.bfloat16)
    row = many(y[:7, :5].T.contiguous(), N).T.contiguous()                 # [7, N]
    for t in range(0, T, 7 * 1024):
        part = y[t:t + 7 * 1024][:T - t]
        assert torch.equal(part, row.repeat(1024, 1)[:len(part)]), t
    assert (y[T] == 7).all()
    coded = ctx.matmul_mx4(ctx.quantize_mx4(many(x, T)), wt)
    assert all(torch.equal(coded[t:t + 8192], y[t:t + 8192]) for t in range(0, T, 8192))
    del y, coded, part
    torch.cuda.empty_cache()


def test_experts_of_more_tiles(ctx):  # noqa: F811
    """66000 tokens on four experts of 131072 features."""
    T, H, F, E = 66000, 32, 131072, 4
    w = [[G.randn(3 * e + i, n, m, std=0.05) for i, (n, m) in enumerate(((F, H), (F, H), (H, F)))] for e in range(E)]
    ex = Mx4Experts(ctx, w, DEV)
    kind = G.randn(4, 8, H)
    x = kind.repeat(T // 8, 1)
    idx = (torch.arange(T, device=DEV) // 8 % E).int()[:, None].contiguous()
    y = ctx.moe_ffn_mx4(x, idx, torch.ones((T, 1), device=DEV), ex.table, F, out_dtype=B.OUT_F32)
    vals = [[Q.values(*Q.quantize(G.f64(t)))[:, :t.shape[1]] for t in m] for m in w]
    ref, bound = Q.moe_ffn(Q.values(*Q.quantize(G.f64(x[:32])))[:, :H], idx[:32].cpu().numpy(), torch.ones((32, 1)).numpy(), vals)
    G.close(y[:32], ref, bound, torch.float32)
    assert torch.equal(y, y[:32].repeat(-(-T // 32), 1)[:T])
    torch.cuda.empty_cache()
