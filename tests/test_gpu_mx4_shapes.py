"""GPU tests of the microscaled 4-bit products across the shapes that a call is computed in: each at sizes that reach its steady state, with ragged
rows, columns and last tiles, against the oracle with test_gpu_mx4's bounds."""
import numpy as np
import pytest
import torch

import test_gpu_mx4 as G
from oracle import mx4_oracle as Q
from paper_2603_19172_amd import binding as B
from paper_2603_19172_amd.layer import Mx4Experts
from gpu_helpers import DEV
from test_gpu_mx4 import ctx  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

# shape, T, N, K: steps of 256 columns from one to more than a shape has on their way, odd and even, last tiles of every number of fragments
PRODUCTS = [("small", 3, 13001, 300), ("small", 30, 12900, 777), ("small", 90, 1500, 2600), ("small", 40, 70, 9000),
            ("tile32", 97, 3201, 1300), ("tile32", 130, 2600, 256), ("tile32", 250, 1900, 1537), ("tile32", 33, 14000, 300), ("tile32", 222, 1295, 2300),
            ("tile64", 500, 2500, 520), ("tile64", 449, 2700, 1100), ("tile64", 610, 1700, 2049), ("tile64", 520, 2300, 200),
            ("tile64w", 900, 5000, 300), ("tile64w", 935, 4500, 800), ("tile64w", 1030, 4700, 1100),
            ("tile128", 1950, 5000, 257), ("tile128", 2091, 4300, 520), ("tile128", 2113, 4000, 1025), ("tile128", 2170, 4000, 200)]

# T, H, F, E, k, splits: experts in tall tiles
TALL = [(200, 264, 1000, 2, 1, 1), (300, 700, 520, 4, 2, 1), (200, 264, 2100, 2, 1, 2), (410, 1030, 3100, 3, 2, 2), (150, 300, 8300, 2, 1, 4),
        (420, 520, 256, 2, 2, 1)]

# T, H, F, E, k, waves of the up and of the down projection: experts in strips
STRIPS = [(20, 1100, 300, 6, 2, 4, 2), (5, 300, 2500, 4, 2, 2, 8), (30, 200, 70, 40, 8, 1, 1), (9, 640, 1100, 4, 2, 2, 4), (250, 800, 1300, 60, 4, 1, 1)]

# T, H, F, E, k: a few pairs
THIN = [(1, 4096, 1000, 2, 2), (2, 1030, 3100, 4, 2), (1, 270, 300, 64, 64), (4, 520, 770, 128, 8), (8, 256, 256, 64, 2), (1, 100, 14336, 3, 1)]


@pytest.mark.parametrize("shape,T,N,K", PRODUCTS)
def test_products(ctx, shape, T, N, K):  # noqa: F811
    wt, wv = G.weight(ctx, N, N, K)
    x = G.randn(T + K, T, K)
    bias = G.randn(7, N, dtype=torch.float32)
    prod, bound = Q.matmul(Q.values(*Q.quantize(G.f64(x)))[:, :K], wv)
    ref = prod + G.f64(bias)
    for out in (torch.float32, torch.bfloat16):
        y = torch.full((T + 1, N + 3), 9.0, dtype=out, device=DEV)
        ctx.matmul_mx4(x, wt, bias=bias, y=y[:T, :N])
        G.close(y[:T, :N], ref, bound + 2.0 ** -24 * np.abs(ref), out)
        assert (y[T:] == 9).all() and (y[:, N:] == 9).all()
    y = ctx.matmul_mx4(x, wt, out_dtype=B.OUT_F16)
    G.close(y, prod, bound, torch.float16)
    assert torch.equal(y, ctx.matmul_mx4(ctx.quantize_mx4(x), wt, out_dtype=B.OUT_F16))


def check(ctx, T, H, F, E, k, popular):
    ex, vals = G.make_experts(ctx, T + F, E, H, F)
    idx, gate = G.choices(T, T, E, k, popular=popular)
    x = G.randn(T + H, T, H)
    y, ref = G.check_ffn(ctx, x, idx, gate, ex, vals, out=torch.float32)
    # 16-bit outputs are the fp32 ones rounded
    for t in (torch.bfloat16, torch.float16):
        assert torch.equal(ctx.moe_ffn_mx4(x, idx, gate, ex.table, F, out_dtype=G.OUT[t]), y.to(t))
    return idx


@pytest.mark.parametrize("T,H,F,E,k,splits", TALL)
@pytest.mark.parametrize("popular", [0.0, 1.5])
def test_experts_in_tall_tiles(ctx, T, H, F, E, k, splits, popular):  # noqa: F811
    check(ctx, T, H, F, E, k, popular)


@pytest.mark.parametrize("T,H,F,E,k,up,down", STRIPS)
def test_experts_in_strips(ctx, T, H, F, E, k, up, down):  # noqa: F811
    check(ctx, T, H, F, E, k, 0.5)


@pytest.mark.parametrize("T,H,F,E,k", THIN)
def test_experts_of_a_few_pairs(ctx, T, H, F, E, k):  # noqa: F811
    check(ctx, T, H, F, E, k, 0.0)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 64, 96, 97, 127, 128, 129, 160, 256, 257, 300])
def test_experts_of_every_number_of_pairs(ctx, n):  # noqa: F811
    """One expert with n pairs, another with the rest, in tall tiles; the rows that share a tile do not matter."""
    E, H, F = 3, 520, 300
    T = 340
    ex, vals = G.make_experts(ctx, 3, E, H, F)
    idx = (torch.arange(T) >= n).to(torch.int32)[torch.randperm(T, generator=torch.Generator().manual_seed(n))][:, None].contiguous().to(DEV)
    assert int((idx == 0).sum()) == n
    G.check_ffn(ctx, G.randn(n, T, H), idx, torch.ones((T, 1), device=DEV), ex, vals, out=torch.float32)


def test_more_pairs_than_the_plans_registers_and_lds_hold(ctx):  # noqa: F811
    E, H, F, k, T = 16, 96, 64, 8, 2500
    ex, vals = G.make_experts(ctx, 4, E, H, F)
    idx, gate = G.choices(5, T, E, k, popular=0.7)
    G.check_ffn(ctx, G.randn(6, T, H), idx, gate, ex, vals)


def test_more_tiles_than_the_plans_lds_holds(ctx):  # noqa: F811
    """32 tokens or fewer an expert in tiles of 32 rows cannot pass 4096 tiles; tall tiles of many pairs can."""
    E, H, F, T = 2, 32, 32, 4100 * 128
    w = [[G.randn(3 * e + i, n, m, std=0.3) for i, (n, m) in enumerate(((F, H), (F, H), (H, F)))] for e in range(E)]
    ex = Mx4Experts(ctx, w, DEV)
    x = G.randn(1, 1000, H).repeat(-(-T // 1000), 1)[:T].contiguous()
    idx = (torch.arange(T, device=DEV) % 1000 % 2).to(torch.int32)[:, None].contiguous()
    y = ctx.moe_ffn_mx4(x, idx, torch.ones((T, 1), device=DEV), ex.table, F, out_dtype=B.OUT_F32)
    vals = [[Q.values(*Q.quantize(G.f64(t)))[:, :t.shape[1]] for t in m] for m in w]
    ref, bound = Q.moe_ffn(Q.values(*Q.quantize(G.f64(x[:1000])))[:, :H], idx[:1000].cpu().numpy(), np.ones((1000, 1)), vals)
    G.close(y[:1000], ref, bound, torch.float32)
    # one K tile: every row's sums are taken alike, whatever tile it is in
    assert torch.equal(y, y[:1000].repeat(-(-T // 1000), 1)[:T])


def test_a_long_rows_products(ctx):  # noqa: F811
    """Rows of 131072 columns through every shape that takes them, weights of one block's width."""
    K = 131072
    w = G.randn(2, 40, K, std=0.02)
    wt, wv = ctx.quantize_mx4(w, layout=B.LAYOUT_TILE), Q.values(*Q.quantize(G.f64(w)))
    for T in (1, 33):
        x = G.randn(T, T, K)
        prod, bound = Q.matmul(Q.values(*Q.quantize(G.f64(x))), wv)
        G.close(ctx.matmul_mx4(x, wt, out_dtype=B.OUT_F32), prod, bound, torch.float32)


def test_products_of_codes_beyond_32_bits_of_bytes(ctx):  # noqa: F811
    """70000 rows of 131072 columns, 4.6e9 bytes of codes: one row and its negative, sums of +-1 that 32 bits hold."""
    T, N, K = 70000, 40, 131072
    g = torch.Generator().manual_seed(5)
    one = lambda *shape: (torch.randint(0, 2, shape, generator=g) * 2 - 1).half().to(DEV)  # noqa: E731
    row, w, sign = one(1, K), one(N, K), one(T, 1)
    wt = ctx.quantize_mx4(w, layout=B.LAYOUT_TILE)
    x = sign * row
    ref = sign.float() * (row.double() @ w.double().T).float()
    assert torch.equal(ctx.matmul_mx4(x, wt, out_dtype=B.OUT_F32), ref)
    for layout in (B.LAYOUT_ROWMAJOR, B.LAYOUT_TILE):
        m = ctx.quantize_mx4(x, layout=layout)
        if layout == B.LAYOUT_ROWMAJOR:
            assert torch.equal(ctx.matmul_mx4(m, wt, out_dtype=B.OUT_F32), ref)
        assert torch.equal(ctx.dequantize_mx4(m, out_dtype=B.OUT_F16), x)
        del m
    torch.cuda.empty_cache()


def test_experts_with_an_intermediate_beyond_32_bits_of_bytes(ctx):  # noqa: F811
    """Two kinds of token on four entries of one expert: every row has the bits of its kind, those of fewer tokens in the same shape."""
    T, H, F, E = 60000, 256, 131072, 4
    mats = [ctx.quantize_mx4(G.randn(i, n, m, std=0.05), layout=B.LAYOUT_TILE) for i, (n, m) in enumerate(((F, H), (F, H), (H, F)))]
    table = B.make_mx4_table([mats] * E, DEV)
    kind = G.randn(4, 2, H)
    x = kind.repeat(T // 2, 1)
    idx = torch.randint(0, E, (T, 1), generator=torch.Generator().manual_seed(6)).int().to(DEV)
    gate = torch.ones((T, 1), device=DEV)
    few = ctx.moe_ffn_mx4(x[:9000], idx[:9000].contiguous(), gate[:9000].contiguous(), table, F, out_dtype=B.OUT_F32)
    assert torch.equal(few, few[:2].repeat(4500, 1)) and torch.isfinite(few).all() and (few.abs().amax(dim=1) > 0).all()
    y = ctx.moe_ffn_mx4(x, idx, gate, table, F, out_dtype=B.OUT_F32)
    assert torch.equal(y, few[:2].repeat(T // 2, 1))
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,N", [(1, 160), (40, 160), (300, 160), (1500, 5000)])
def test_products_at_the_ends_of_the_range(ctx, T, N):  # noqa: F811
    """One sum of 512 equal products: subnormal ones are kept, those beyond the range are infinite, zeros stay zeros beside any power of two."""
    K = 512
    x, w = torch.ones((T, K), device=DEV), torch.ones((N, K), device=DEV)
    w[1], w[2], w[3, ::2] = 0.0, -1.0, -1.0
    for ex, ew in ((-70, -60), (-75, -70), (-100, -100), (60, 60), (100, 100), (-126, 120)):
        y = ctx.matmul_mx4(x * 2.0 ** ex, ctx.quantize_mx4(w * 2.0 ** ew, layout=B.LAYOUT_TILE), out_dtype=B.OUT_F32)
        want = torch.full((N,), 512 * 2.0 ** ex * 2.0 ** ew, dtype=torch.float64).float()
        want[1], want[2], want[3] = 0.0, -want[2], 0.0
        assert torch.equal(y, want.to(DEV).expand(T, N)), (ex, ew)


@pytest.mark.parametrize("T", [2, 40, 300])
def test_calls_at_once_on_two_streams(ctx, T):  # noqa: F811
    """Workspaces of their own: nothing else is shared."""
    H, F, E, k = 256, 512, 8, 2
    ex, _ = G.make_experts(ctx, 25, E, H, F)
    wt, _ = G.weight(ctx, 26, 400, H)
    x, logits = G.randn(27, T, H), G.randn(28, T, E, dtype=torch.float32)
    idx, gate = G.choices(28, T, E, k)
    calls = (lambda: ctx.moe_ffn_mx4(x, idx, gate, ex.table, F), lambda: ctx.matmul_mx4(x, wt),
             lambda: ctx.route_balance(logits, idx, 0.1)[1], lambda: ctx.dequantize_mx4(ctx.quantize_mx4(x)))
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(24):
        with torch.cuda.stream(streams[i % 2]):
            got.append(calls[(i + i // 4) % 4]())
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[(i + i // 4) % 4]) for i, y in enumerate(got))


@pytest.mark.parametrize("handle", [False, True])
def test_memory_of_a_call_belongs_to_its_stream(ctx, monkeypatch, handle):  # noqa: F811
    """What a call on another stream allocates is not given to the current stream's work before the call has run."""
    x, wt = G.randn(3, 200, 512), G.weight(ctx, 9, 300, 512)[0]
    ex, _ = G.make_experts(ctx, 9, 4, 512, 256)
    idx, gate = G.choices(9, 200, 4, 2)
    logits = G.randn(4, 200, 4, dtype=torch.float32)
    want = ctx.matmul_mx4(x, wt), ctx.moe_ffn_mx4(x, idx, gate, ex.table, 256), ctx.route_balance(logits, idx, 0.1)[1]
    taken, empty = [], B._empty

    def spy(shape, dtype, device, stream):
        t = empty(shape, dtype, device, stream)
        taken.append((t.data_ptr(), t.numel(), dtype))
        return t
    monkeypatch.setattr(B, "_empty", spy)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    stream = s.cuda_stream if handle else s
    got = (ctx.matmul_mx4(x, wt, stream=stream), ctx.moe_ffn_mx4(x, idx, gate, ex.table, 256, stream=stream),
           ctx.route_balance(logits, idx, 0.1, stream=stream)[1])
    assert len(taken) == 2 + 2 + 4
    for ptr, n, dtype in taken:
        assert all(torch.empty(n, dtype=dtype, device=DEV).data_ptr() != ptr for _ in range(2))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_tensors_on_another_device_are_refused(ctx):  # noqa: F811
    x, wt = G.randn(3, 8, 512), G.weight(ctx, 9, 32, 512)[0]
    for call in (lambda: ctx.matmul_mx4(x.cpu(), wt), lambda: ctx.matmul_mx4(x, wt._replace(codes=wt.codes.cpu())), lambda: ctx.quantize_mx4(x.cpu()),
                 lambda: ctx.dequantize_mx4(wt._replace(scale=wt.scale.cpu())), lambda: ctx.matmul_mx4(x, wt, bias=torch.zeros(32)),
                 lambda: ctx.route_balance(x.float(), torch.zeros((8, 2), dtype=torch.int32), 0.1)):
        with pytest.raises(ValueError, match="device"):
            call()
