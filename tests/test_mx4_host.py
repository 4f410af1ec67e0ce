"""Host side of the microscaled 4-bit calls and of the router's training side: argument checks before any device work, and what the
binding refuses before a call reads out of a matrix.  No GPU needed."""
import math

import pytest
import torch

from paper_2603_19172_amd import binding as B

lib = B.lib
P = 0x10000  # a non-null, aligned dummy "pointer"; never dereferenced by validation


def call(name, *a, device=0, **kw):
    class Fake:
        _h = None
        _mx4 = B.Context._mx4
    Fake.device = device
    return getattr(B.Context, name)(Fake(), *a, stream=0, **kw)


def test_rows_refusals():
    q = lambda x=P, dt=0, rows=5, K=100, ld=100, layout=0, codes=P, scale=P: lib.dymoe_quantize_mx4(None, x, dt, rows, K, ld, layout, codes, scale, None)
    assert q() == B.ENOCTX and q(rows=0, x=None, codes=None, scale=None) == B.ENOCTX and q(dt=1) == B.ENOCTX and q(dt=2, layout=1) == B.ENOCTX
    for bad in (dict(x=None), dict(codes=None), dict(scale=None), dict(dt=3), dict(dt=4), dict(dt=-1), dict(rows=-1), dict(K=0), dict(ld=99), dict(layout=2),
                dict(x=P + 1), dict(codes=P + 8), dict(scale=P + 2), dict(x=P + 2, dt=1)):
        assert q(**bad) == B.EINVAL, bad
    assert q(K=B.MX4_MAX_K + 1, ld=1 << 20) == B.ENOTSUP and q(rows=1 << 31) == B.ENOTSUP
    d = lambda codes=P, scale=P, rows=5, K=100, layout=0, dt=0, y=P, ld=100: lib.dymoe_dequantize_mx4(None, codes, scale, rows, K, layout, dt, y, ld, None)
    assert d() == B.ENOCTX and d(rows=0, y=None, codes=None, scale=None) == B.ENOCTX
    for bad in (dict(codes=None), dict(scale=None), dict(y=None), dict(rows=-1), dict(K=0), dict(layout=-1), dict(dt=3), dict(ld=99), dict(y=P + 1),
                dict(codes=P + 4), dict(scale=P + 1)):
        assert d(**bad) == B.EINVAL, bad
    assert d(K=B.MX4_MAX_K + 1, ld=1 << 20) == B.ENOTSUP


def test_matmul_refusals():
    nb = B.matmul_mx4_workspace_bytes(7, 40, 300)
    assert nb >= 7 * 512 * 17 // 32 and nb % 256 == 0
    for bad in ((-1, 4, 4), (4, 0, 4), (4, 4, 0), (4, 4, B.MX4_MAX_K + 1)):
        assert B.matmul_mx4_workspace_bytes(*bad) == 0
    m = lambda x=P, dt=0, xs=None, ld=300, w=P, ws=P, bias=None, T=7, N=40, K=300, out=0, y=P, ldy=40, buf=P, n=nb: lib.dymoe_matmul_mx4(
        None, x, dt, xs, ld, w, ws, bias, T, N, K, out, y, ldy, buf, n, None)
    assert m() == B.ENOCTX and m(dt=4, xs=P, ld=512, buf=None, n=0) == B.ENOCTX and m(T=0, x=None, y=None, buf=None, n=0) == B.ENOCTX
    for bad in (dict(x=None), dict(y=None), dict(w=None), dict(ws=None), dict(buf=None), dict(dt=3), dict(dt=5), dict(out=3), dict(ld=299), dict(ldy=39),
                dict(T=-1), dict(N=0), dict(K=0), dict(dt=4, xs=None, ld=512), dict(dt=4, xs=P, ld=300), dict(w=P + 8), dict(ws=P + 2), dict(x=P + 1),
                dict(y=P + 1), dict(out=1, y=P + 2), dict(bias=P + 2), dict(buf=P + 128), dict(dt=4, xs=P, ld=512, x=P + 8), dict(dt=4, xs=P + 1, ld=512)):
        assert m(**bad) == B.EINVAL, bad
    assert m(n=nb - 1) == B.ENOSPC
    assert m(K=B.MX4_MAX_K + 1, ld=1 << 20, n=1 << 60) == B.ENOTSUP and m(T=(1 << 24) + 1, n=1 << 60) == B.ENOTSUP
    assert m(T=1 << 20, N=1 << 20, ldy=1 << 20, n=1 << 60) == B.ENOTSUP


def test_experts_refusals():
    nb = B.moe_ffn_mx4_workspace_bytes(7, 300, 200, 8, 2)
    for bad in ((-1, 4, 4, 4, 1), (4, 0, 4, 4, 1), (4, 4, 0, 4, 1), (4, 4, 4, 0, 1), (4, 4, 4, 4, 0), (4, 4, 4, 4, 5)):
        assert B.moe_ffn_mx4_workspace_bytes(*bad) == 0
    f = lambda x=P, dt=0, idx=P, w=P, table=P, T=7, H=300, F=200, E=8, k=2, out=0, y=P, buf=P, n=nb: lib.dymoe_moe_ffn_mx4(
        None, x, dt, idx, w, table, T, H, F, E, k, out, y, buf, n, None)
    assert f() == B.ENOCTX and f(T=0, x=None, idx=None, w=None, y=None) == B.ENOCTX
    for bad in (dict(x=None), dict(idx=None), dict(w=None), dict(table=None), dict(y=None), dict(buf=None), dict(dt=3), dict(dt=4), dict(out=4), dict(T=-1),
                dict(H=0), dict(F=0), dict(E=0), dict(k=0), dict(k=9), dict(x=P + 1), dict(y=P + 1), dict(idx=P + 2), dict(w=P + 2), dict(table=P + 4),
                dict(buf=P + 16)):
        assert f(**bad) == B.EINVAL, bad
    assert f(n=nb - 1) == B.ENOSPC
    assert f(E=1025, n=1 << 60) == B.ENOTSUP and f(H=B.MX4_MAX_K + 1, n=1 << 60) == B.ENOTSUP and f(F=B.MX4_MAX_K + 1, n=1 << 60) == B.ENOTSUP
    assert f(T=1 << 28, n=1 << 60) == B.ENOTSUP and f(T=1 << 24, H=1024, k=1, n=1 << 60) == B.ENOTSUP


def test_balance_and_gradient_refusals():
    nb = B.route_balance_workspace_bytes(700, 30)
    assert nb % 256 == 0 and B.route_balance_workspace_bytes(-1, 30) == 0 and B.route_balance_workspace_bytes(5, 0) == 0
    b = lambda l=P, dt=0, idx=P, keep=None, T=700, E=30, k=3, score=0, coef=0.1, counts=P, mean=P, loss=P, buf=P, n=nb: lib.dymoe_route_balance(
        None, l, dt, idx, keep, T, E, k, score, coef, counts, mean, loss, buf, n, None)
    assert b() == B.ENOCTX and b(keep=P + 1) == B.ENOCTX and b(T=0, l=None, idx=None) == B.ENOCTX and b(coef=-1.0) == B.ENOCTX
    for bad in (dict(l=None), dict(idx=None), dict(counts=None), dict(mean=None), dict(loss=None), dict(buf=None), dict(dt=3), dict(score=2), dict(T=-1),
                dict(E=0), dict(k=0), dict(k=31), dict(coef=math.nan), dict(coef=math.inf), dict(l=P + 1), dict(idx=P + 2), dict(counts=P + 1),
                dict(mean=P + 2), dict(loss=P + 2), dict(buf=P + 64)):
        assert b(**bad) == B.EINVAL, bad
    assert b(n=nb - 1) == B.ENOSPC
    assert b(E=1025, n=1 << 60) == B.ENOTSUP and b(E=100, k=65, n=1 << 60) == B.ENOTSUP and b(T=1 << 25, n=1 << 60) == B.ENOTSUP
    g = lambda l=P, dt=0, idx=P, dw=P, T=7, E=30, k=3, score=0, renorm=1, factor=1.0, counts=P, coef=0.1, dloss=None, keep=None, gt=0, grad=P: \
        lib.dymoe_route_scored_backward(None, l, dt, idx, dw, T, E, k, score, renorm, factor, counts, coef, dloss, keep, gt, grad, None)
    assert g() == B.ENOCTX and g(dw=None) == B.ENOCTX and g(counts=None) == B.ENOCTX and g(dw=None, idx=None) == B.ENOCTX and g(T=0, l=None, grad=None) == B.ENOCTX
    for bad in (dict(l=None), dict(idx=None), dict(grad=None), dict(dw=None, counts=None), dict(dt=3), dict(gt=3), dict(score=-1), dict(factor=0.0),
                dict(factor=math.inf), dict(factor=math.nan), dict(coef=math.nan), dict(T=-1), dict(k=31), dict(dw=P + 2), dict(counts=P + 2),
                dict(dloss=P + 1), dict(grad=P + 1), dict(gt=1, grad=P + 2)):
        assert g(**bad) == B.EINVAL, bad
    assert g(E=1025) == B.ENOTSUP and g(E=100, k=65) == B.ENOTSUP and g(T=1 << 25) == B.ENOTSUP


def matrix(rows, cols, layout=B.LAYOUT_TILE, device="cpu"):
    codes, scale = B.mx4_shapes(rows, cols, layout)
    return B.Mx4Matrix(torch.zeros(codes, dtype=torch.uint8, device=device), torch.zeros(scale, dtype=torch.uint8, device=device), rows, cols, layout)


def expert(H, F, device="cpu"):
    return [matrix(F, H, device=device), matrix(F, H, device=device), matrix(H, F, device=device)]


def test_matrices_in_the_wrong_layout_or_of_other_shapes():
    x = torch.zeros(4, 300)
    with pytest.raises(ValueError, match="tile layout"):
        call("matmul_mx4", device=-1, x=matrix(4, 300, B.LAYOUT_ROWMAJOR), w=matrix(40, 300, B.LAYOUT_ROWMAJOR))
    with pytest.raises(ValueError, match="row-major"):
        call("matmul_mx4", device=-1, x=matrix(4, 300), w=matrix(40, 300))
    with pytest.raises(ValueError, match="columns"):
        call("matmul_mx4", device=-1, x=matrix(4, 299, B.LAYOUT_ROWMAJOR), w=matrix(40, 300))
    m = matrix(40, 300)
    for bad in (m._replace(rows=65), m._replace(cols=513), m._replace(scale=m.codes), m._replace(codes=m.codes.to(torch.int8))):
        with pytest.raises((ValueError, TypeError)):
            call("dequantize_mx4", bad, device=-1, out=torch.zeros(bad.rows, bad.cols))
    with pytest.raises(ValueError, match="shape"):
        call("dequantize_mx4", m, device=-1, out=torch.zeros(40, 301))
    with pytest.raises(ValueError, match="shape"):
        call("quantize_mx4", x.bfloat16(), device=-1, out=(torch.zeros(4, 255, dtype=torch.uint8), torch.zeros(4, 16, dtype=torch.uint8)))


def test_experts_of_other_sizes_or_formats_than_the_tables_are_refused():
    table = B.make_mx4_table([expert(200, 40), None, expert(200, 40)], "cpu")
    assert table.numel() == 144
    ffn = lambda H, F, t: call("moe_ffn_mx4", torch.zeros(4, H), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), t, F)
    for H, F in ((200, 41), (200, 8000), (201, 40), (40, 200)):
        with pytest.raises(ValueError, match="the table's experts"):
            ffn(H, F, table)
    with pytest.raises(ValueError, match="context is of device"):       # the table's own sizes: only the tensors' device is wrong here
        ffn(200, 40, table)
    with pytest.raises(ValueError, match="context is of device"):
        ffn(200, 41, torch.zeros((3, 6), dtype=torch.int64))
    for bad in (torch.zeros(100, dtype=torch.uint8), torch.zeros(0, dtype=torch.uint8)):
        with pytest.raises(ValueError, match="whole entries"):
            ffn(200, 40, bad)
    pair = lambda n, k: (torch.zeros((-(-n // 32) * 32, -(-k // 128) * 128), dtype=torch.int8), torch.zeros(n))
    int8 = B.make_int8_table([[pair(40, 200), pair(40, 200), pair(200, 40)]], "cpu")
    with pytest.raises(ValueError, match="format"):
        ffn(200, 40, int8)
    with pytest.raises(ValueError, match="format"):
        call("moe_ffn_int8", torch.zeros(4, 200), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), table, 40)


def test_tables_refuse_what_a_kernel_could_not_follow():
    good = expert(200, 40)
    for bad in (expert(200, 40, "meta"), good[:2] + expert(200, 40, "meta")[2:]):
        with pytest.raises(ValueError, match="device"):
            B.make_mx4_table([bad], "cpu")
    for bad in ([good[0], good[1], good[0]], [good[0]._replace(layout=B.LAYOUT_ROWMAJOR), good[1], good[2]], [good[0], matrix(41, 200), good[2]]):
        with pytest.raises(ValueError, match="layout"):
            B.make_mx4_table([bad], "cpu")
    with pytest.raises(ValueError, match="one size"):
        B.make_mx4_table([good, expert(200, 41)], "cpu")
    with pytest.raises(ValueError, match="shapes"):
        B.make_mx4_table([[good[0]._replace(codes=good[0].codes[:, :64]), good[1], good[2]]], "cpu")
    flat = torch.zeros(good[0].codes.numel() + 16, dtype=torch.uint8)
    with pytest.raises(ValueError, match="aligned"):
        B.make_mx4_table([[good[0]._replace(codes=flat[8:8 + good[0].codes.numel()].view(good[0].codes.shape)), good[1], good[2]]], "cpu")
    n = good[0].scale.numel()
    with pytest.raises(ValueError, match="aligned"):
        B.make_mx4_table([[good[0]._replace(scale=flat[2:2 + n].view(good[0].scale.shape)), good[1], good[2]]], "cpu")


def test_router_calls_check_shapes():
    logits, idx = torch.zeros(5, 8), torch.zeros((5, 2), dtype=torch.int32)
    for kw in (dict(keep=torch.zeros(4, dtype=torch.uint8)), dict(counts=torch.zeros(8, dtype=torch.int32)), dict(keep=torch.zeros(5))):
        with pytest.raises((ValueError, TypeError)):
            call("route_balance", logits, idx, 0.1, **kw)
    with pytest.raises(ValueError, match="context is of device"):
        call("route_scored_backward", logits, idx, dw=torch.zeros(5, 2))
