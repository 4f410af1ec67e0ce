"""Pins of the oracle of the routing by scores and the 8-bit integer products, and the host side of their entry points: argument
checks before any device work, workspace sizes, the binding's shape checks.  No GPU needed."""
import math

import numpy as np
import pytest
import torch

from oracle import int8_oracle as Q
from paper_2603_19172_amd import binding as B
from paper_2603_19172_amd.layer import Int8Experts, Int8MoELayer

P = 0x10000  # a non-null, aligned dummy "pointer"; never dereferenced by validation


def test_route_oracle_hand_examples():
    l = np.array([[0.0, 2.0, 1.0, -1.0]])
    idx, w, s = Q.route_scored(l, 2)
    assert idx.tolist() == [[1, 2]] and abs(w.sum() - 1) < 1e-15
    assert np.allclose(s[0], 1 / (1 + np.exp(-l[0])), rtol=1e-15)
    # the bias decides who, not with which weight
    idx, w, s = Q.route_scored(l, 1, bias=np.array([0.0, 0.0, 0.0, 5.0]), renorm=False)
    assert idx.tolist() == [[3]] and abs(w[0, 0] - 1 / (1 + math.e)) < 1e-15
    # groups {0, 1}, {2, 3}: by the largest the first, by the two largest the second
    l = np.array([[3.0, -9.0, 2.0, 2.0]])
    assert Q.route_scored(l, 2, groups=2, top_groups=1, group_best=1)[0].tolist() == [[0, 1]]
    assert Q.route_scored(l, 2, groups=2, top_groups=1, group_best=2)[0].tolist() == [[2, 3]]
    # softmax: weights without renormalising are probabilities
    _, w, s = Q.route_scored(l, 4, sigmoid=False, renorm=False, factor=2.0)
    assert abs(w.sum() - 2.0) < 1e-14 and abs(s.sum() - 1.0) < 1e-14


def test_route_oracle_masks():
    inf = math.inf
    idx, w, _ = Q.route_scored(np.array([[-inf, -inf, -inf]]), 2, sigmoid=False)
    assert idx.tolist() == [[0, 1]] and (w == 0).all()
    idx, w, _ = Q.route_scored(np.array([[-inf, 1.0, -inf]]), 2, bias=np.zeros(3))
    assert idx.tolist() == [[1, 0]] and w.tolist() == [[1.0, 0.0]]
    idx, w, _ = Q.route_scored(np.array([[math.nan, 1.0, 0.0]]), 2)
    assert idx.tolist() == [[1, 2]] and np.isnan(w).all()
    # a masked neighbour adds nothing to its group's value
    assert Q.route_scored(np.array([[4.0, -inf, 1.0, 1.0]]), 1, groups=2, group_best=2, bias=np.zeros(4))[0].tolist() == [[2]]
    assert Q.route_scored(np.array([[4.0, -inf, -2.0, -2.0]]), 1, groups=2, group_best=2, bias=np.zeros(4))[0].tolist() == [[0]]


def test_quantiser_oracle():
    x = np.array([[1.0, -2.0, 0.5, 0.0], [0.0, 0.0, 0.0, 0.0], [math.inf, 1.0, 0.0, 0.0], [math.nan, 1.0, 0.0, 0.0]])
    c, s = Q.quantize_rows(x)
    assert c.tolist() == [[64, -127, 32, 0], [0] * 4, [0] * 4, [0] * 4]      # 63.5 -> 64, 31.75 -> 32
    assert s[0] == np.float32(2.0) / np.float32(127.0) and s[1] == 0 and np.isnan(s[2:]).all()
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 64))
    c, s = Q.quantize_rows(x)
    assert (np.abs(c).max(axis=1) == 127).all()
    assert (np.abs(c * s[:, None].astype(np.float64) - x) <= 0.5000001 * s[:, None]).all()


def test_tiles_and_products_of_the_oracle():
    rng = np.random.default_rng(2)
    c = rng.integers(-127, 128, (37, 130)).astype(np.int8)
    t = Q.tiles(c).reshape(-1)
    for row, col in ((0, 0), (5, 17), (31, 127), (36, 129), (33, 128), (12, 64)):
        tile = (row // 32) * 2 + col // 128
        i = col % 128
        assert t[tile * 4096 + (i % 64) // 16 * 1024 + (32 * (i // 64) + row % 32) * 16 + i % 16] == c[row, col]
    assert t.astype(np.int64).sum() == c.astype(np.int64).sum()
    x = rng.integers(-127, 128, (3, 130)).astype(np.int8)
    one = np.ones(37, np.float32)
    y = Q.matmul(x, np.ones(3, np.float32), c, one)
    assert y[2, 36] == sum(int(a) * int(b) for a, b in zip(x[2], c[36]))


def test_ffn_oracle_against_a_dense_swiglu():
    rng = np.random.default_rng(3)
    T, H, F = 3, 40, 24
    x = rng.standard_normal((T, H))
    experts = []
    for _ in range(2):
        experts.append([Q.quantize_rows(rng.standard_normal(s) * 0.1) for s in ((F, H), (F, H), (H, F))])
    idx = np.array([[0, 1], [1, 0], [1, -1]])
    gate = rng.random((T, 2))
    y, tol, _, _ = Q.moe_ffn(x, idx, gate, experts, 0.0)
    ref = np.zeros((T, H))
    for t in range(T):
        for j in range(2):
            if idx[t, j] >= 0:
                w1, w3, w2 = (c * s[:, None].astype(np.float64) for c, s in experts[idx[t, j]])
                a = w1 @ x[t]
                ref[t] += gate[t, j] * (w2 @ (a / (1 + np.exp(-a)) * (w3 @ x[t])))
    assert (tol == 0).all()
    assert np.abs(y - ref).max() < 0.05 * np.abs(ref).max()         # apart by the quantisation of x and of the intermediate
    assert (Q.moe_ffn(x, idx, gate, [experts[0], None], 0.0)[0][2] == 0).all()


def test_argument_checks_come_before_device_work():
    lib = B.lib
    rs = lambda logits=P, dtype=1, T=4, E=64, k=8, score=1, groups=8, top=4, best=2, factor=1.0, idx=P, w=P: lib.dymoe_route_scored(
        None, logits, dtype, None, T, E, k, score, groups, top, best, 1, factor, idx, w, None, None)
    assert rs() == B.ENOCTX and rs(T=0, logits=None, idx=None, w=None) == B.ENOCTX
    for bad in (dict(logits=None), dict(idx=None), dict(w=None), dict(dtype=3), dict(T=-1), dict(E=0), dict(k=0), dict(k=65, E=64),
                dict(score=2), dict(groups=0), dict(groups=7), dict(top=0), dict(top=9), dict(best=0), dict(best=3),
                dict(top=1, k=9), dict(factor=0.0), dict(factor=float("nan")), dict(factor=float("inf")), dict(logits=P + 2), dict(idx=P + 2)):
        assert rs(**bad) == B.EINVAL, bad
    assert rs(E=1032) == B.ENOTSUP and rs(E=130, k=65, groups=1, top=1) == B.ENOTSUP and rs(E=130, groups=65, top=65) == B.ENOTSUP
    qr = lambda x=P, dt=0, rows=4, K=100, ldx=100, layout=0, codes=P, scale=P: lib.dymoe_quantize_rows(None, x, dt, rows, K, ldx, layout, codes, scale, None)
    assert qr() == B.ENOCTX and qr(rows=0, x=None, codes=None, scale=None) == B.ENOCTX and qr(x=P + 2) == B.ENOCTX
    for bad in (dict(x=None), dict(codes=None), dict(scale=None), dict(dt=3), dict(rows=-1), dict(K=0), dict(ldx=99), dict(layout=2),
                dict(x=P + 1), dict(codes=P + 8), dict(scale=P + 2), dict(dt=1, x=P + 2)):
        assert qr(**bad) == B.EINVAL, bad
    assert qr(K=B.INT8_MAX_K + 1, ldx=1 << 20) == B.ENOTSUP and qr(rows=1 << 31) == B.ENOTSUP
    need = B.matmul_int8_workspace_bytes(4, 60, 100)
    assert need > 0 and B.matmul_int8_workspace_bytes(-1, 60, 100) == 0 and B.matmul_int8_workspace_bytes(4, 60, B.INT8_MAX_K + 1) == 0
    mm = lambda x=P, xd=0, xs=None, ldx=100, w=P, wsc=P, b=None, T=4, N=60, K=100, od=0, y=P, ldy=60, ws=P, n=need: lib.dymoe_matmul_int8(
        None, x, xd, xs, ldx, w, wsc, b, T, N, K, od, y, ldy, ws, n, None)
    assert mm() == B.ENOCTX and mm(T=0, x=None, y=None, ws=None, n=0) == B.ENOCTX
    assert mm(xd=B.DTYPE_I8, xs=P, ldx=128, ws=None, n=0) == B.ENOCTX
    for bad in (dict(x=None), dict(xd=4), dict(xd=B.DTYPE_I8, ldx=128), dict(xd=B.DTYPE_I8, xs=P, ldx=100), dict(ldx=99), dict(w=None),
                dict(wsc=None), dict(T=-1), dict(N=0), dict(K=0), dict(od=3), dict(y=None), dict(ldy=59), dict(ws=None), dict(w=P + 8),
                dict(ws=P + 16), dict(y=P + 1), dict(b=P + 2)):
        assert mm(**bad) == B.EINVAL, bad
    assert mm(n=need - 1) == B.ENOSPC and mm(K=B.INT8_MAX_K + 1, ldx=1 << 20) == B.ENOTSUP and mm(N=(1 << 24) + 1, ldy=1 << 25) == B.ENOTSUP
    need = B.moe_ffn_int8_workspace_bytes(4, 100, 60, 8, 2)
    assert need > 0 and B.moe_ffn_int8_workspace_bytes(4, 100, 60, 8, 9) == 0
    ff = lambda x=P, xd=0, idx=P, w=P, table=P, T=4, H=100, F=60, E=8, k=2, od=0, y=P, ws=P, n=need: lib.dymoe_moe_ffn_int8(
        None, x, xd, idx, w, table, T, H, F, E, k, od, y, ws, n, None)
    assert ff() == B.ENOCTX and ff(T=0, x=None, idx=None, w=None, y=None) == B.ENOCTX
    for bad in (dict(x=None), dict(xd=3), dict(idx=None), dict(w=None), dict(table=None), dict(T=-1), dict(H=0), dict(F=0), dict(E=0),
                dict(k=0), dict(k=9), dict(od=3), dict(y=None), dict(ws=None), dict(ws=P + 64), dict(table=P + 4), dict(idx=P + 1)):
        assert ff(**bad) == B.EINVAL, bad
    assert ff(n=need - 1) == B.ENOSPC and ff(E=1025, n=1 << 40) == B.ENOTSUP and ff(F=B.INT8_MAX_K + 1, n=1 << 40) == B.ENOTSUP
    assert ff(T=1 << 29, n=1 << 62) == B.ENOTSUP


def test_calls_beyond_a_grid_are_refused():
    lib = B.lib
    rs = lambda T: lib.dymoe_route_scored(None, P, 0, None, T, 8, 2, 1, 1, 1, 1, 1, 1.0, P, P, None, None)
    assert rs((1 << 26) - 1) == B.ENOCTX and rs(1 << 26) == B.ENOTSUP
    ff = lambda T, H, k: lib.dymoe_moe_ffn_int8(None, P, 0, P, P, P, T, H, 8, 8, k, 0, P, P, 1 << 62, None)
    assert ff((1 << 23) - 1, 128, 1) == B.ENOCTX and ff(1 << 23, 128, 1) == B.ENOTSUP
    assert ff((1 << 22) - 1, 1024, 8) == B.ENOCTX and ff(1 << 22, 1024, 8) == B.ENOTSUP
    assert ff((1 << 22) - 1, 2050, 1) == B.ENOTSUP and ff((1 << 20) - 1, 4096, 1) == B.ENOCTX


def test_binding_checks_shapes_and_types():
    class Fake:
        _h, device = None, 0
    call = lambda name, *a, **kw: getattr(B.Context, name)(Fake(), *a, stream=0, **kw)
    f = torch.zeros
    with pytest.raises(TypeError):
        call("route_scored", f(2, 8, dtype=torch.float64), 2)
    with pytest.raises(ValueError):
        call("route_scored", f(2, 8), 2, bias=f(7))
    with pytest.raises(ValueError):
        call("route_scored", f(2, 8), 2, idx=f(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError):
        call("quantize_rows", f(8, 4).t())
    with pytest.raises(ValueError):
        call("quantize_rows", f(1, 4).expand(8, 4))                             # rows that lie on each other
    with pytest.raises(ValueError):
        call("quantize_rows", f(4, 4), out=(f(4, 4, dtype=torch.int8), f(4)))  # codes are padded to 128 columns
    w = (f(32, 128, dtype=torch.int8), f(20))
    with pytest.raises(ValueError):
        call("matmul_int8", f(4, 129), w)
    with pytest.raises(ValueError):
        call("matmul_int8", f(4, 100, dtype=torch.int8), w, x_scale=f(4))
    with pytest.raises(ValueError):
        call("matmul_int8", f(4, 100), w, y=f(4, 21))
    with pytest.raises(ValueError):
        call("moe_ffn_int8", f(4, 16), f(3, 2, dtype=torch.int32), f(4, 2), f(96, dtype=torch.uint8), 16)
    with pytest.raises(ValueError):                                             # everything in order, but not on the context's device
        call("matmul_int8", f(4, 100), w)


def test_layer_class_refuses_experts_of_other_sizes():
    class Ctx:
        def quantize_rows(self, m, layout):
            n, k = -(-m.shape[0] // 32) * 32, -(-m.shape[1] // 128) * 128
            return torch.zeros((n, k), dtype=torch.int8), torch.zeros(m.shape[0])
    ex = lambda H, F: [torch.zeros(F, H), torch.zeros(F, H), torch.zeros(H, F)]
    good = Int8Experts(Ctx(), [ex(40, 24), None, ex(40, 24)], "cpu")
    assert (good.E, good.H, good.F) == (3, 40, 24) and good.table.numel() == 3 * 48
    for bad in ([ex(40, 24), ex(40, 25)], [None], [ex(40, 24)[:2] + [torch.zeros(24, 40)]], [ex(40, 24)[:2]]):
        with pytest.raises(ValueError):
            Int8Experts(Ctx(), bad, "cpu")
    for sizes in ((3, 40, 32), (3, 41, 24), (4, 40, 24)):
        E, H, F = sizes
        layer = Int8MoELayer(Ctx(), 4, H, F, E, 2, device="cpu")
        with pytest.raises(ValueError):
            layer.step(torch.zeros(4, H), good, logits=torch.zeros(4, E))


def test_table_refuses_matrices_that_do_not_fit_together():
    pair = lambda n, k: (torch.zeros((-(-n // 32) * 32, -(-k // 128) * 128), dtype=torch.int8), torch.zeros(n))
    ex = lambda H, F: [pair(F, H), pair(F, H), pair(H, F)]
    assert B.make_int8_table([ex(200, 40), None, ex(200, 40)], "cpu").numel() == 3 * 48
    for bad in ([ex(200, 40), ex(200, 41)], [[pair(40, 200), pair(41, 200), pair(200, 40)]], [[pair(40, 200), pair(40, 300), pair(200, 40)]],
                [[pair(40, 200), pair(40, 200), pair(200, 140)]], [ex(200, 40)[:2]]):
        with pytest.raises(ValueError):
            B.make_int8_table(bad, "cpu")
    with pytest.raises(TypeError):
        B.make_int8_table([[(c.float(), s) for c, s in ex(200, 40)]], "cpu")
