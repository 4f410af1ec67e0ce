"""GPU tests of the router's gradient where what comes from above is no number: masked logits have gradient 0 all the same."""
import math

import pytest
import torch

import test_gpu_route_train as R
from paper_2603_19172_amd import binding as B
from gpu_helpers import DEV
from test_gpu_route_train import ctx  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E,k", [(20, 4), (80, 6), (200, 3), (300, 5), (1000, 8)])
@pytest.mark.parametrize("score", R.SCORES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_masked_logits_whatever_comes_from_above(ctx, E, k, score, dtype):  # noqa: F811
    T = 12
    logits, idx = R.randn(E, T, E, dtype=dtype), R.choose(E, T, E, k)
    mask = torch.rand((T, E), generator=torch.Generator().manual_seed(E)) < 0.4
    mask[3] = True                                             # nothing is left of this row
    mask[:, 0] = False
    mask[3, 0] = True
    mask = mask.to(DEV)
    logits[mask] = -math.inf
    logits[5, mask[5]] = torch.finfo(dtype).min
    idx[:, 0] = 0                                               # a slot whose expert is not masked, others wherever they fall
    counts, _, _ = ctx.route_balance(logits, idx, 0.1, score=score)
    dw = R.randn(2, T, k)
    for bad in (math.nan, math.inf, -math.inf):
        dloss = torch.tensor([bad], device=DEV)
        for renorm in (True, False):
            kw = dict(score=score, renorm=renorm, factor=1.5)
            g = ctx.route_scored_backward(logits, idx, dw=dw, counts=counts, coef=0.1, dloss=dloss, **kw)
            assert (g[mask] == 0).all()
            # and the tokens that the loss has no part in keep theirs
            keep = torch.zeros((T,), dtype=torch.uint8, device=DEV)
            keep[2] = 1
            g = ctx.route_scored_backward(logits, idx, dw=dw, counts=counts, coef=0.1, dloss=dloss, keep=keep, **kw)
            alone = ctx.route_scored_backward(logits, idx, dw=dw, **kw)
            rest = keep == 0
            assert (g[mask] == 0).all() and torch.equal(g[rest], alone[rest]) and not torch.isfinite(g[2][~mask[2]]).all()
            # a weight's gradient that is no number reaches its own token's scores alone, and none that is masked
            d2 = dw.clone()
            d2[4, 0] = bad
            g = ctx.route_scored_backward(logits, idx, dw=d2, **kw)
            others = torch.arange(T, device=DEV) != 4
            assert (g[mask] == 0).all() and torch.equal(g[others], alone[others]) and not torch.isfinite(g[4, 0])
        g = ctx.route_scored_backward(logits, idx, counts=counts, coef=0.1, dloss=dloss, score=score)
        assert (g[mask] == 0).all()
