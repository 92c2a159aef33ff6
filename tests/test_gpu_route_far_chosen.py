"""Experts that a bias chooses although their sigmoid scores lie far below the largest chosen one: renormalised weights and their
gradients are ratios, which are normal numbers where the scores themselves are not."""
import pytest
import torch

import test_gpu_route as R

pytestmark = pytest.mark.gpu


def far(N, E, k, dtype, seed, top):
    """Logits from 80 below `top` up to it, the first chosen expert at `top`; the bias chooses the first k experts."""
    g = torch.Generator().manual_seed(seed)
    x = top - 80 * torch.rand((N, E), generator=g)
    x[:, 0] = top
    bias = torch.where(torch.arange(E) < k, 8.0 - torch.arange(E) / 8, torch.full((E,), -9.0))
    return x.to(dtype), bias


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("top", [-60.0, -39.0, -31.0, -25.0, -10.0, -0.5, 0.0, 3.0, 30.0])
@pytest.mark.parametrize("N,E,k,groups", [(40, 64, 8, 1), (40, 256, 12, 1), (40, 64, 6, 4), (12, 100, 40, 1)])
def test_weights(dtype, top, N, E, k, groups):
    x, bias = far(N, E, k, dtype, E + k, top)
    for renormalise in (True, False):
        kw = dict(score="sigmoid", renormalise=renormalise, scale=2.5, groups=groups, groups_kept=groups)
        R.check(x, R.call(x, k, bias=bias, **kw), k, bias=bias.expand(N, -1), **kw)


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("top", [-60.0, -31.0, -10.0, 3.0])
def test_weights_of_many_rows_by_logits(dtype, top):
    """A lane per row: rows of eight experts that are all chosen."""
    x, _ = far(60, 8, 8, dtype, 5, top)
    kw = dict(score="sigmoid", renormalise=True)
    topk, w = R.call(x.repeat(1000, 1), 8, **kw)
    R.check(x, (topk[:60], w[:60]), 8, **kw)
    assert (w.reshape(1000, 60, 8) == w[None, :60]).all()


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("top", [-60.0, -39.0, -31.0, -25.0, -10.0, 0.0, 3.0])
@pytest.mark.parametrize("E,k", [(64, 8), (256, 12), (100, 40)])
def test_gradients(dtype, top, E, k):
    x, _ = far(30, E, k, dtype, E, top)
    topk = torch.arange(k, dtype=torch.int32).expand(30, k).contiguous()
    dw = torch.randn((30, k), generator=torch.Generator().manual_seed(k))
    R.check_grad(x, topk, dw, "sigmoid", True, 2.0)
