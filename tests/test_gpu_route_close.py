"""Biased keys next to each other where the router subtracts a far reference from them: the choice is that of 64-bit arithmetic."""
import pytest
import torch

import test_gpu_route as R

pytestmark = pytest.mark.gpu


def near_keys(N, E, at, offset, seed):
    """Rows whose experts `at` have keys 1/2 + offset to about 1e-7, of scores and biases that differ from expert to expert, so that the
    error of an fp32 score can change their order."""
    g = torch.Generator().manual_seed(seed)
    x = torch.zeros((N, E))
    base = 4 * torch.rand(len(at), generator=g) - 2
    x[:, at] = base + 3e-7 * torch.randn((N, len(at)), generator=g)
    bias = torch.full((E,), -3.0)
    bias[at] = (0.5 + offset - torch.sigmoid(base.double())).float()
    return x, bias


@pytest.mark.parametrize("seed", [0, 1])
@pytest.mark.parametrize("k,each,step", [(8, 4, 1), (8, 4, 4), (16, 8, 1), (16, 8, 4)])
def test_a_group_that_is_not_kept_holds_the_largest_key(seed, k, each, step):
    """Group 7's largest key is 999.5, its second largest about -5000: it is not kept, and the kept groups' keys, about 1/2 + 2^-15, are
    999 - 2^-15 below it, in the middle of two fp32 numbers (2^-14 apart there)."""
    E, groups = 256, 8
    at = [32 * g + step * i for g in range(4) for i in range(each)]
    x, bias = near_keys(3000, E, at, 2.0 ** -15, seed)
    bias[224:] = -5000.0
    x[:, 230] = float("inf")                       # its score is one
    bias[230] = 998.5
    kw = dict(score="sigmoid", groups=groups, groups_kept=4, group_top=2)
    R.check(x, R.call(x, k, bias=bias, **kw), k, bias=bias.expand(len(x), -1), **kw)


@pytest.mark.parametrize("seed", [0, 1])
@pytest.mark.parametrize("spread", [1, 4])
def test_the_first_experts_keys_lie_far_below(seed, spread):
    """The first 256 experts' keys are -999.5, those that count are about 1/2 - 2^-15, 1000 - 2^-15 above."""
    E, k = 512, 8
    at = [256 + spread * i for i in range(16)]
    x, bias = near_keys(3000, E, at, -2.0 ** -15, seed)
    bias[:256] = -1000.0
    R.check(x, R.call(x, k, bias=bias, score="sigmoid"), k, bias=bias.expand(len(x), -1), score="sigmoid")


def test_mixed_references():
    """Biases of all sizes at once: references from 2^-10 to 2^20, of either sign, and keys that differ by less than they resolve."""
    g = torch.Generator().manual_seed(3)
    N, E, k = 2000, 256, 8
    for power in range(-10, 21, 3):
        for sign in (-1.0, 1.0):
            at = torch.nonzero(torch.rand(E, generator=g) < 0.2).view(-1)
            x, bias = near_keys(N, E, at, 0.0, power)
            bias[torch.arange(0, 32)] = sign * 2.0 ** power - (5.0 if sign > 0 else 0.0)
            bias[0] = sign * 2.0 ** power
            bias[1:32] -= 2.0 ** power if sign > 0 else 0.0
            kw = dict(score="sigmoid", groups=8, groups_kept=4, group_top=2)
            R.check(x, R.call(x, k, bias=bias, **kw), k, bias=bias.expand(N, -1), **kw)
