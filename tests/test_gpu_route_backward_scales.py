"""The dense gradient of softmax scores over the whole range of its factors."""
import pytest
import torch

import layer_plain as plain

pytestmark = pytest.mark.gpu

F32 = plain.F32


@pytest.mark.parametrize("E", [64, 256, 512, 1024])
@pytest.mark.parametrize("power", list(range(-100, 100, 3)))
def test_gradients_of_equal_logits_are_exact(E, power):
    """Equal logits, E a power of two, one expert chosen: all products are by powers of two, so that no digit may be lost as long as the
    result is a normal number: -g / E^2, and (g - g / E) / E rounded once per operation for the chosen one."""
    import paper_2608_03676_b200 as P
    g = torch.tensor([1.2345678, -1.9999999, 1.0000001, 1.5]) * 2.0 ** power
    x = torch.full((4, E), 0.75)
    topk = torch.tensor([[0], [E - 1], [17], [40]], dtype=torch.int32)
    got = P.route_backward(x.cuda(), topk.cuda(), g[:, None].cuda(), renormalise=False).cpu()
    want = (-g / E / E)[:, None].repeat(1, E)
    assert (want.abs() >= 2.0 ** -126).all()
    chosen = torch.zeros((4, E), dtype=torch.bool).scatter_(1, topk.long(), True)
    assert torch.equal(got[~chosen], want[~chosen])
    exact = (g.double() * (1 - 1 / E) / E)
    assert ((got[chosen].double() - exact).abs() <= F32 * exact.abs()).all()


@pytest.mark.parametrize("power", [-75, -60, -58, -55, -52, -50, -45, -30, 40])
def test_gradients_of_any_size(power):
    import test_gpu_route as R
    g = torch.Generator().manual_seed(power + 100)
    N, E, k = 24, 1024, 8
    x = 0.01 * torch.randn((N, E), generator=g)
    topk = torch.topk(x, k, dim=1).indices.int()
    dw = 2.0 ** power * torch.randn((N, k), generator=g)
    R.check_grad(x, topk, dw, "softmax", False, 1.5)
