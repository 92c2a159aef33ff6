"""How exact the exponentials of the dense gradient of softmax scores are, for fp32 logits."""
import pytest
import torch

import layer_plain as plain

pytestmark = pytest.mark.gpu

F32 = plain.F32


@pytest.mark.parametrize("E", [64, 100, 256, 512, 1024])
def test_exponentials_of_fp32_logits(E):
    """What reaches the experts that are not chosen is -p_e times one number: divided by exp(x_e) it is the same for all of a row, but for
    the roundings of each exponential and of one product.  The largest logit is 0, so that no difference is rounded; the square of
    exp(x / 2): twice an exponential's two halves of an ulp (2 F32 in each), and the square's own rounding: 5 F32, and 1 of the
    product."""
    import paper_2608_03676_b200 as P
    g = torch.Generator().manual_seed(E)
    N = 64
    x = -40.0 * torch.rand((N, E), generator=g)
    x[:, 0] = 0.0
    topk = torch.zeros((N, 1), dtype=torch.int32)
    dw = 1 + torch.rand((N, 1), generator=g)
    got = P.route_backward(x.cuda(), topk.cuda(), dw.cuda(), renormalise=False).double().cpu()
    ratio = (got / x.double().exp())[:, 1:]
    assert (ratio < 0).all()
    spread = (ratio.max(1).values - ratio.min(1).values) / ratio.mean(1).abs()
    assert float(spread.max()) <= 2 * 6 * F32 * (1 + 2.0 ** -10), float(spread.max() / F32)
