"""Tokens of which some entries are delivered and others are not, with more than 32 entries each too."""
import pytest
import torch

import test_gpu_rows as R

pytestmark = pytest.mark.gpu


def positions(B, n, k, left_out, seed):
    """As a dispatcher makes them, single entries left out."""
    g = torch.Generator().manual_seed(seed)
    to = torch.randint(0, 5, (B, n, k), generator=g)
    to[torch.rand((B, n, k), generator=g) < left_out] = 5
    to = to.view(B, n * k)
    order = torch.argsort(to, dim=1, stable=True)
    perm = torch.empty_like(order).scatter_(1, order, torch.arange(n * k).expand(B, -1).contiguous())
    counts = torch.zeros((B, 6), dtype=torch.int64).scatter_add_(1, to, torch.ones_like(to))[:, :5]
    return perm.view(B, n, k).int(), counts.int().contiguous()


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("B,n,k,D", [(2, 9, 33, 96), (1, 7, 64, 264), (3, 5, 40, 77), (1, 700, 64, 64), (2, 6, 8, 4096), (1, 9, 63, 1111), (1, 3, 2, 7)])
@pytest.mark.parametrize("left_out", [0.1, 0.5, 0.95])
def test_entries_left_out(dtype, B, n, k, D, left_out):
    import numpy as np
    import layer_plain as plain
    import paper_2608_03676_b200 as P
    perm, counts = positions(B, n, k, left_out, seed=k + D)
    x, r, dout = (R.rand(B, n, D, dtype=dtype, seed=i) for i in range(3))
    y, w = R.rand(B, n * k, D, dtype=dtype, seed=3), R.rand(B, n, k, dtype=torch.float32, seed=4)
    for b in range(B):
        y[b, int(counts[b].sum()):] = float("nan")
    seven = torch.full((B, n * k, D), 7.0, dtype=dtype)
    sent = P.send(x.cuda(), perm.cuda(), counts=counts.cuda(), out=dict(rows=seven.cuda()))
    want = plain.send(x.double().numpy(), perm.numpy(), counts.double().numpy(), seven.double().numpy().copy())
    assert (sent["rows"].double().cpu().numpy() == want).all()
    out = P.combine(y.cuda(), perm.cuda(), weights=w.cuda(), counts=counts.cuda(), residual=r.cuda())
    R.check_combine(out["out"], y, perm, w, counts, r)
    got = P.combine_backward(dout.cuda(), perm.cuda(), y=y.cuda(), weights=w.cuda(), counts=counts.cuda(), out=dict(dy=seven.cuda()))
    R.check_backward(got, dout, y, perm, w, counts, seven)
    delivered = plain.delivered(perm.numpy(), counts.numpy())
    assert (got["dweights"].cpu().numpy()[~delivered] == 0).all()
    for t in (sent, out, got):
        assert t["info"].tolist() == [0] * B
