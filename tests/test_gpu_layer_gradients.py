"""The gradients of a whole step whose experts differ, the router's logits among them, against automatic differentiation in 64 bits."""
import pytest
import torch

import test_gpu_layer_chain as chain

pytestmark = pytest.mark.gpu

L, R, E, k, per, D, T = chain.L, chain.R, chain.E, chain.k, chain.per, chain.D, chain.T


def factors(topk):
    """What each entry's expert multiplies its row with (1 for padding, which no expert gets)."""
    return torch.where(topk >= 0, 0.5 + 0.1 * topk.double(), torch.ones((), dtype=torch.float64, device=topk.device))


def test_experts_that_differ():
    """The rows of the send buffer are multiplied by their expert's factor, so that the places of a token weigh apart and the weights'
    gradient, in the places that the table gives, reaches the logits."""
    import paper_2608_03676_b200 as P
    pl, s = chain.planner(), chain.inputs(7)
    buffers = lambda t: t.view((L, R, per) + tuple(t.shape[2:]))
    a = P.rms_norm(s["x"], s["weight"], residual=s["residual"])
    logits = a["y"] @ s["gate"] + s["skew"]
    r = P.route(logits, k, bias=s["bias"], mask=s["mask"], **chain.KW)
    d = pl.dispatch(pl.plan(r["topk"])["new_idx"])
    perm, counts = d["perm"].view(L, R, per, k), d["send_counts"]
    rows = P.send(buffers(a["y"]), perm, counts=counts)["rows"]
    factor = torch.ones((L, R, per * k), device="cuda").scatter_(2, perm.view(L, R, per * k).long(), buffers(factors(r["topk"]).float()).reshape(L, R, per * k))
    used = torch.arange(per * k, device="cuda") < counts.sum(-1)[..., None]
    rows = torch.where(used[..., None], rows, torch.zeros((), device="cuda"))
    y = rows * factor[..., None]
    out = P.combine(y, perm, weights=buffers(r["weights"]), counts=counts, residual=buffers(a["h"]))["out"].view(L, T, D)

    c = P.combine_backward(buffers(s["dout"]), perm, y=y, weights=buffers(r["weights"]), counts=counts, out=dict(dy=torch.zeros_like(y)))
    dlogits = P.route_backward(logits, r["topk"], c["dweights"].view(L, T, k), **chain.ROUTE)
    dy = P.combine(c["dy"] * factor[..., None], perm, counts=counts)["out"].view(L, T, D) + dlogits @ s["gate"].transpose(1, 2)
    n = P.rms_norm_backward(dy, a["h"], s["weight"], a["rstd"], dh=s["dout"])
    torch.cuda.synchronize()

    x, res, w, gate = (s[name].double().cpu().requires_grad_() for name in ("x", "residual", "weight", "gate"))
    h = x + res
    yy = h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-6) * w
    ll = yy @ gate + s["skew"].double().cpu()
    ll.retain_grad()
    topk = r["topk"].cpu().long()
    score = torch.sigmoid(ll).gather(-1, topk.clamp(min=0)) * (topk >= 0)
    weights = 2.0 * score / score.sum(-1, keepdim=True).clamp(min=1e-300)
    oo = h + yy * (weights * factors(topk)).sum(-1, keepdim=True)
    (oo * s["dout"].double().cpu()).sum().backward()

    # some tens of fp32 roundings on the way of each value, which add up as squares
    assert float((out.double().cpu() - oo).detach().norm() / oo.detach().norm()) < 1e-6
    assert float(ll.grad.norm()) > 1e-3 * float(s["dout"].norm())  # far above rounding error, which is all of it where the experts are alike
    for got, want in ((dlogits, ll.grad), (n["dx"], x.grad), (n["dweight"], w.grad)):
        assert float((got.double().cpu() - want).norm() / want.norm()) < 1e-5
    assert torch.allclose(x.grad, res.grad)
    pl.close()
