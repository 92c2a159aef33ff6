"""The layer's operators together with the planner, as a step runs them: norm, router, plan, dispatch, rows out and back, and the
gradients; captured, replayed, on other streams, next to each other."""
import numpy as np
import pytest
import torch

import layer_plain as plain
import workloads as W

pytestmark = pytest.mark.gpu

L, R, E, K, k, per, D = 2, 8, 32, 2, 4, 48, 256
T = R * per


def planner():
    import paper_2608_03676_b200 as P
    return P.Planner(L=L, R=R, E=E, K=K, k=k, T=T, e2r=W.expert_to_rank(E, R, "contiguous"), C=W.cost_matrix(R, 4, (0.0, 1.0, 8.0), None),
                     eps=0.4, max_iters=200)


def inputs(seed, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    skew = torch.linspace(1.5, -1.5, E, device="cuda")
    return dict(x=rand(L, T, D).to(dtype), residual=rand(L, T, D).to(dtype), weight=(1 + 0.1 * rand(D)).to(dtype), gate=rand(L, D, E) / D ** 0.5,
                skew=skew, bias=0.05 * rand(L, E), mask=torch.rand((L, T), generator=g, device="cuda") > 0.1, dout=rand(L, T, D).to(dtype))


KW = dict(score="sigmoid", groups=4, groups_kept=2, group_top=2, scale=2.0)
ROUTE = {name: v for name, v in KW.items() if name in ("score", "scale")}


def forward(pl, s):
    """Everything up to the layer's output; the 'experts' double their rows, in the send buffer's order."""
    import paper_2608_03676_b200 as P
    a = P.rms_norm(s["x"], s["weight"], residual=s["residual"], group=128)
    logits = a["y"].float() @ s["gate"] + s["skew"]
    r = P.route(logits, k, bias=s["bias"], mask=s["mask"], **KW)
    plan = pl.plan(r["topk"])
    d = pl.dispatch(plan["new_idx"])
    perm = d["perm"].view(L, R, per, k)
    buffers = lambda t: t.view((L, R, per) + tuple(t.shape[2:]))
    eight = P.send(buffers(a["q"]), perm, counts=d["send_counts"], scales=buffers(a["scales"]))
    rows = P.send(buffers(a["y"]), perm, counts=d["send_counts"])
    y = rows["rows"] * 2
    out = P.combine(y, perm, weights=buffers(r["weights"]), counts=d["send_counts"], residual=buffers(a["h"]))
    return dict(a=a, logits=logits, r=r, plan=plan, d=d, perm=perm, eight=eight, rows=rows, y=y, out=out)


def backward(s, f):
    import paper_2608_03676_b200 as P
    buffers = lambda t: t.view((L, R, per) + tuple(t.shape[2:]))
    c = P.combine_backward(buffers(s["dout"]), f["perm"], y=f["y"], weights=buffers(f["r"]["weights"]), counts=f["d"]["send_counts"])
    dy = P.combine(c["dy"] * 2, f["perm"], counts=f["d"]["send_counts"])["out"].view(L, T, D)
    dlogits = P.route_backward(f["logits"], f["r"]["topk"], c["dweights"].view(L, T, k), **ROUTE)
    dy = dy + (dlogits @ s["gate"].transpose(1, 2)).to(dy.dtype)
    n = P.rms_norm_backward(dy, f["a"]["h"], s["weight"], f["a"]["rstd"], dh=s["dout"])
    return dict(dlogits=dlogits, dweights=c["dweights"], dx=n["dx"], dweight=n["dweight"])


def test_a_step_gives_what_its_definition_gives():
    """The table is the definition's on the same logits; each padded token is left out all the way; the layer's output is the
    residual plus the doubled rows times the sum of the weights, wherever the planner sent them."""
    import paper_2608_03676_b200 as P
    pl, s = planner(), inputs(1)
    f = forward(pl, s)
    torch.cuda.synchronize()
    want, ww = plain.route(f["logits"].cpu().view(L * T, E), k, bias=s["bias"].cpu().repeat_interleave(T, 0), mask=s["mask"].view(-1).cpu().numpy(), **KW)
    assert (f["r"]["topk"].cpu().numpy().reshape(L * T, k) == want).all()
    pads = int((~s["mask"]).sum()) * k
    assert int(f["d"]["send_counts"].sum()) == L * T * k - pads and pads > 0
    assert all(int(v) & P.INFO_BAD_INDEX for v in f["plan"]["info"]) and all(int(v) == P.INFO_BAD_INDEX for v in f["d"]["info"])
    assert not f["rows"]["info"].any() and not f["out"]["info"].any() and not f["eight"]["info"].any()
    total = f["r"]["weights"].sum(-1).cpu()
    assert torch.allclose(total, 2.0 * s["mask"].float().cpu(), atol=1e-6)
    y, h, out = (t.double().cpu() for t in (f["a"]["y"], f["a"]["h"], f["out"]["out"].view(L, T, D)))
    want = h + 2 * y * f["r"]["weights"].double().sum(-1, keepdim=True).cpu()
    size = h.abs() + 2 * y.abs() * 2.0
    assert ((out - want).abs() <= (k + 3) * plain.F32 * size).all()
    # 8-bit rows stand at the same positions as the others, with their scales
    valid = int(f["d"]["send_counts"][1, 3].sum())
    back = f["eight"]["rows"][1, 3, :valid].float() * f["eight"]["scales"][1, 3, :valid].repeat_interleave(128, 1)
    full = f["rows"]["rows"][1, 3, :valid]
    most = full.abs().view(valid, 2, 128).amax(2).repeat_interleave(128, 1)
    assert ((back - full).abs() <= 2.0 ** -4 * (1 + 1e-5) * full.abs() + 2.0 ** -10 / 448 * 1.01 * most).all()
    pl.close()


def test_the_gradients_of_a_step_against_automatic_differentiation():
    """The whole chain's gradients against torch's automatic differentiation of its definition in 64 bits."""
    pl, s = planner(), inputs(2)
    f = forward(pl, s)
    got = backward(s, f)
    torch.cuda.synchronize()
    x, res, w, gate = (s[n].double().cpu().requires_grad_() for n in ("x", "residual", "weight", "gate"))
    h = x + res
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-6) * w
    logits = y @ gate + s["skew"].double().cpu()
    at = f["r"]["topk"].cpu().long()
    score = torch.sigmoid(logits).gather(-1, at.clamp(min=0)) * (at >= 0)
    weights = 2.0 * score / score.sum(-1, keepdim=True).clamp(min=1e-300)
    out = h + 2 * y * weights.sum(-1, keepdim=True)
    # (the weights sum to 2, so that dlogits is rounding error here: weigh the places apart, as experts that differ would)
    ((out * s["dout"].double().cpu()).sum()).backward()
    for name, leaf in (("dx", x), ("dweight", w)):
        d, want = got[name].double().cpu(), leaf.grad
        assert float((d - want).norm() / want.norm()) < 1e-5                     # some tens of fp32 roundings, which add up as squares
    assert torch.allclose(x.grad, res.grad)
    pl.close()


def test_a_step_is_captured_and_replayed_on_new_inputs():
    pl, s, other = planner(), inputs(3, torch.bfloat16), inputs(4, torch.bfloat16)
    fresh = {name: t.clone() for name, t in s.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            forward(pl, s)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f = forward(pl, s)
        b = backward(s, f)
    keep = lambda f, b: [t.clone() for t in (f["r"]["topk"], f["r"]["weights"], f["out"]["out"], f["a"]["q"].view(torch.uint8), b["dx"], b["dweight"], b["dlogits"])]
    got = []
    for src in (fresh, other, fresh):
        for name in s:
            s[name].copy_(src[name])
        graph.replay()
        got.append(keep(f, b))
    for src, g in zip((fresh, other, fresh), got):
        ff = forward(pl, src)
        for x, y in zip(g, keep(ff, backward(src, ff))):
            assert torch.equal(x, y)
    pl.close()


def test_calls_on_two_streams_at_once():
    """The operators keep nothing between calls: two streams that run them side by side get what each gets alone."""
    import paper_2608_03676_b200 as P
    g = torch.Generator(device="cuda").manual_seed(5)
    n, Dn, En = 4096, 2048, 128
    sets = []
    for i in range(2):
        rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")
        sets.append(dict(x=rand(n, Dn).bfloat16(), r=rand(n, Dn).bfloat16(), w=(1 + 0.1 * rand(Dn)).bfloat16(), logits=rand(n, En), dw=rand(n, 8)))

    def work(s):
        a = P.rms_norm(s["x"], s["w"], residual=s["r"], group=128)
        b = P.rms_norm_backward(s["x"], a["h"], s["w"], a["rstd"])
        t = P.route(s["logits"], 8)
        d = P.route_backward(s["logits"], t["topk"], s["dw"])
        return [a["y"], a["q"].view(torch.uint8), a["scales"], b["dx"], b["dweight"], t["topk"], t["weights"], d]

    alone = [work(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        both = []
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                both.append(work(s))
        torch.cuda.synchronize()
        for x, y in zip(alone, both):
            assert all(torch.equal(a, b) for a, b in zip(x, y))


def test_two_graphs_share_no_workspace():
    import paper_2608_03676_b200 as P
    g = torch.Generator(device="cuda").manual_seed(6)
    sets = []
    for i in range(2):
        h, dy = (torch.randn((777, 512), generator=g, device="cuda") for _ in range(2))
        sets.append((dy, h, torch.ones(512, device="cuda"), (h.square().mean(1) + 1e-6).rsqrt()))
    want = [P.rms_norm_backward(*s) for s in sets]
    torch.cuda.synchronize()
    graphs, got = [], []
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(P.rms_norm_backward(*s))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a["dx"], b["dx"]) and torch.equal(a["dweight"], b["dweight"])


def test_offsets_beyond_32_bits():
    """Row offsets past 2^31 elements: a buffer of 2^31 + 2^20 16-bit elements, whose last rows are read and written."""
    import paper_2608_03676_b200 as P
    Dn = 1 << 16
    rows = (1 << 15) + 16                          # 2^31 + 2^20 elements, 4.3 GB
    buf = torch.zeros((rows, Dn), dtype=torch.bfloat16, device="cuda")
    buf[-16:] = torch.randn((16, Dn), device="cuda").bfloat16()
    w = torch.ones(Dn, dtype=torch.bfloat16, device="cuda")
    wide = buf.view(rows, Dn)[:, :64]              # rows of 64 columns, 2^16 elements apart
    y = P.rms_norm(wide, w[:64].contiguous())["y"]
    assert torch.equal(y[-16:], P.rms_norm(wide[-16:].contiguous(), w[:64].contiguous())["y"]) and not y[:-16].any()
    perm = torch.arange(rows, dtype=torch.int32, device="cuda").flip(0).contiguous().view(1, rows, 1)
    out = P.combine(wide[None], perm)["out"][0]
    assert torch.equal(out[:16], wide[-16:].flip(0)) and not out[16:].any()
    logits = P.route(wide, 4)["topk"]
    assert torch.equal(logits[-16:], P.route(wide[-16:].contiguous(), 4)["topk"]) and (logits[0].cpu() == torch.arange(4)).all()
    P.send(y[None].flip(1).contiguous(), perm, out=dict(rows=wide[None]))
    assert torch.equal(wide[-16:], y[-16:])


def test_offsets_of_gradients_beyond_32_bits():
    """The same for the backward passes: the last rows of arrays whose rows are 2^16 elements apart."""
    import paper_2608_03676_b200 as P
    Dn, rows, cols = 1 << 16, (1 << 15) + 16, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    a, b = (torch.zeros((rows, Dn), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (a, b):
        t[:, :cols] = torch.randn((rows, cols), generator=g, device="cuda").bfloat16()
    x, y = a[:, :cols], b[:, :cols]
    tail = lambda t: t[-16:].contiguous()
    w, rstd = torch.ones(cols, dtype=torch.bfloat16, device="cuda"), torch.rand(rows, generator=g, device="cuda")
    got = P.rms_norm_backward(y, x, w, rstd, dh=y)
    assert torch.equal(got["dx"][-16:], P.rms_norm_backward(tail(y), tail(x), w, tail(rstd), dh=tail(y))["dx"])
    topk, dw = P.route(x, 4)["topk"], torch.randn((rows, 4), generator=g, device="cuda")
    for renormalise in (True, False):
        want = P.route_backward(tail(x), tail(topk), tail(dw), renormalise=renormalise)
        assert torch.equal(P.route_backward(x, topk, dw, renormalise=renormalise, out=b[:, 64:128])[-16:], want)
    perm = torch.arange(rows, dtype=torch.int32, device="cuda").view(1, rows, 1)
    weights = torch.rand((1, rows, 1), generator=g, device="cuda")
    got = P.combine_backward(x[None], perm, y=y[None], weights=weights, out=dict(dy=b[None, :, 128:192]))
    want = P.combine_backward(tail(x)[None], perm[:, :16].contiguous(), y=tail(y)[None], weights=weights[:, -16:].contiguous())
    assert torch.equal(b[-16:, 128:192], want["dy"][0]) and torch.equal(got["dweights"][0, -16:], want["dweights"][0])
