"""Performance cases of the operators around the planner in a mixture-of-experts layer: what a training or serving step
asks of them, over the range of sizes they are used at.

A case is one call through the package's public entry points.  Kinds:
  norm          `rms_norm`: residual's addition, RMS norm, the normalised rows in the inputs' type and in 8 bits with scales
  norm_grad     `rms_norm_backward`
  route         `route`: router logits to the routing table that `Planner.plan` takes, and the experts' weights
  route_grad    `route_backward`
  send          `send`: rows to the send buffer by the positions that `Planner.dispatch` gives
  combine       `combine`: weighted sum of the rows that came back, and the residual
  combine_grad  `combine_backward`

With `own` false the operators are computed by elementary torch operations instead.
"""
import math

import torch

#: whether run() calls the package's kernels
own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}
E4M3_MAX = 448.0
LEAST_SCALE = 2.0 ** -126


# ---------------------------------------------------------------------------------------------------------------------
# the cases


def _norm(name, N, D, dtype, residual=True, group=128, grad=False):
    """group: columns that share a scale of the 8-bit rows (0: no 8-bit rows)."""
    c = dict(kind="norm_grad" if grad else "norm", N=N, D=D, dtype=dtype, residual=residual, group=0 if grad else group)
    if name:
        c["name"] = name
    return c


def _route(name, L, T, E, k, dtype, score, bias=False, groups=1, kept=1, top=1, renormalise=True, scale=1.0, padded=0.0,
           grad=False):
    """top: how many of a group's largest keys make its score; padded: share of the tokens that are padding."""
    c = dict(kind="route_grad" if grad else "route", L=L, T=T, E=E, k=k, dtype=dtype, score=score, bias=bias,
             groups=groups, kept=kept, top=top, renormalise=renormalise, scale=scale, padded=padded)
    if name:
        c["name"] = name
    return c


def _rows(name, kind, B, n, k, D, dtype, ranks, weights=True, residual=True, padded=0.0):
    """B send buffers of n tokens with k entries each, to `ranks` ranks.  dtype e4m3: with a scale per 128 columns."""
    c = dict(kind=kind, B=B, n=n, k=k, D=D, dtype=dtype, ranks=ranks, weights=weights, residual=residual, padded=padded)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # four sequences that each decode one token: nothing but latency
        _norm("norm_4_tokens", 4, 4096, "bf16"),
        # a rank's tokens of a training step, on their way into the layer
        _norm("norm_8192_tokens", 8192, 4096, "bf16"),
        # and the gradients on their way back
        _norm("norm_grad_8192_tokens", 8192, 4096, "bf16", grad=True),
        # sizes that are no multiple of anything, in the type that small models train in
        _norm("norm_grad_ragged", 7007, 1111, "f32", grad=True),
        # the router of the four decoded tokens: biased sigmoid scores, the best four of eight groups
        _route("route_4_tokens", 1, 4, 256, 8, "f32", "sigmoid", True, 8, 4, 2, True, 2.5),
        # the same router for a rank's tokens of a training step
        _route("route_8192_tokens", 1, 8192, 256, 8, "f32", "sigmoid", True, 8, 4, 2, True, 2.5),
        # all ranks' tokens of one layer of the 256-rank job, as a planner that sees the whole job is fed
        _route("route_1048576_tokens", 1, 1048576, 128, 8, "bf16", "softmax"),
        # the gradient of softmax scores that are not renormalised: dense over the experts, two layers at once
        _route("route_grad_dense", 2, 65536, 256, 8, "bf16", "softmax", renormalise=False, grad=True),
        # a rank's tokens in 8 bits with their scales, eight copies each, to 64 ranks
        _rows("send_8192_tokens_8_bit", "send", 1, 8192, 8, 4096, "e4m3", 64),
        # the rows that came back, weighted and added to the residual
        _rows("combine_8192_tokens", "combine", 1, 8192, 8, 4096, "bf16", 64),
        # a few padded sequences of odd sizes
        _rows("combine_ragged", "combine", 3, 37, 6, 1111, "f16", 8, padded=0.2),
        # the gradients of the weighted sum: rows for the send buffer, and the router's weights
        _rows("combine_grad_8192_tokens", "combine_grad", 1, 8192, 8, 4096, "bf16", 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case, no larger than the largest listed one of its kind."""
    kind = rng.choice(("norm", "norm_grad", "route", "route", "route_grad", "send", "combine", "combine_grad"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if kind.startswith("norm"):
        D = _log(rng, 64, 16384)
        if rng.random() < 0.7:
            D = max(64, D // 64 * 64)
        N = _log(rng, 1, max(1, min(65536, 8192 * 4096 // D)))
        return _norm(None, N, D, dtype, rng.random() < 0.8, rng.choice((0, 32, 64, 128, 128, 256)), kind == "norm_grad")
    if kind.startswith("route"):
        E = _log(rng, 4, 1024)
        if rng.random() < 0.7:
            E = max(8, E // 8 * 8)
        k = min(E, rng.choice((1, 2, 4, 6, 8, 8, 8, 10, 16)))
        score = rng.choice(("softmax", "sigmoid"))
        bias = rng.random() < 0.5
        groups = kept = top = 1
        if E % 8 == 0 and rng.random() < 0.5:
            groups = rng.choice((2, 4, 8))
            kept = rng.randrange(1, groups + 1)
            while kept * (E // groups) < k:
                kept += 1
            top = rng.choice((1, 2))
        L = _log(rng, 1, 8)
        T = _log(rng, 1, max(1, 1048576 * 128 // (E * L * (4 if kind == "route_grad" else 1))))
        renormalise = k > 1 and rng.random() < 0.7               # (one renormalised weight is the scale, whatever the score)
        return _route(None, L, T, E, k, dtype, score, bias, groups, kept, top, renormalise,
                      rng.choice((1.0, 2.5)), rng.choice((0.0, 0.0, 0.1)), kind == "route_grad")
    D = _log(rng, 64, 8192)
    if rng.random() < 0.7:
        D = max(64, D // 64 * 64)
    B, k = _log(rng, 1, 8), rng.choice((1, 2, 4, 6, 8))
    n = _log(rng, 1, max(1, min(16384, 8192 * 8 * 4096 // (B * k * D))))
    if kind == "send" and rng.random() < 0.5:
        dtype = "e4m3"
    return _rows(None, kind, B, n, k, D, dtype, rng.choice((1, 8, 16, 64)), rng.random() < 0.8, rng.random() < 0.7,
                 rng.choice((0.0, 0.0, 0.2)))


# ---------------------------------------------------------------------------------------------------------------------
# inputs


def _lowest(dtype):
    return torch.finfo(dtype).min


def _prepare_norm(case, g):
    N, D, dt = case["N"], case["D"], DTYPES[case["dtype"]]
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    spread = torch.exp(0.5 * rand(D))                          # some columns are larger than others, as in a trained model
    s = dict(case=case, weight=(1.0 + 0.1 * rand(D)).to(dt))
    if case["kind"] == "norm":
        s["x"] = (0.3 * rand(N, D)).to(dt)
        s["residual"] = (rand(N, D) * spread).to(dt) if case["residual"] else None
        empty = lambda shape, t: torch.empty(shape, dtype=t, device="cuda")
        s["out"] = dict(y=empty((N, D), dt), rstd=empty((N,), torch.float32))
        if case["residual"]:
            s["out"]["h"] = empty((N, D), dt)
        if case["group"]:
            s["out"]["q"] = empty((N, D), torch.float8_e4m3fn)
            s["out"]["scales"] = empty((N, -(-D // case["group"])), torch.float32)
        return s
    s["h"] = (rand(N, D) * spread).to(dt)
    s["dy"] = rand(N, D).to(dt)
    s["dh"] = rand(N, D).to(dt) if case["residual"] else None
    s["rstd"] = (s["h"].double().square().mean(1) + 1e-6).rsqrt().float()
    s["out"] = dict(dx=torch.empty((N, D), dtype=dt, device="cuda"), dweight=torch.empty((D,), device="cuda"))
    return s


def _prepare_route(case, g):
    L, T, E, k, dt = case["L"], case["T"], case["E"], case["k"], DTYPES[case["dtype"]]
    logits = torch.randn((L, T, E), generator=g, device="cuda")
    logits += 0.7 * torch.randn((L, 1, E), generator=g, device="cuda")           # popular and unpopular experts
    s = dict(case=case, logits=logits.to(dt), bias=None, mask=None)
    if case["bias"]:
        s["bias"] = 0.05 * torch.randn((L, E), generator=g, device="cuda")
    if case["padded"]:
        s["mask"] = torch.rand((L, T), generator=g, device="cuda") >= case["padded"]
    if case["kind"] == "route":
        s["out"] = dict(topk=torch.empty((L, T, k), dtype=torch.int32, device="cuda"),
                        weights=torch.empty((L, T, k), device="cuda"))
        return s
    topk = torch.empty((L, T, k), dtype=torch.int32, device="cuda")
    for l in range(L):
        topk[l] = torch.topk(logits[l], k, dim=-1).indices
    if s["mask"] is not None:
        topk.masked_fill_(~s["mask"][..., None], -1)
    s["topk"] = topk
    s["dweights"] = torch.randn((L, T, k), generator=g, device="cuda")
    s["out"] = torch.empty_like(s["logits"])
    return s


def _prepare_rows(case, g):
    B, n, k, D, R = case["B"], case["n"], case["k"], case["D"], case["ranks"]
    # positions as a dispatcher makes them: entries sorted by destination rank, undeliverable ones last
    to = torch.randint(0, R, (B, n, k), generator=g, device="cuda")
    if case["padded"]:
        to.masked_fill_((torch.rand((B, n), generator=g, device="cuda") < case["padded"])[..., None], R)
    to = to.view(B, n * k)
    order = torch.argsort(to, dim=1, stable=True)
    perm = torch.empty_like(order).scatter_(1, order, torch.arange(n * k, device="cuda").expand(B, -1).contiguous())
    counts = torch.zeros((B, R + 1), dtype=torch.int64, device="cuda").scatter_add_(1, to, torch.ones_like(to))
    s = dict(case=case, perm=perm.int().view(B, n, k), counts=counts[:, :R].int().contiguous())
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    dt = DTYPES.get(case["dtype"])
    info = torch.zeros((B,), dtype=torch.int32, device="cuda")
    weights = torch.rand((B, n, k), generator=g, device="cuda") / k if case["weights"] else None
    if case["kind"] == "send":
        s["scales"] = None
        s["out"] = dict(info=info)
        if case["dtype"] == "e4m3":
            groups = -(-D // 128)
            s["x"] = (100.0 * rand(B, n, D)).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
            s["scales"] = torch.rand((B, n, groups), generator=g, device="cuda") * 0.01
            s["out"]["scales"] = torch.zeros((B, n * k, groups), device="cuda")
            s["out"]["rows"] = torch.zeros((B, n * k, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        else:
            s["x"] = rand(B, n, D).to(dt)
            s["out"]["rows"] = torch.zeros((B, n * k, D), dtype=dt, device="cuda")
        return s
    s["weights"] = weights
    s["y"] = rand(B, n * k, D).to(dt)
    if case["kind"] == "combine":
        s["residual"] = rand(B, n, D).to(dt) if case["residual"] else None
        s["out"] = dict(out=torch.empty((B, n, D), dtype=dt, device="cuda"), info=info)
        return s
    s["dout"] = rand(B, n, D).to(dt)
    s["out"] = dict(dy=torch.zeros((B, n * k, D), dtype=dt, device="cuda"), info=info)
    if case["weights"]:
        s["out"]["dweights"] = torch.empty((B, n, k), device="cuda")
    return s


def _family(case):
    return case["kind"].split("_")[0]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    make = {"norm": _prepare_norm, "route": _prepare_route}.get(_family(case), _prepare_rows)
    return make(case, g)


# ---------------------------------------------------------------------------------------------------------------------
# plain forms


def _plain_norm(s):
    c, dt = s["case"], s["x"].dtype
    h = s["x"]
    if s["residual"] is not None:
        h = (s["x"].float() + s["residual"].float()).to(dt)
    hf = h.float()
    rstd = 1.0 / torch.sqrt((hf * hf).mean(1) + 1e-6)
    y = hf * rstd[:, None] * s["weight"].float()
    out = dict(y=y.to(dt), rstd=rstd)
    if s["residual"] is not None:
        out["h"] = h
    if c["group"]:
        N, D, gr = c["N"], c["D"], c["group"]
        G = -(-D // gr)
        yp = torch.zeros((N, G * gr), device="cuda")
        yp[:, :D] = y
        yp = yp.view(N, G, gr)
        scales = torch.clamp(yp.abs().amax(2) / E4M3_MAX, min=LEAST_SCALE)
        out["q"] = (yp / scales[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(N, G * gr)[:, :D].contiguous()
        out["scales"] = scales
    return out


def _plain_norm_grad(s):
    h, dy, w, r = s["h"].float(), s["dy"].float(), s["weight"].float(), s["rstd"][:, None]
    xhat = h * r
    g = dy * w
    dx = r * (g - xhat * (g * xhat).mean(1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return dict(dx=dx.to(s["h"].dtype), dweight=(dy * xhat).sum(0))


def _open_logits(logits):
    """Logits in 64 bits (keys lie next to each other), infinities as the largest finite value, and which experts are open."""
    big = torch.finfo(logits.dtype).max
    is_open = logits > _lowest(logits.dtype)
    x = logits.double().clamp(max=big)
    return torch.where(is_open, x, torch.full_like(x, -math.inf)), is_open


def _plain_scores(x, is_open, score):
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-x))
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    e = torch.exp(x - top)
    return e / e.sum(-1, keepdim=True).clamp(min=1e-300)


def _plain_weights(x, score, scores, topk, renormalise, scale):
    """Weights of the chosen experts; renormalised ones relative to the largest chosen score, so that no sum vanishes."""
    chosen = topk >= 0
    at = topk.clamp(min=0).long()
    if not renormalise:
        return torch.where(chosen, scores.gather(-1, at), torch.zeros((), dtype=scores.dtype, device="cuda")) * scale
    lx = x.gather(-1, at)
    if score == "sigmoid":                                                       # logarithm of the score
        lx = torch.clamp(lx, max=0.0) - torch.log1p(torch.exp(-lx.abs()))
    lx = torch.where(chosen, lx, torch.full_like(lx, -math.inf))
    top = lx.amax(-1, keepdim=True)
    e = torch.exp(lx - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    return e / e.sum(-1, keepdim=True).clamp(min=1e-300) * scale


def _plain_route(s):
    c = s["case"]
    x, is_open = _open_logits(s["logits"])
    scores = _plain_scores(x, is_open, c["score"])
    none = torch.full((), -math.inf, dtype=torch.float64, device="cuda")
    keys = x if s["bias"] is None else torch.where(is_open, scores + s["bias"].double()[:, None, :], none)
    if c["groups"] > 1:
        G = c["groups"]
        gk = scores if s["bias"] is None else keys
        gk = torch.where(is_open, gk, none).view(c["L"], c["T"], G, c["E"] // G)
        best = torch.sort(gk, dim=-1, descending=True, stable=True).values[..., :c["top"]]
        group = torch.where(torch.isinf(best), torch.zeros_like(best), best).sum(-1)
        group = torch.where(torch.isinf(best[..., 0]), none, group)
        first = torch.sort(group, dim=-1, descending=True, stable=True).indices[..., :c["kept"]]
        kept = torch.zeros_like(group, dtype=torch.bool).scatter_(-1, first, True)
        kept = kept[..., None].expand(-1, -1, -1, c["E"] // G).reshape(c["L"], c["T"], c["E"])
        keys = torch.where(kept, keys, none)
    best, at = torch.sort(keys, dim=-1, descending=True, stable=True)
    topk = torch.where(torch.isinf(best[..., :c["k"]]), -1, at[..., :c["k"]])
    if s["mask"] is not None:
        topk = torch.where(s["mask"][..., None], topk, -1)
    w = _plain_weights(x, c["score"], scores, topk, c["renormalise"], c["scale"])
    return dict(topk=topk.int(), weights=w.float())


def _plain_route_grad(s):
    c, scale = s["case"], s["case"]["scale"]
    x, is_open = _open_logits(s["logits"])
    x, chosen, at = x.float(), s["topk"] >= 0, s["topk"].clamp(min=0).long()
    g = torch.where(chosen, s["dweights"], torch.zeros((), device="cuda"))
    if c["renormalise"]:
        q = _plain_weights(x, c["score"], None, s["topk"], True, 1.0)
        d = scale * q * (g - (g * q).sum(-1, keepdim=True))
        if c["score"] == "sigmoid":
            d = d / (1.0 + torch.exp(x.gather(-1, at)))
    elif c["score"] == "sigmoid":
        lx = x.gather(-1, at)
        d = scale * g / (1.0 + torch.exp(-lx)) / (1.0 + torch.exp(lx))
    else:
        p = _plain_scores(x, is_open, "softmax")
        pg = p.gather(-1, at) * g
        out = -scale * p * pg.sum(-1, keepdim=True)
        return out.scatter_add_(-1, at, scale * pg).to(s["logits"].dtype)
    d = torch.where(chosen, d, torch.zeros_like(d))
    return torch.zeros_like(x).scatter_add_(-1, at, d).to(s["logits"].dtype)


def _delivered(s):
    """Positions as rows of one table, and which entries are delivered."""
    B, n, k = s["perm"].shape
    valid = s["perm"] < s["counts"].sum(1)[:, None, None]
    at = s["perm"].long() + (torch.arange(B, device="cuda") * (n * k))[:, None, None]
    return at, valid


def _plain_send(s):
    c = s["case"]
    at, valid = _delivered(s)
    src = torch.arange(c["B"] * c["n"], device="cuda").view(c["B"], c["n"], 1).expand(-1, -1, c["k"])[valid]
    rows = torch.zeros((c["B"] * c["n"] * c["k"], c["D"]), dtype=s["x"].dtype, device="cuda")
    if c["dtype"] == "e4m3":
        rows.view(torch.uint8)[at[valid]] = s["x"].view(torch.uint8).view(-1, c["D"])[src]
        scales = torch.zeros((rows.shape[0], s["scales"].shape[-1]), device="cuda")
        scales[at[valid]] = s["scales"].view(-1, s["scales"].shape[-1])[src]
        return dict(rows=rows.view(c["B"], -1, c["D"]), scales=scales.view(c["B"], c["n"] * c["k"], -1))
    rows[at[valid]] = s["x"].view(-1, c["D"])[src]
    return dict(rows=rows.view(c["B"], -1, c["D"]))


def _plain_combine(s):
    c = s["case"]
    at, valid = _delivered(s)
    rows = s["y"].view(-1, c["D"])[at].float()
    w = valid.float() if s["weights"] is None else torch.where(valid, s["weights"], torch.zeros((), device="cuda"))
    out = (rows * w[..., None]).sum(2)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return dict(out=out.to(s["y"].dtype))


def _plain_combine_grad(s):
    c = s["case"]
    at, valid = _delivered(s)
    dout = s["dout"].float()
    w = valid.float() if s["weights"] is None else s["weights"]
    dy = torch.zeros((c["B"] * c["n"] * c["k"], c["D"]), dtype=s["y"].dtype, device="cuda")
    dy[at[valid]] = (w[..., None] * dout[:, :, None, :])[valid].to(s["y"].dtype)
    out = dict(dy=dy.view(c["B"], -1, c["D"]))
    if s["weights"] is not None:
        rows = s["y"].view(-1, c["D"])[at].float()
        out["dweights"] = torch.where(valid, (rows * dout[:, :, None, :]).sum(-1), torch.zeros((), device="cuda"))
    return out


PLAIN = dict(norm=_plain_norm, norm_grad=_plain_norm_grad, route=_plain_route, route_grad=_plain_route_grad,
             send=_plain_send, combine=_plain_combine, combine_grad=_plain_combine_grad)


def _kernels(s):
    import paper_2608_03676_b200 as taot
    c, kind, out = s["case"], s["case"]["kind"], s["out"]
    if kind == "norm":
        return taot.rms_norm(s["x"], s["weight"], eps=1e-6, residual=s["residual"], group=c["group"], out=out)
    if kind == "norm_grad":
        return taot.rms_norm_backward(s["dy"], s["h"], s["weight"], s["rstd"], dh=s["dh"], out=out)
    if kind == "route":
        return taot.route(s["logits"], c["k"], score=c["score"], bias=s["bias"], groups=c["groups"],
                          groups_kept=c["kept"], group_top=c["top"], renormalise=c["renormalise"], scale=c["scale"],
                          mask=s["mask"], out=out)
    if kind == "route_grad":
        return taot.route_backward(s["logits"], s["topk"], s["dweights"], score=c["score"],
                                   renormalise=c["renormalise"], scale=c["scale"], out=out)
    if kind == "send":
        got = taot.send(s["x"], s["perm"], counts=s["counts"], scales=s["scales"], out=out)
    elif kind == "combine":
        got = taot.combine(s["y"], s["perm"], weights=s["weights"], counts=s["counts"], residual=s["residual"], out=out)
    else:
        got = taot.combine_backward(s["dout"], s["perm"], y=s["y"] if s["weights"] is not None else None,
                                    weights=s["weights"], counts=s["counts"], out=out)
    return {name: t for name, t in got.items() if name != "info" and t is not None}


def run(state):
    if own:
        return _kernels(state)
    return PLAIN[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    kind, b = case["kind"], BYTES[case["dtype"]]
    if _family(case) == "norm":
        N, D = case["N"], case["D"]
        if kind == "norm_grad":
            rows = 3 + (1 if case["residual"] else 0)
            return {"bytes": N * D * b * rows + 4 * N + D * (b + 4), "flops": 10 * N * D}
        rows = 4 if case["residual"] else 2
        eight = N * D + 4 * N * -(-D // case["group"]) if case["group"] else 0
        return {"bytes": N * D * b * rows + eight + 4 * N + D * b, "flops": 8 * N * D}
    if _family(case) == "route":
        N, E, k = case["L"] * case["T"], case["E"], case["k"]
        if kind == "route":
            return {"bytes": N * E * b + 8 * N * k + (4 * case["L"] * E if case["bias"] else 0), "flops": 4 * N * E}
        dense = case["score"] == "softmax" and not case["renormalise"]
        return {"bytes": N * E * b + (N * E * b if dense else N * k * b) + 8 * N * k, "flops": (4 * N * E if dense else 8 * N * k)}
    B, n, k, D = case["B"], case["n"], case["k"], case["D"]
    row = D * b
    index = 4 * B * (n * k + case["ranks"])
    weights = 4 * B * n * k if case["weights"] else 0
    if kind == "send":
        row += 4 * -(-D // 128) if case["dtype"] == "e4m3" else 0
        return {"bytes": B * n * (k + 1) * row + index, "flops": 0}
    if kind == "combine":
        return {"bytes": B * n * (k + 1 + (1 if case["residual"] else 0)) * row + index + weights, "flops": 2 * B * n * k * D}
    reads = 1 + (k if case["weights"] else 0)
    return {"bytes": B * n * (k + reads) * row + index + 2 * weights, "flops": B * n * k * D * (3 if case["weights"] else 0)}


# ---------------------------------------------------------------------------------------------------------------------
# the same outputs from the definitions, in 64 bits


def _exact_norm(s):
    c, dt = s["case"], s["x"].dtype
    h = s["x"] if s["residual"] is None else (s["x"].double() + s["residual"].double()).to(dt)
    v = h.double()
    rstd = torch.pow(torch.linalg.vector_norm(v, dim=1).square() / c["D"] + 1e-6, -0.5)
    y = torch.einsum("nd,n,d->nd", v, rstd, s["weight"].double())
    out = dict(y=y, rstd=rstd)
    if s["residual"] is not None:
        out["h"] = h.double()
    if c["group"]:
        parts = torch.split(y, c["group"], dim=1)
        scales = [p.abs().max(1).values.div(E4M3_MAX).clamp(min=LEAST_SCALE) for p in parts]
        out["scales"] = torch.stack(scales, 1)
        out["q"] = torch.cat([(p / t[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).double()
                              for p, t in zip(parts, scales)], 1)
    return out


def _exact_norm_grad(s):
    N, D = s["h"].shape
    dx, dw = torch.empty((N, D), dtype=torch.float64, device="cuda"), torch.zeros(D, dtype=torch.float64, device="cuda")
    w = s["weight"].double()
    for a in range(0, N, 1024):
        part = slice(a, a + 1024)
        h, dy, r = s["h"][part].double(), s["dy"][part].double(), s["rstd"][part].double()
        inner = torch.einsum("nd,nd,d->n", dy, h, w)
        dx[part] = torch.einsum("nd,d,n->nd", dy, w, r) - h * (r ** 3 * inner / D)[:, None]
        if s["dh"] is not None:
            dx[part] += s["dh"][part].double()
        dw += torch.einsum("nd,nd,n->d", dy, h, r)
    return dict(dx=dx, dweight=dw)


def _exact_route(s):
    """Weights for the experts of the plain definition, chosen one after another; the table itself is held to equality."""
    c = s["case"]
    L, T, E, G, k = c["L"], c["T"], c["E"], c["groups"], c["k"]
    topk = torch.full((L * T, k), -1, dtype=torch.int64, device="cuda")
    weights = torch.zeros((L * T, k), dtype=torch.float64, device="cuda")
    low, big = _lowest(s["logits"].dtype), torch.finfo(s["logits"].dtype).max
    flat, step = s["logits"].view(L * T, E), max(1, (1 << 24) // E)
    for a in range(0, L * T, step):
        x = flat[a:a + step]
        shut = ~(x > low)
        x = x.double().clamp(max=big).masked_fill(shut, -1e300)
        score = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.softmax(x, 1)
        score = score.masked_fill(shut, 0.0)
        key = x.clone()
        if s["bias"] is not None:
            layer = torch.arange(a, a + x.shape[0], device="cuda") // T
            key = score + s["bias"].double()[layer]
        key.masked_fill_(shut, -math.inf)
        if G > 1:
            gk = (score if s["bias"] is None else key).masked_fill(shut, -math.inf).view(-1, G, E // G)
            total = torch.zeros(gk.shape[:2], dtype=torch.float64, device="cuda")
            left = gk.clone()
            for j in range(min(c["top"], E // G)):
                m = left.max(2)
                total += torch.where(torch.isinf(m.values), -math.inf if j == 0 else 0.0, m.values)
                left.scatter_(2, m.indices[..., None], -math.inf)
            drop = torch.ones_like(total, dtype=torch.bool)
            for _ in range(c["kept"]):
                m = total.max(1, keepdim=True).values
                first = (torch.cumsum((total == m) & drop, 1) == 1) & (total == m) & drop
                drop &= ~first
                total = total.masked_fill(first, -math.inf)
            key = key.masked_fill(drop[:, :, None].expand(-1, -1, E // G).reshape(-1, E), -math.inf)
        for j in range(k):
            m = key.max(1, keepdim=True).values
            first = torch.argmax((key == m).to(torch.uint8), 1)
            some = ~torch.isinf(m[:, 0])
            topk[a:a + step, j] = torch.where(some, first, -1)
            key.scatter_(1, first[:, None], -math.inf)
        if s["mask"] is not None:
            topk[a:a + step].masked_fill_(~s["mask"].view(-1)[a:a + step, None], -1)
        at = topk[a:a + step]
        v = score.gather(1, at.clamp(min=0)).masked_fill(at < 0, 0.0)
        if c["renormalise"]:
            v = v / v.sum(1, keepdim=True).clamp(min=1e-300)
        weights[a:a + step] = v * c["scale"]
    return dict(topk=topk.int().view(L, T, k), weights=weights.view(L, T, k))


def _exact_route_grad(s):
    """The derivative of the weights by automatic differentiation in 64 bits."""
    c = s["case"]
    flat, topk, dw = s["logits"].view(-1, c["E"]), s["topk"].view(-1, c["k"]).long(), s["dweights"].view(-1, c["k"])
    out = torch.empty(flat.shape, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 24) // c["E"])
    for a in range(0, flat.shape[0], step):
        x = flat[a:a + step].double().requires_grad_()
        score = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.softmax(x, 1)
        at = topk[a:a + step]
        v = score.gather(1, at.clamp(min=0)) * (at >= 0)
        if c["renormalise"]:
            v = v / v.sum(1, keepdim=True).clamp(min=1e-300)
        (v * dw[a:a + step].double()).sum().mul(c["scale"]).backward()
        out[a:a + step] = x.grad
    return out.view(s["logits"].shape)


def _exact_rows(s):
    c = s["case"]
    B, n, k, D = c["B"], c["n"], c["k"], c["D"]
    valid = s["counts"].sum(1).tolist()
    perm = s["perm"].view(B, n * k).long()
    kind = c["kind"]
    if kind == "send":
        rows = torch.zeros((B, n * k, D), dtype=torch.float64, device="cuda")
        out = dict(rows=rows)
        if s["scales"] is not None:
            out["scales"] = torch.zeros((B, n * k, s["scales"].shape[-1]), dtype=torch.float64, device="cuda")
        for b in range(B):
            source = torch.argsort(perm[b])[:valid[b]] // k                      # which token stands at each position
            rows[b, :valid[b]] = s["x"][b].double()[source]
            if s["scales"] is not None:
                out["scales"][b, :valid[b]] = s["scales"][b].double()[source]
        return out
    if kind == "combine":
        out = torch.zeros((B, n, D), dtype=torch.float64, device="cuda")
        for b in range(B):
            order = torch.argsort(perm[b])[:valid[b]]
            v = s["y"][b, :valid[b]].double()
            if s["weights"] is not None:
                v = v * s["weights"][b].reshape(-1).double()[order][:, None]
            out[b].index_add_(0, order // k, v)
        if s["residual"] is not None:
            out += s["residual"].double()
        return dict(out=out)
    dy = torch.zeros((B, n * k, D), dtype=torch.float64, device="cuda")
    dw = torch.zeros((B, n * k), dtype=torch.float64, device="cuda")
    for b in range(B):
        order = torch.argsort(perm[b])[:valid[b]]
        d = s["dout"][b].double()[order // k]
        if s["weights"] is not None:
            dw[b, order] = torch.einsum("nd,nd->n", d, s["y"][b, :valid[b]].double())
            d = d * s["weights"][b].reshape(-1).double()[order][:, None]
        dy[b, :valid[b]] = d
    out = dict(dy=dy)
    if s["weights"] is not None:
        out["dweights"] = dw.view(B, n, k)
    return out


EXACT = dict(norm=_exact_norm, norm_grad=_exact_norm_grad, route=_exact_route, route_grad=_exact_route_grad)


def exact(case, seed):
    return EXACT.get(case["kind"], _exact_rows)(prepare(case, seed))
