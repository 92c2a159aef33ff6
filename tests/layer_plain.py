"""The layer's operators by their definitions, in 64 bits on the CPU, one row after another where that is plainer."""
import math

import numpy as np
import torch

E4M3_MAX = 448.0
LEAST_SCALE = 2.0 ** -126
F32 = 2.0 ** -24                                  # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rms_norm(x, weight, eps, residual=None, group=0):
    """x, residual, weight on the CPU, of the type under test.  h rounded to it; y and scales not rounded."""
    h = x if residual is None else (x.double() + residual.double()).to(x.dtype)
    v = h.double()
    rstd = 1.0 / torch.sqrt((v * v).mean(-1) + eps)
    y = v * rstd[..., None] * weight.double()
    out = dict(h=h, y=y, rstd=rstd)
    if group:
        parts = [p for p in torch.split(y, group, dim=-1)]
        out["scales"] = torch.stack([(p.abs().amax(-1) / E4M3_MAX).clamp(min=LEAST_SCALE) for p in parts], -1)
        out["scale_of"] = torch.cat([s[..., None].expand(p.shape) for s, p in zip(out["scales"].unbind(-1), parts)], -1)
    return out


def rms_norm_backward(dy, h, weight, rstd, dh=None):
    dy, h, w, r = dy.double(), h.double(), weight.double(), rstd.double()[..., None]
    g = dy * w
    dx = r * (g - h * r * (g * h * r).mean(-1, keepdim=True))
    if dh is not None:
        dx = dx + dh.double()
    return dx, (dy * h * r).sum(0)


def open_logits(logits):
    """Logits as 64-bit numbers, minus infinity for closed experts, an infinite one as the largest finite value."""
    info = torch.finfo(logits.dtype)
    x = logits.double().numpy().copy()
    with np.errstate(invalid="ignore"):
        shut = ~(x > info.min)
    x = np.minimum(x, info.max)
    x[shut] = -math.inf
    return x


def scores(x, score):
    """Scores of one row of open logits."""
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-x))
    top = x.max()
    if top == -math.inf:
        return np.zeros_like(x)
    e = np.exp(x - top)
    return e / e.sum()


def chosen_weights(x, at, score, renormalise):
    """Weights (without the scale) of the places `at` (>= 0) of one row."""
    if not renormalise:
        return scores(x, score)[at]
    lx = x[at]
    if score == "sigmoid":                        # the logarithm of the score, so that nothing vanishes
        lx = np.minimum(lx, 0.0) - np.log1p(np.exp(-np.abs(lx)))
    if len(lx) == 0 or lx.max() == -math.inf:
        return np.zeros_like(lx)
    e = np.exp(lx - lx.max())
    return e / e.sum()


def route(logits, k, score="softmax", bias=None, groups=1, groups_kept=1, group_top=1, renormalise=True, scale=1.0, mask=None):
    """logits [N, E], bias [N, E] or None (a row's own), mask [N] or None -> topk [N, k], weights [N, k]."""
    X = open_logits(logits)
    N, E = X.shape
    topk, weights = np.full((N, k), -1, dtype=np.int32), np.zeros((N, k))
    for n in range(N):
        if mask is not None and not mask[n]:
            continue
        x = X[n]
        s = scores(x, score)
        key = x.copy()
        opened = x > -math.inf
        if bias is not None:
            b = bias[n].double().numpy()
            opened &= np.isfinite(b)
            key = np.where(opened, s + np.where(np.isfinite(b), b, 0.0), -math.inf)
        if groups > 1:
            value = key if bias is not None else np.where(opened, s, -math.inf)
            members = value.reshape(groups, E // groups)
            total = []
            for g in range(groups):
                best = sorted([v for v in members[g] if v > -math.inf], reverse=True)[:group_top]
                total.append(sum(best) if best else -math.inf)
            first = sorted(range(groups), key=lambda g: (-total[g], g))[:groups_kept]
            kept = np.zeros(groups, dtype=bool)
            kept[first] = True
            key = np.where(np.repeat(kept, E // groups), key, -math.inf)
        order = np.argsort(-key, kind="stable")[:k]
        at = np.array([e for e in order if key[e] > -math.inf], dtype=np.int64)
        topk[n, :len(at)] = at
        weights[n, :len(at)] = scale * chosen_weights(x, at, score, renormalise)
    return topk, weights


def route_backward(logits, topk, dweights, score, renormalise, scale):
    """By the formula.  Also a bound on the sum of the magnitudes that each element is made of, for tolerances."""
    X = open_logits(logits)
    N, E = X.shape
    out, size = np.zeros((N, E)), np.zeros((N, E))
    for n in range(N):
        x = X[n]
        valid = (topk[n] >= 0) & (topk[n] < E)
        at, g = topk[n][valid], scale * dweights[n][valid].astype(np.float64)
        if renormalise:
            q = chosen_weights(x, at, score, True)
            d, m = q * (g - (q * g).sum()), q * (np.abs(g) + np.abs(q * g).sum())
        elif score == "softmax":
            p = scores(x, score)
            out[n] -= p * (p[at] * g).sum()
            size[n] += p * np.abs(p[at] * g).sum()
            d = p[at] * g
            m = np.abs(d)
        else:
            d = scores(x, score)[at] * g
            m = np.abs(d)
        if score == "sigmoid":
            with np.errstate(over="ignore"):
                rest = np.where(x[at] > -math.inf, 1.0 / (1.0 + np.exp(x[at])), 0.0)
            d, m = d * rest, m * rest
        np.add.at(out[n], at, d)
        np.add.at(size[n], at, m)
    return out, size


def weights_of_table(logits, topk, score, renormalise, scale):
    """The weights [N, k] of a given table, for differences."""
    X = open_logits(logits)
    w = np.zeros(topk.shape)
    for n in range(X.shape[0]):
        valid = (topk[n] >= 0) & (topk[n] < X.shape[1])
        w[n, valid] = scale * chosen_weights(X[n], topk[n][valid], score, renormalise)
    return w


def delivered(perm, counts):
    """Which entries of perm [B, n, k] are delivered."""
    B, n, k = perm.shape
    limit = np.full(B, n * k) if counts is None else np.minimum(counts.sum(-1), n * k)
    return (perm >= 0) & (perm < limit[:, None, None])


def send(x, perm, counts, rows):
    """rows [B, n*k, D] is changed; whatever the type."""
    ok = delivered(perm, counts)
    for b, t, j in zip(*np.nonzero(ok)):
        rows[b, perm[b, t, j]] = x[b, t]
    return rows


def combine(y, perm, weights, counts, residual):
    """Also the sum of magnitudes per element."""
    B, n, k = perm.shape
    out = np.zeros((B, n, y.shape[-1])) if residual is None else residual.copy()
    size = np.abs(out)
    for b, t, j in zip(*np.nonzero(delivered(perm, counts))):
        term = (1.0 if weights is None else weights[b, t, j]) * y[b, perm[b, t, j]]
        out[b, t] += term
        size[b, t] += np.abs(term)
    return out, size


def combine_backward(dout, y, perm, weights, counts, dy):
    """dy [B, n*k, D] is changed.  Returns it, dweights and the sums of magnitudes of the latter."""
    dw, size = np.zeros(perm.shape), np.zeros(perm.shape)
    for b, t, j in zip(*np.nonzero(delivered(perm, counts))):
        at = perm[b, t, j]
        dy[b, at] = (1.0 if weights is None else weights[b, t, j]) * dout[b, t]
        if y is not None:
            dw[b, t, j] = (dout[b, t] * y[b, at]).sum()
            size[b, t, j] = np.abs(dout[b, t] * y[b, at]).sum()
    return dy, dw, size
