"""Routing to experts and the gradient of the weights, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import layer_plain as plain

pytestmark = pytest.mark.gpu

F32 = plain.F32
TYPES = [torch.float32, torch.bfloat16, torch.float16]
INF, NAN = float("inf"), float("nan")


def call(logits, k, bias=None, mask=None, **kw):
    import paper_2608_03676_b200 as P
    out = P.route(logits.cuda(), k, bias=None if bias is None else bias.cuda(), mask=None if mask is None else mask.cuda(), **kw)
    return out["topk"].cpu().numpy(), out["weights"].cpu().numpy()


def spread(logits, topk):
    """The largest distance of a chosen logit from the row's largest one, per entry."""
    x = plain.open_logits(logits)
    top = x.max(1, keepdims=True)
    at = np.maximum(topk, 0)
    d = top - np.take_along_axis(x, at, 1)
    return np.where((topk >= 0) & np.isfinite(d), d, 0.0)


def check(logits, got, k, bias=None, mask=None, **kw):
    topk, w = got
    N, E = logits.shape
    topk, w = topk.reshape(N, k), w.reshape(N, k)
    want, ww = plain.route(logits, k, bias=bias, mask=None if mask is None else mask.numpy(), **kw)
    assert (topk == want).all(), [(n, topk[n], want[n]) for n in np.nonzero((topk != want).any(1))[0][:4]]
    # the difference from the largest logit is rounded, exp follows its argument; exp, sums of up to 1024 by a tree, divisions
    rel = (2 * spread(logits, want) + 64) * F32
    assert (np.abs(w - ww) <= rel * np.abs(ww) + 2.0 ** -125 * kw.get("scale", 1.0)).all(), float(np.abs(w - ww).max())


def make(N, E, dtype, seed=0, scale=1.5):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn((N, E), generator=g)).to(dtype)


SHAPES = [(1, 1, 1), (5, 2, 1), (3, 4, 4), (9, 8, 2), (33, 32, 2), (31, 64, 8), (65, 72, 6), (17, 100, 7), (130, 128, 8), (66, 256, 8),
          (21, 257, 5), (20, 512, 8), (11, 1000, 10), (13, 1024, 8), (7, 1024, 64), (9, 40, 40), (6, 96, 33), (12, 256, 16), (258, 256, 9)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,E,k", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route(dtype, N, E, k, score, renormalise):
    x = make(N, E, dtype, seed=E + k)
    kw = dict(score=score, renormalise=renormalise, scale=1.5)
    check(x, call(x, k, **kw), k, **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,E,k", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_with_bias(dtype, N, E, k, score):
    x = make(N, E, dtype, seed=E + k + 1)
    bias = 0.1 * torch.randn(E, generator=torch.Generator().manual_seed(E))
    check(x, call(x, k, bias=bias, score=score), k, bias=bias.expand(N, -1), score=score)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,E,k,groups,kept", [(40, 256, 8, 8, 4), (33, 64, 4, 8, 3), (21, 72, 6, 9, 5), (17, 12, 3, 12, 3), (9, 64, 2, 64, 7),
                                               (30, 128, 8, 2, 1), (12, 1024, 8, 32, 4), (25, 160, 6, 8, 3), (19, 256, 8, 4, 2), (7, 512, 8, 8, 4),
                                               (14, 536, 8, 8, 2), (9, 98, 6, 2, 1), (16, 268, 8, 4, 3), (9, 40, 16, 4, 4), (6, 6, 2, 2, 1), (8, 656, 8, 4, 4),
                                               (7, 1000, 16, 8, 3), (10, 72, 6, 8, 5), (11, 256, 16, 8, 4), (10, 512, 40, 16, 9), (23, 128, 6, 16, 4), (12, 1024, 8, 64, 3), (8, 40, 2, 20, 2)])
@pytest.mark.parametrize("score,with_bias,top", [("sigmoid", True, 2), ("softmax", False, 1), ("sigmoid", False, 2), ("softmax", True, 1)])
def test_route_by_groups(dtype, N, E, k, groups, kept, score, with_bias, top):
    x = make(N, E, dtype, seed=E + groups)
    bias = 0.1 * torch.randn(E, generator=torch.Generator().manual_seed(E)) if with_bias else None
    kw = dict(score=score, groups=groups, groups_kept=kept, group_top=top, scale=2.5)
    check(x, call(x, k, bias=bias, **kw), k, bias=None if bias is None else bias.expand(N, -1), **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("score,with_bias,groups,kept", [("softmax", False, 1, 1), ("sigmoid", True, 1, 1), ("sigmoid", True, 8, 4), ("softmax", True, 8, 4),
                                                         ("softmax", False, 8, 4)])
@pytest.mark.parametrize("E,k", [(64, 6), (128, 8), (256, 8), (256, 12), (512, 8)])
def test_route_ties(dtype, score, with_bias, groups, kept, E, k):
    """Logits on a coarse grid: many equal keys and equal groups, which go to the lowest index."""
    N = 64
    g = torch.Generator().manual_seed(E + k)
    x = (torch.randint(-4, 4, (N, E), generator=g) / 4).to(dtype)
    x[0] = 0.5                                     # all equal
    x[1] = 0.0
    x[2] = -0.0
    x[3, ::2] = -0.0                               # both zeros are the same number
    x[3, 1::2] = 0.0
    bias = torch.randint(-1, 2, (E,), generator=g) / 8 if with_bias else None
    # (sums of two biased keys can be equal in the reals and differ in the last bit: then there is no tie to speak of)
    kw = dict(score=score, groups=groups, groups_kept=kept, group_top=1 if with_bias else 2)
    check(x, call(x, k, bias=bias, **kw), k, bias=None if bias is None else bias.expand(N, -1), **kw)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,kept", [(1, 1), (8, 4)])
@pytest.mark.parametrize("E,k", [(64, 8), (256, 8), (256, 16), (1024, 8)])
def test_route_keys_next_to_each_other(score, groups, kept, E, k):
    """fp32 logits and biases whose keys differ by far less than fp32 arithmetic resolves: decided as in 64 bits."""
    N = 48
    g = torch.Generator().manual_seed(7)
    x = 0.5 + 1e-6 * torch.randn((N, E), generator=g)
    x[: N // 2] += torch.randint(0, 3, (N // 2, E), generator=g)
    for bias in (None, 1e-7 * torch.randn(E, generator=g), 1.0 + 1e-7 * torch.randn(E, generator=g)):
        kw = dict(score=score, groups=groups, groups_kept=kept, group_top=2)
        check(x, call(x, k, bias=bias, **kw), k, bias=None if bias is None else bias.expand(N, -1), **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("E,k,groups,with_bias", [(64, 8, 1, False), (64, 8, 4, True), (256, 8, 8, False), (256, 8, 8, True), (100, 12, 1, True)])
def test_route_closed_experts(dtype, score, renormalise, E, k, groups, with_bias):
    """Masked logits (minus infinity, the type's lowest value, NaN), rows with fewer than k open experts or none, infinite ones."""
    N = 24
    x = make(N, E, dtype, seed=E)
    low = torch.finfo(dtype).min
    x[0] = -INF
    x[1] = low
    x[2] = NAN
    x[3, 3:] = -INF                                # three open ones
    x[4, ::2] = low
    x[5, 1::2] = NAN
    x[6, : E - 1] = -INF                           # the last alone
    x[7, 5] = INF
    x[8, 5] = x[8, 9] = INF
    x[9, 5] = torch.finfo(dtype).max
    x[10] = INF
    x[11, 7] = -INF
    x[12, : E // groups] = -INF                    # a whole group
    x[13, : E - 2] = low
    x[14] = low / 2                                # far down, but open
    x[15, 1:] = low / 2
    bias = None
    if with_bias:
        bias = 0.1 * torch.randn(E, generator=torch.Generator().manual_seed(1))
        bias[4], bias[20], bias[33] = INF, -INF, NAN
        bias[10] = -50.0                           # never chosen while others are open
        bias[11] = 3.0
    kw = dict(score=score, renormalise=renormalise, groups=groups, groups_kept=max(1, groups // 2), group_top=2)
    check(x, call(x, k, bias=bias, **kw), k, bias=None if bias is None else bias.expand(N, -1), **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_far_logits(dtype, score, renormalise):
    """Scores that saturate or vanish in fp32 keep their order, and renormalised weights stay what they are."""
    N, E, k = 40, 64, 6
    g = torch.Generator().manual_seed(3)
    x = torch.randn((N, E), generator=g) * torch.logspace(-3, 3, N)[:, None]
    x[10:20] += 200.0
    x[20:30] -= 200.0
    x[30] -= 1e4
    x = x.to(dtype)
    kw = dict(score=score, renormalise=renormalise)
    check(x, call(x, k, **kw), k, **kw)
    bias = torch.linspace(-1, 1, E)
    check(x, call(x, k, bias=bias, **kw), k, bias=bias.expand(N, -1), **kw)
    bias = torch.linspace(-1e30, 1e30, E)
    check(x, call(x, k, bias=bias, **kw), k, bias=bias.expand(N, -1), **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [-1e5, 1e5, -1e30, 1e38])
def test_route_biases_beyond_the_logits_type(dtype, shift):
    """Biases are fp32 whatever the logits' type: keys far outside it are keys like others."""
    x = make(20, 64, dtype, seed=2)
    bias = shift * (1 + torch.linspace(0, 1, 64))
    check(x, call(x, 6, bias=bias, score="sigmoid"), 6, bias=bias.expand(20, -1), score="sigmoid")


@pytest.mark.parametrize("E,k,groups", [(64, 6, 1), (256, 8, 8)])
def test_route_layers_masks_and_strides(E, k, groups):
    import paper_2608_03676_b200 as P
    L, T = 3, 29
    x = make(L * T, E + 24, torch.float32, seed=8).view(L, T, E + 24).cuda()
    g = torch.Generator().manual_seed(2)
    bias = 0.2 * torch.randn((L, E), generator=g)
    mask = torch.rand((L, T), generator=g) < 0.7
    kw = dict(score="sigmoid", groups=groups, groups_kept=max(1, groups // 2), group_top=1)
    for start in (0, 1, 8):
        part = x[:, :, start:start + E]
        flat = part.cpu().contiguous().view(L * T, E)
        got = P.route(part, k, bias=bias.cuda(), mask=mask.cuda(), **kw)
        check(flat, (got["topk"].cpu().numpy(), got["weights"].cpu().numpy()), k, bias=bias.repeat_interleave(T, 0), mask=mask.view(-1), **kw)
    one = P.route(part, k, bias=bias[0].cuda(), **kw)
    check(flat, (one["topk"].cpu().numpy(), one["weights"].cpu().numpy()), k, bias=bias[0].expand(L * T, -1), **kw)
    only = P.route(part, k, bias=bias[0].cuda(), want_weights=False, **kw)
    assert set(only) == {"topk"} and torch.equal(only["topk"], one["topk"])
    again = P.route(part, k, bias=bias[0].cuda(), out=one, **kw)
    assert again["topk"].data_ptr() == one["topk"].data_ptr() and torch.equal(only["topk"], again["topk"])
    none = P.route(part[:, :0], k, **kw)
    assert none["topk"].shape == (L, 0, k) and none["weights"].shape == (L, 0, k)


def special_rows(E, dtype, seed):
    """Rows of every kind that the tests above have: spread, far apart, coarse, next to each other, masked, empty, infinite."""
    g = torch.Generator().manual_seed(seed)
    x = 1.5 * torch.randn((60, E), generator=g)
    x[8:16] = torch.randint(-4, 4, (8, E), generator=g) / 4
    x[16:24] = 0.5 + 1e-6 * torch.randn((8, E), generator=g) + torch.randint(0, 3, (8, E), generator=g)
    x[24] = 0.25
    x[25, ::2] = -0.0
    x[26:30] *= 40
    x[30] -= 200
    x = x.to(dtype)
    low = torch.finfo(dtype).min
    x[31] = -INF
    x[32] = low
    x[33] = NAN
    x[34, 3:] = -INF
    x[35, ::2] = low
    x[36, 1::2] = NAN
    x[37, : E - 1] = -INF
    x[38, 5] = INF
    x[39, 5] = x[39, 7] = INF
    x[40, 5] = torch.finfo(dtype).max
    x[41, 5] = torch.finfo(dtype).max
    x[41, 7] = INF
    x[42] = INF
    x[43] = low / 2
    x[44, 1:] = low / 2
    x[45, : E - 2] = low
    x[46] = x[46].abs()
    x[47] = -x[47].abs()
    return x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,k", [(8, 1), (16, 8), (32, 2), (64, 8), (72, 6), (104, 7), (128, 8), (128, 4), (256, 8), (512, 8), (1024, 8), (40, 3), (256, 12)])
@pytest.mark.parametrize("score,renormalise", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_route_many_rows(dtype, E, k, score, renormalise):
    """The same rows again and again, in other lanes each time: every copy gets what the definition gives the row."""
    x = special_rows(E, dtype, seed=E + k)
    N, times = x.shape[0], 1101
    kw = dict(score=score, renormalise=renormalise, scale=1.5)
    topk, w = call(x.repeat(times, 1), k, **kw)
    check(x, (topk[:N], w[:N]), k, **kw)
    topk, w = topk.reshape(times, N, k), w.reshape(times, N, k)
    assert (topk == topk[:1]).all() and (w == w[:1]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,k", [(64, 8), (256, 8), (128, 6)])
@pytest.mark.parametrize("score,groups,with_bias", [("sigmoid", 8, True), ("softmax", 4, False), ("sigmoid", 1, True), ("softmax", 2, True)])
def test_route_many_rows_with_bias_and_groups(dtype, E, k, score, groups, with_bias):
    x = special_rows(E, dtype, seed=E + groups)
    N, times = x.shape[0], 601
    bias = 0.1 * torch.randn(E, generator=torch.Generator().manual_seed(E)) if with_bias else None
    kw = dict(score=score, groups=groups, groups_kept=(groups + 1) // 2, group_top=2, scale=2.5)
    topk, w = call(x.repeat(times, 1), k, bias=bias, **kw)
    check(x, (topk[:N], w[:N]), k, bias=None if bias is None else bias.expand(N, -1), **kw)
    topk, w = topk.reshape(times, N, k), w.reshape(times, N, k)
    assert (topk == topk[:1]).all() and (w == w[:1]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_route_many_rows_strided_masked_in_layers(dtype):
    import paper_2608_03676_b200 as P
    L, T, E, k = 3, 20000, 96, 5
    x = special_rows(E + 32, dtype, seed=4).repeat(L * T // 60, 1).view(L, T, E + 32).cuda()
    mask = torch.rand((L, T), generator=torch.Generator().manual_seed(1)) < 0.8
    for start in (0, 1, 16):
        part = x[:, :, start:start + E]
        got = P.route(part, k, mask=mask.cuda())
        want = P.route(part[0, :60].contiguous(), k)               # (few rows: another kernel)
        for name, none in (("topk", -1), ("weights", 0)):
            all_rows = want[name].repeat(L * T // 60, 1).view(L, T, k)
            all_rows = torch.where(mask.cuda()[..., None], all_rows, torch.full_like(all_rows, none))
            if name == "topk":
                assert torch.equal(got[name], all_rows)
            else:
                assert torch.allclose(got[name], all_rows, rtol=400 * F32, atol=1e-37)


def grad(logits, topk, dw, **kw):
    import paper_2608_03676_b200 as P
    return P.route_backward(logits.cuda(), topk.cuda(), dw.cuda(), **kw).double().cpu().numpy()


def check_grad(logits, topk, dw, score, renormalise, scale):
    got = grad(logits, topk, dw, score=score, renormalise=renormalise, scale=scale)
    want, size = plain.route_backward(logits, topk.numpy(), dw.numpy(), score, renormalise, scale)
    far = np.maximum(spread(logits, np.clip(topk.numpy(), -1, logits.shape[1] - 1)).max(1, keepdims=True), 0)
    if score == "softmax" and not renormalise:     # every open expert's own distance counts
        x = plain.open_logits(logits)
        d = x.max(1, keepdims=True) - x
        far = np.where(np.isfinite(d), d, 0.0) + far
    bound = plain.half_step(logits.dtype) * (1 + 2 ** -8) * np.abs(want) + (4 * far + 128) * F32 * size + \
        torch.finfo(logits.dtype).tiny * torch.finfo(logits.dtype).eps
    assert np.isfinite(got).all() and (np.abs(got - want) <= bound).all(), float((np.abs(got - want) - bound).max())
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,E,k", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_backward(dtype, N, E, k, score, renormalise):
    x = make(N, E, dtype, seed=E * 2 + k)
    topk = torch.topk(x.float(), k, dim=1).indices.int()
    topk[0, k // 2] = -1                           # a place that nothing filled
    if N > 2:
        topk[2] = -1                               # padding
    dw = torch.randn((N, k), generator=torch.Generator().manual_seed(N))
    check_grad(x, topk, dw, score, renormalise, 1.5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("E,k", [(16, 4), (128, 8), (200, 40)])
def test_route_backward_odd_tables(dtype, score, renormalise, E, k):
    """The same expert twice, entries outside the experts, closed experts in the table, rows without open experts, far logits."""
    N = 16
    x = make(N, E, dtype, seed=5)
    g = torch.Generator().manual_seed(6)
    topk = torch.randint(0, E, (N, k), generator=g).int()
    topk[0] = 3
    topk[1, :2] = 7
    topk[2, 0], topk[2, 1], topk[2, 2] = E, -5, 2 ** 31 - 1
    x[3] = -INF
    x[4, topk[4, 0].long()] = NAN
    x[5, topk[5, 1].long()] = torch.finfo(dtype).min
    x[6, topk[6, 1].long()] = INF
    x[7] = -300.0
    x[8] = 300.0
    x[9] *= 50
    dw = torch.randn((N, k), generator=g)
    got = check_grad(x, topk, dw, score, renormalise, 0.5)
    assert (got[3] == 0).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_backward_against_differences(score, renormalise):
    N, E, k = 5, 12, 4
    x = make(N, E, torch.float32, seed=9)
    topk = torch.topk(x, k, dim=1).indices.int()
    dw = torch.randn((N, k), generator=torch.Generator().manual_seed(4))
    got = grad(x, topk, dw, score=score, renormalise=renormalise, scale=2.0)
    step = 1e-5
    for e in range(E):
        up, down = x.double().clone(), x.double().clone()
        up[:, e] += step
        down[:, e] -= step
        slope = sum(s * (plain.weights_of_table(t, topk.numpy(), score, renormalise, 2.0) * dw.double().numpy()).sum(1)
                    for s, t in ((1, up), (-1, down))) / (2 * step)
        # differences: step^2 / 6 times a third derivative below 100; the kernel: some tens of fp32 roundings of terms below 10
        assert (np.abs(got[:, e] - slope) < 1e-6 + 300 * F32).all()


def test_route_backward_strides_and_layers():
    import paper_2608_03676_b200 as P
    L, T, E, k = 2, 33, 72, 6
    wide = make(L * T, E + 9, torch.bfloat16, seed=1).view(L, T, E + 9).cuda()
    for start in (0, 1, 8):
        x = wide[:, :, start:start + E]
        topk = P.route(x, k)["topk"]
        dw = torch.randn((L, T, k), generator=torch.Generator().manual_seed(2))
        room = torch.full((L, T, E + 9), 7.0, dtype=torch.bfloat16, device="cuda")
        got = P.route_backward(x, topk, dw.cuda(), out=room[:, :, start:start + E])
        want, size = plain.route_backward(x.cpu().reshape(L * T, E), topk.cpu().numpy().reshape(L * T, k), dw.numpy().reshape(L * T, k), "softmax", True, 1.0)
        off = np.abs(got.double().cpu().numpy().reshape(L * T, E) - want)
        assert (off <= 2 ** -8 * 1.01 * np.abs(want) + 300 * F32 * size).all()
        assert (room[:, :, :start] == 7).all() and (room[:, :, start + E:] == 7).all()
    none = P.route_backward(x[:, :0], topk[:, :0].contiguous(), dw[:, :0].contiguous().cuda())
    assert none.shape == (L, 0, E)


def test_route_refuses():
    import paper_2608_03676_b200 as P
    x = make(8, 64, torch.float32).cuda()
    topk, dw = torch.zeros((8, 4), dtype=torch.int32, device="cuda"), torch.zeros((8, 4), device="cuda")
    bad = [lambda: P.route(x.cpu(), 4), lambda: P.route(x.double(), 4), lambda: P.route(x, 0), lambda: P.route(x, 65), lambda: P.route(x[0], 4),
           lambda: P.route(x, 4, score="relu"), lambda: P.route(x, 4, groups=7), lambda: P.route(x, 4, groups=0), lambda: P.route(x, 4, groups=8, groups_kept=9),
           lambda: P.route(x, 9, groups=8, groups_kept=1), lambda: P.route(x, 4, groups=8, groups_kept=4, group_top=3),
           lambda: P.route(x, 4, scale=float("inf")), lambda: P.route(x, 4, bias=torch.zeros(63, device="cuda")),
           lambda: P.route(x, 4, bias=torch.zeros(64, dtype=torch.bfloat16, device="cuda")), lambda: P.route(x, 4, bias=torch.zeros(64)),
           lambda: P.route(x, 4, mask=torch.ones(8, device="cuda")), lambda: P.route(x, 4, mask=torch.ones(7, dtype=torch.bool, device="cuda")),
           lambda: P.route(x, 4, out=dict(topk=topk.long())), lambda: P.route(x, 4, out=dict(topk=topk[:, :3])),
           lambda: P.route(x.t(), 4), lambda: P.route(make(2, 1025, torch.float32).cuda(), 4),
           lambda: P.route(make(2, 1024, torch.float32).cuda(), 4, groups=128, groups_kept=4),
           lambda: P.route(x, 4, out=dict(topk=x.view(torch.int32).view(-1)[:32].view(8, 4))),
           lambda: P.route_backward(x, topk.long(), dw), lambda: P.route_backward(x, topk, dw[:7]), lambda: P.route_backward(x, topk, dw, out=x),
           lambda: P.route_backward(x, topk, dw, score="x"), lambda: P.route_backward(x, topk, dw, out=x[:, :32])]
    before = x.clone()
    for i, f in enumerate(bad):
        with pytest.raises(P.TaotError):
            f()
            print("not refused:", i)
    assert torch.equal(before, x)
