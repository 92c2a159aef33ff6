"""Rows to the send buffer and back, and the gradients, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import layer_plain as plain

pytestmark = pytest.mark.gpu

F32 = plain.F32
TYPES = [torch.float32, torch.bfloat16, torch.float16]
#       B, n, k, D, ranks (0: no counts), share of padding
CASES = [(1, 1, 1, 1, 0, 0.0), (1, 1, 8, 4096, 8, 0.0), (2, 3, 2, 7, 1, 0.0), (1, 5, 6, 1111, 4, 0.3), (3, 37, 6, 130, 8, 0.2), (2, 64, 8, 264, 64, 0.0),
         (1, 300, 4, 1000, 0, 0.0), (4, 9, 1, 2048, 3, 0.5), (1, 130, 8, 4096, 16, 0.1), (2, 4, 64, 96, 5, 0.0), (1, 7, 3, 20000, 2, 0.0), (1, 6, 8, 512, 9, 1.0)]


def positions(B, n, k, ranks, padded, seed=0):
    """Positions and counts as a dispatcher makes them: entries by destination, undeliverable ones last."""
    g = torch.Generator().manual_seed(seed)
    R = max(ranks, 1)
    to = torch.randint(0, R, (B, n, k), generator=g)
    to[torch.rand((B, n), generator=g) < padded] = R
    to = to.view(B, n * k)
    order = torch.argsort(to, dim=1, stable=True)
    perm = torch.empty_like(order).scatter_(1, order, torch.arange(n * k).expand(B, -1).contiguous())
    counts = torch.zeros((B, R + 1), dtype=torch.int64).scatter_add_(1, to, torch.ones_like(to))[:, :R]
    return perm.view(B, n, k).int(), counts.int().contiguous() if ranks else None


def cuda(t):
    return None if t is None else t.cuda()


def array(t):
    return None if t is None else t.double().numpy()


def rand(*shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", TYPES + [torch.float8_e4m3fn, torch.uint8, torch.int32])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("cols", [0, 1, 9, 32])
def test_send(dtype, case, cols):
    import paper_2608_03676_b200 as P
    B, n, k, D, ranks, padded = case
    perm, counts = positions(B, n, k, ranks, padded, seed=n + D)
    raw = torch.randint(0, 256, (B, n, D * torch.empty((), dtype=dtype).element_size()), generator=torch.Generator().manual_seed(1), dtype=torch.uint8)
    x = raw.view(dtype)                            # any bits at all
    scales = rand(B, n, cols, dtype=torch.float32, seed=2) if cols else None
    rows = torch.full((B, n * k, raw.shape[-1]), 77, dtype=torch.uint8, device="cuda").view(dtype)
    given = dict(rows=rows)
    if cols:
        given["scales"] = torch.full((B, n * k, cols), 5.0, device="cuda")
    out = P.send(x.cuda(), perm.cuda(), counts=cuda(counts), scales=cuda(scales), out=given)
    want = plain.send(raw.numpy(), perm.numpy(), array(counts), np.full((B, n * k, raw.shape[-1]), 77, dtype=np.uint8))
    assert out["rows"].data_ptr() == rows.data_ptr() and (rows.view(torch.uint8).cpu().numpy() == want).all()
    if cols:
        want = plain.send(scales.numpy(), perm.numpy(), array(counts), np.full((B, n * k, cols), 5.0, dtype=np.float32))
        assert (out["scales"].cpu().numpy() == want).all()
    else:
        assert "scales" not in out
    assert out["info"].tolist() == [0] * B


def check_combine(got, y, perm, weights, counts, residual):
    k = perm.shape[-1]
    want, size = plain.combine(array(y), perm.numpy(), array(weights), array(counts), array(residual))
    off = np.abs(got.double().cpu().numpy() - want)
    tiny = torch.finfo(y.dtype).tiny * torch.finfo(y.dtype).eps
    bound = plain.half_step(y.dtype) * (1 + 2 ** -8) * np.abs(want) + (k + 1) * F32 * size + tiny     # k additions and products
    assert (off <= bound).all(), float((off - bound).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("weighted,with_residual", [(True, True), (False, False), (True, False), (False, True)])
def test_combine(dtype, case, weighted, with_residual):
    import paper_2608_03676_b200 as P
    B, n, k, D, ranks, padded = case
    perm, counts = positions(B, n, k, ranks, padded, seed=n + D + 1)
    y = rand(B, n * k, D, dtype=dtype, seed=3)
    if counts is not None:                         # rows that are not in use hold anything
        for b in range(B):
            y[b, int(counts[b].sum()):] = float("nan")
    w = rand(B, n, k, dtype=torch.float32, seed=4) if weighted else None
    r = rand(B, n, D, dtype=dtype, seed=5) if with_residual else None
    out = P.combine(y.cuda(), perm.cuda(), weights=cuda(w), counts=cuda(counts), residual=cuda(r))
    check_combine(out["out"], y, perm, w, counts, r)
    assert out["info"].tolist() == [0] * B
    if with_residual:                              # over the residual
        rs = r.cuda()
        got = P.combine(y.cuda(), perm.cuda(), weights=cuda(w), counts=cuda(counts), residual=rs, out=dict(out=rs))
        assert got["out"].data_ptr() == rs.data_ptr() and torch.equal(rs, out["out"])


def check_backward(got, dout, y, perm, weights, counts, before):
    dtype, D = dout.dtype, dout.shape[-1]
    dy, dw, size = plain.combine_backward(array(dout), array(y), perm.numpy(), array(weights), array(counts), array(before))
    tiny = torch.finfo(dtype).tiny * torch.finfo(dtype).eps
    if "dy" in got:
        off = np.abs(got["dy"].double().cpu().numpy() - dy)
        fine = np.isfinite(dy)
        assert (np.isnan(got["dy"].double().cpu().numpy()) == ~fine).all()
        assert (off[fine] <= (plain.half_step(dtype) * (1 + 2 ** -8) + F32) * np.abs(dy)[fine] + tiny).all()
    if "dweights" in got:
        off = np.abs(got["dweights"].double().cpu().numpy() - dw)
        assert (off <= (D / 256 + 24) * F32 * size).all(), float(off.max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("weighted", [True, False])
def test_combine_backward(dtype, case, weighted):
    import paper_2608_03676_b200 as P
    B, n, k, D, ranks, padded = case
    perm, counts = positions(B, n, k, ranks, padded, seed=n + D + 2)
    y = rand(B, n * k, D, dtype=dtype, seed=6)
    if counts is not None:
        for b in range(B):
            y[b, int(counts[b].sum()):] = float("nan")
    dout = rand(B, n, D, dtype=dtype, seed=7)
    w = rand(B, n, k, dtype=torch.float32, seed=8) if weighted else None
    before = torch.full((B, n * k, D), 3.0, dtype=dtype)
    args = dict(weights=cuda(w), counts=cuda(counts))
    got = P.combine_backward(dout.cuda(), perm.cuda(), y=y.cuda(), out=dict(dy=before.cuda()), **args)
    check_backward(got, dout, y, perm, w, counts, before)
    rows = P.combine_backward(dout.cuda(), perm.cuda(), out=dict(dy=before.cuda()), **args)
    assert set(rows) == {"dy", "info"} and torch.equal(rows["dy"], got["dy"])
    dw = P.combine_backward(dout.cuda(), perm.cuda(), y=y.cuda(), want_dy=False, **args)
    assert set(dw) == {"dweights", "info"} and torch.equal(dw["dweights"], got["dweights"])
    ys = y.cuda()                                  # over the rows themselves
    into = P.combine_backward(dout.cuda(), perm.cuda(), y=ys, out=dict(dy=ys), **args)
    check_backward(into, dout, y, perm, w, counts, y)
    assert torch.equal(into["dweights"], got["dweights"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("start,D,ld", [(0, 512, 520), (1, 511, 512), (3, 77, 131), (4, 1020, 1030)])
def test_strided_rows_and_odd_starts(dtype, start, D, ld):
    import paper_2608_03676_b200 as P
    B, n, k = 2, 21, 3
    perm, counts = positions(B, n, k, 4, 0.2, seed=D)
    w = rand(B, n, k, dtype=torch.float32, seed=1)
    wide = lambda rows, seed: rand(B, rows, ld, dtype=dtype, seed=seed).cuda()
    cut = lambda t: t[:, :, start:start + D]
    x, y, r, dout = wide(n, 2), wide(n * k, 3), wide(n, 4), wide(n, 5)
    seven = lambda rows: torch.full((B, rows, ld), 7.0, dtype=dtype, device="cuda")
    into = seven(n * k)
    P.send(cut(x), perm.cuda(), counts=counts.cuda(), out=dict(rows=cut(into)))
    want = plain.send(cut(x).cpu().double().numpy(), perm.numpy(), counts.numpy(), np.full((B, n * k, D), 7.0))
    assert (cut(into).cpu().double().numpy() == want).all()
    out = seven(n)
    P.combine(cut(y), perm.cuda(), weights=w.cuda(), counts=counts.cuda(), residual=cut(r), out=dict(out=cut(out)))
    check_combine(cut(out).cpu(), cut(y).cpu(), perm, w, counts, cut(r).cpu())
    dy = seven(n * k)
    got = P.combine_backward(cut(dout), perm.cuda(), y=cut(y), weights=w.cuda(), counts=counts.cuda(), out=dict(dy=cut(dy)))
    check_backward(got, cut(dout).cpu(), cut(y).cpu(), perm, w, counts, torch.full((B, n * k, D), 7.0, dtype=dtype))
    for t in (into, out, dy):
        assert (t[:, :, :start] == 7).all() and (t[:, :, start + D:] == 7).all()


def test_bad_positions_are_left_out_and_reported():
    """A position outside the buffer is caught on the device: flag of its buffer, no access, the other entries as ever."""
    import paper_2608_03676_b200 as P
    B, n, k, D = 3, 10, 4, 72
    perm, _ = positions(B, n, k, 0, 0.0)
    for v, (t, j) in zip((-1, n * k, 2 ** 31 - 1, -2 ** 31), ((0, 0), (3, 1), (5, 3), (9, 2))):
        perm[1, t, j] = v
    x, y, dout = (rand(B, m, D, dtype=torch.float32, seed=m) for m in (n, n * k, n))
    w = rand(B, n, k, dtype=torch.float32, seed=3)
    calls = [P.send(x.cuda(), perm.cuda(), out=dict(rows=torch.zeros((B, n * k, D), device="cuda"))),
             P.combine(y.cuda(), perm.cuda(), weights=w.cuda()),
             P.combine_backward(dout.cuda(), perm.cuda(), y=y.cuda(), weights=w.cuda(), out=dict(dy=torch.zeros((B, n * k, D), device="cuda")))]
    for got in calls:
        assert got["info"].tolist() == [0, P.INFO_BAD_INDEX, 0]
    assert (calls[0]["rows"].cpu().numpy() == plain.send(x.numpy(), perm.numpy(), None, np.zeros((B, n * k, D)))).all()
    check_combine(calls[1]["out"], y, perm, w, None, None)
    check_backward(calls[2], dout, y, perm, w, None, torch.zeros((B, n * k, D)))
    kept = torch.full((B,), 8, dtype=torch.int32, device="cuda")                 # status words are OR-ed into
    P.combine(y.cuda(), perm.cuda(), weights=w.cuda(), out=dict(info=kept))
    assert kept.tolist() == [8, 8 | P.INFO_BAD_INDEX, 8]


def test_counts_of_any_sum():
    """Counts that sum to more than the buffer, to nothing or to less than nothing."""
    import paper_2608_03676_b200 as P
    B, n, k, D = 4, 5, 2, 40
    perm, _ = positions(B, n, k, 0, 0.0)
    counts = torch.tensor([[100, 100], [0, 0], [-7, 3], [2 ** 31 - 1, 2 ** 31 - 1]], dtype=torch.int32)
    y = rand(B, n * k, D, dtype=torch.float32, seed=2)
    out = P.combine(y.cuda(), perm.cuda(), counts=counts.cuda())["out"]
    check_combine(out, y, perm, None, counts.long(), None)
    assert (out[1] == 0).all() and (out[2] == 0).all()


def test_no_entries():
    import paper_2608_03676_b200 as P
    y, r = torch.zeros((2, 0, 16), device="cuda"), torch.ones((2, 3, 16), device="cuda")
    perm = torch.zeros((2, 3, 0), dtype=torch.int32, device="cuda")
    assert torch.equal(P.combine(y, perm, residual=r)["out"], r) and (P.combine(y, perm)["out"] == 0).all()
    assert P.send(r, perm)["rows"].shape == (2, 0, 16)
    assert P.combine(y, perm, residual=r)["info"].tolist() == [0, 0]             # no entry, so no bad one
    none = torch.zeros((0, 3, 2), dtype=torch.int32, device="cuda")
    assert P.combine(torch.zeros((0, 6, 16), device="cuda"), none)["out"].shape == (0, 3, 16)
    got = P.combine_backward(torch.zeros((2, 0, 16), device="cuda"), torch.zeros((2, 0, 4), dtype=torch.int32, device="cuda"), y=y)
    assert got["dy"].shape == (2, 0, 16) and got["dweights"].shape == (2, 0, 4)


def test_the_gradient_of_send_is_combine_without_weights():
    """<send(x), d> = <x, combine(d)> in whole numbers, which both sums hold exactly."""
    import paper_2608_03676_b200 as P
    B, n, k, D = 2, 50, 6, 200
    perm, counts = positions(B, n, k, 8, 0.2, seed=1)
    g = torch.Generator().manual_seed(2)
    x, d = (torch.randint(-8, 9, (B, m, D), generator=g).float().cuda() for m in (n, n * k))
    rows = P.send(x, perm.cuda(), counts=counts.cuda(), out=dict(rows=torch.zeros((B, n * k, D), device="cuda")))["rows"]
    dx = P.combine(d, perm.cuda(), counts=counts.cuda())["out"]
    assert float((rows.double() * d.double()).sum()) == float((x.double() * dx.double()).sum())


def test_combine_backward_against_differences():
    import paper_2608_03676_b200 as P
    B, n, k, D = 1, 6, 3, 20
    perm, counts = positions(B, n, k, 4, 0.0, seed=3)
    y, dout = rand(B, n * k, D, dtype=torch.float32, seed=1), rand(B, n, D, dtype=torch.float32, seed=2)
    w = rand(B, n, k, dtype=torch.float32, seed=3)
    got = P.combine_backward(dout.cuda(), perm.cuda(), y=y.cuda(), weights=w.cuda(), counts=counts.cuda())
    value = lambda yy, ww: (plain.combine(yy, perm.numpy(), ww, counts.numpy(), None)[0] * array(dout)).sum()
    rng = np.random.default_rng(4)
    for _ in range(6):
        a, b = rng.standard_normal(y.shape), rng.standard_normal(w.shape)
        along = (value(array(y) + 1e-3 * a, array(w)) - value(array(y) - 1e-3 * a, array(w))) / 2e-3       # linear: no error of its own
        assert abs((got["dy"].double().cpu().numpy() * a).sum() - along) < 1e-4
        along = (value(array(y), array(w) + 1e-3 * b) - value(array(y), array(w) - 1e-3 * b)) / 2e-3
        assert abs((got["dweights"].double().cpu().numpy() * b).sum() - along) < 1e-4


def test_rows_refuse():
    import paper_2608_03676_b200 as P
    B, n, k, D = 2, 4, 2, 16
    perm, counts = (t.cuda() for t in positions(B, n, k, 3, 0.0))
    x, y = torch.zeros((B, n, D), device="cuda"), torch.zeros((B, n * k, D), device="cuda")
    w = torch.ones((B, n, k), device="cuda")
    bad = [lambda: P.send(x, perm.long()), lambda: P.send(x, perm.cpu()), lambda: P.send(x[:, :3], perm), lambda: P.send(x.double(), perm),
           lambda: P.send(x.cpu(), perm), lambda: P.send(x, perm, counts=counts.long()), lambda: P.send(x, perm, counts=counts[:1]),
           lambda: P.send(x, perm, scales=w[:, :3].contiguous()), lambda: P.send(x, perm, out=dict(rows=y[:, :7])),
           lambda: P.send(y[:, :n], perm, out=dict(rows=y)), lambda: P.send(x, perm, out=dict(info=torch.zeros(3, dtype=torch.int32, device="cuda"))),
           lambda: P.combine(y, perm, weights=w.bfloat16()), lambda: P.combine(y, perm, weights=w[:1]), lambda: P.combine(y[:, :7], perm),
           lambda: P.combine(y.double(), perm), lambda: P.combine(y, perm, residual=x.half()), lambda: P.combine(y, perm, out=dict(out=y[:, :n])),
           lambda: P.combine(y, torch.zeros((1, 1, 65), dtype=torch.int32, device="cuda")), lambda: P.combine(y, perm, counts=counts[:, :0]),
           lambda: P.combine(y.int(), perm), lambda: P.combine(y, perm[0, 0]),
           lambda: P.combine(torch.zeros((1, 65, D), device="cuda"), torch.zeros((1, 1, 65), dtype=torch.int32, device="cuda")),
           lambda: P.combine_backward(x, perm, want_dy=False), lambda: P.combine_backward(x, perm, y=y.half()),
           lambda: P.combine_backward(x, perm, y=y, out=dict(dy=torch.zeros((B, n * k, 2 * D), device="cuda")[:, :, :D])),
           lambda: P.combine_backward(y[:, :n], perm, out=dict(dy=y)), lambda: P.combine_backward(x, perm, y=y, out=dict(dweights=w.half()))]
    for i, f in enumerate(bad):
        with pytest.raises(P.TaotError):
            f()
            print("not refused:", i)
    assert not x.any() and not y.any()
