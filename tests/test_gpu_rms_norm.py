"""RMS norm with the residual's addition and 8-bit rows, and its gradients, against the definition in 64 bits."""
import pytest
import torch

import layer_plain as plain

pytestmark = pytest.mark.gpu

F32 = plain.F32
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def sum_steps(D):
    """Roundings on the way of one term of a sum over D columns: a thread's own terms, then the tree over threads."""
    return D / 256 + 16


def make(N, D, dtype, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g)
    x, r, w = (scale * rand(N, D)).to(dtype), (scale * rand(N, D)).to(dtype), (1 + 0.2 * rand(D)).to(dtype)
    return x, r, w


def close(got, want, rel, absolute=0.0):
    got = got.double().cpu()
    bound = rel * want.abs() + absolute
    off = (got - want).abs()
    assert torch.isfinite(got).all()
    assert (off <= bound).all(), float((off - bound).max())


def check_norm(out, x, w, eps, residual, group):
    """Against the definition: h to the bit, y and scales by the roundings on their way, q by half a step of e4m3."""
    D = x.shape[-1]
    want = plain.rms_norm(x, w, eps, residual, group)
    if residual is not None:
        assert torch.equal(out["h"].cpu(), want["h"])
    # the sum of squares: its roundings, halved by the square root; then division, root, reciprocal; two products
    rel = (sum_steps(D) / 2 + 8) * F32
    close(out["rstd"], want["rstd"], rel)
    least = torch.finfo(x.dtype).tiny * torch.finfo(x.dtype).eps
    if "y" in out:
        close(out["y"], want["y"], plain.half_step(x.dtype) * (1 + 2 ** -8) + rel, least)
    if group:
        close(out["scales"], want["scales"], rel + 4 * F32)
        s = out["scales"].double().cpu()
        per = torch.repeat_interleave(s, group, dim=-1)[..., :D]
        # half a step: 2^-4 of the value, or half the smallest step 2^-9 near zero; and the fp32 value that is rounded
        close(out["q"].float().double().cpu() * per, want["y"], 2.0 ** -4 + rel + 8 * F32, 2.0 ** -10 * per * (1 + 1e-6))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,D,group", [(1, 1, 32), (1, 7, 0), (3, 8, 32), (5, 33, 32), (2, 256, 64), (4, 264, 128), (1, 1000, 256),
                                       (130, 1111, 128), (9, 2048, 128), (300, 4096, 128), (3, 5000, 64), (2, 12288, 32),
                                       (2, 20000, 128), (1, 65536, 256)])
@pytest.mark.parametrize("with_residual", [False, True])
def test_norm(dtype, N, D, group, with_residual):
    import paper_2608_03676_b200 as P
    x, r, w = make(N, D, dtype, seed=N + D)
    res = r if with_residual else None
    out = P.rms_norm(x.cuda(), w.cuda(), eps=1e-5, residual=None if res is None else r.cuda(), group=group)
    assert set(out) == {"y", "rstd"} | ({"h"} if with_residual else set()) | ({"q", "scales"} if group else set())
    check_norm(out, x, w, 1e-5, res, group)
    if group:                                      # the 8-bit rows alone
        only = P.rms_norm(x.cuda(), w.cuda(), eps=1e-5, residual=None if res is None else r.cuda(), group=group, want_y=False)
        assert "y" not in only and torch.equal(only["q"].view(torch.uint8), out["q"].view(torch.uint8))
        assert torch.equal(only["scales"], out["scales"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("start,D,ld", [(0, 512, 520), (1, 511, 512), (3, 77, 131), (8, 1024, 1040), (4, 1020, 1030)])
def test_norm_strided_rows_and_odd_starts(dtype, start, D, ld):
    import paper_2608_03676_b200 as P
    N = 37
    big = [t.cuda() for t in make(N, ld, dtype, seed=D)[:2]]
    x, r = (t[:, start:start + D] for t in big)
    w = make(1, D, dtype, seed=3)[2]
    y = torch.full((N, ld), 7.0, dtype=dtype, device="cuda")
    h = torch.full((N, ld), 7.0, dtype=dtype, device="cuda")
    q = torch.full((N, ld), 7.0, device="cuda").to(torch.float8_e4m3fn)
    out = P.rms_norm(x, w.cuda(), residual=r, group=64,
                     out=dict(y=y[:, start:start + D], h=h[:, start:start + D], q=q[:, start:start + D]))
    check_norm(out, x.cpu(), w, 1e-6, r.cpu(), 64)
    for t in (y, h, q.float()):                    # what lies between the rows is as it was
        assert (t[:, :start] == 7).all() and (t[:, start + D:] == 7).all()


@pytest.mark.parametrize("N,D", [(64, 4096), (5, 77), (3, 20000)])
def test_norm_in_place(N, D):
    import paper_2608_03676_b200 as P
    x, r, w = make(N, D, torch.bfloat16, seed=1)
    want = P.rms_norm(x.cuda(), w.cuda(), residual=r.cuda(), group=128)
    for into in ("residual", "x"):
        xs, rs = x.cuda(), r.cuda()
        got = P.rms_norm(xs, w.cuda(), residual=rs, group=128, out=dict(h=rs if into == "residual" else xs))
        assert got["h"].data_ptr() == (rs if into == "residual" else xs).data_ptr()
        for name in want:
            assert torch.equal(got[name].view(torch.uint8), want[name].view(torch.uint8)), name
    xs = x.cuda()
    assert torch.equal(P.rms_norm(xs, w.cuda(), out=dict(y=xs))["y"], P.rms_norm(x.cuda(), w.cuda())["y"])


def test_norm_rows_without_values():
    """Rows of zeros, of the smallest and of huge values, and rows that hold a NaN or an infinity, which stay by themselves."""
    import paper_2608_03676_b200 as P
    x, _, w = make(8, 640, torch.float32, seed=2)
    x[0] = 0.0
    x[1] = 1e-30
    x[2] = 1e18                                    # squares still add up in fp32
    x[3, 5] = float("nan")
    x[4, 600] = float("inf")
    x[5, :128] = 0.0                               # one group of columns without a value
    out = {name: t.cpu() for name, t in P.rms_norm(x.cuda(), w.cuda(), group=128).items()}
    fine = [0, 1, 2, 5, 6, 7]
    check_norm({name: t[fine] for name, t in out.items()}, x[fine], w, 1e-6, None, 128)
    assert (out["y"][0] == 0).all() and (out["q"][0].float() == 0).all() and (out["scales"][0] == 2.0 ** -126).all()
    assert (out["scales"][5][0] == 2.0 ** -126) and (out["q"][5][:128].float() == 0).all()
    assert out["y"][3].isnan().all() and out["scales"][3].isnan().all() and out["q"][3].float().isnan().all()
    assert out["y"][4][600].isnan() and (out["y"][4][:600] == 0).all() and (out["y"][4][601:] == 0).all()
    assert out["scales"][4][4].isnan() and (out["q"][4][:512].float() == 0).all()


def test_norm_eps_and_shapes():
    import paper_2608_03676_b200 as P
    x, r, w = make(24, 96, torch.float16, seed=4, scale=1e-3)
    for eps in (0.0, 1e-6, 1.0):
        out = P.rms_norm(x.view(2, 3, 4, 96).cuda(), w.cuda(), eps=eps, residual=r.view(2, 3, 4, 96).cuda(), group=32)
        assert out["y"].shape == (2, 3, 4, 96) and out["rstd"].shape == (2, 3, 4) and out["scales"].shape == (2, 3, 4, 3)
        check_norm({n: t.reshape((24,) + tuple(t.shape[3:])) for n, t in out.items()}, x, w, eps, r, 32)
    one = P.rms_norm(x[0].cuda(), w.cuda())
    assert one["y"].shape == (96,) and one["rstd"].shape == ()
    none = P.rms_norm(x[:0].cuda(), w.cuda(), residual=r[:0].cuda(), group=32)
    assert none["y"].shape == (0, 96) and none["scales"].shape == (0, 3)


def check_grad(got, dy, h, w, rstd, dh):
    N, D = h.shape
    dx, dw = plain.rms_norm_backward(dy, h, w, rstd, dh)
    g, xhat = (dy.double() * w.double()).abs(), (h.double() * rstd.double()[:, None]).abs()
    # the parts that dx is the sum of; the mean's own roundings, and six on the way of each part
    size = rstd.double()[:, None] * (g + xhat * (g * xhat).mean(1, keepdim=True) * (1 + sum_steps(D)))
    size = size if dh is None else size + dh.double().abs()
    close(got["dx"], dx, plain.half_step(h.dtype) * (1 + 2 ** -8), 6 * F32 * size + torch.finfo(h.dtype).tiny * torch.finfo(h.dtype).eps)
    if "dweight" in got:
        # N terms of three factors, added over rows of a span and over spans, at most N additions in a row
        close(got["dweight"], dw, 0.0, (min(N, N / 16 + 1024) + 4) * F32 * (dy.double().abs() * xhat).sum(0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,D", [(1, 1), (2, 7), (1, 4096), (3, 33), (130, 1111), (700, 256), (257, 2048), (300, 4096), (5, 12288),
                                 (3, 20000), (2000, 64)])
@pytest.mark.parametrize("with_dh", [False, True])
def test_norm_backward(dtype, N, D, with_dh):
    import paper_2608_03676_b200 as P
    dy, h, w = make(N, D, dtype, seed=N * 3 + D)
    dh = make(N, D, dtype, seed=9)[0] if with_dh else None
    rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
    args = (dy.cuda(), h.cuda(), w.cuda(), rstd.cuda())
    got = P.rms_norm_backward(*args, dh=None if dh is None else dh.cuda())
    check_grad(got, dy, h, w, rstd, dh)
    again = P.rms_norm_backward(*args, dh=None if dh is None else dh.cuda())
    assert torch.equal(again["dx"], got["dx"]) and torch.equal(again["dweight"], got["dweight"])      # the same bits
    only = P.rms_norm_backward(*args, dh=None if dh is None else dh.cuda(), want_dweight=False)
    assert set(only) == {"dx"} and torch.equal(only["dx"], got["dx"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("start,D,ld", [(0, 512, 520), (1, 511, 512), (3, 77, 131), (4, 1020, 1030)])
def test_norm_backward_strided_and_in_place(dtype, start, D, ld):
    import paper_2608_03676_b200 as P
    N = 41
    parts = [t.cuda() for t in make(N, ld, dtype, seed=D)[:2]] + [make(N, ld, dtype, seed=5)[0].cuda()]
    dy, h, dh = (t[:, start:start + D] for t in parts)
    w = make(1, D, dtype, seed=3)[2]
    rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
    before = [t.clone() for t in parts]
    got = P.rms_norm_backward(dy, h, w.cuda(), rstd, dh=dh)
    cpu = (before[0][:, start:start + D].cpu(), before[1][:, start:start + D].cpu(), w, rstd.cpu(), before[2][:, start:start + D].cpu())
    check_grad(got, *cpu)
    into = P.rms_norm_backward(dy, h, w.cuda(), rstd, dh=dh, out=dict(dx=dy))
    assert into["dx"].data_ptr() == dy.data_ptr() and torch.equal(dy, got["dx"]) and torch.equal(into["dweight"], got["dweight"])
    assert torch.equal(parts[0][:, :start], before[0][:, :start]) and torch.equal(parts[0][:, start + D:], before[0][:, start + D:])
    parts[0].copy_(before[0])
    P.rms_norm_backward(dy, h, w.cuda(), rstd, dh=dh, out=dict(dx=dh))
    assert torch.equal(dh, got["dx"]) and torch.equal(parts[1], before[1])


def test_norm_backward_without_rows_sets_the_weights_gradient_to_zero():
    import paper_2608_03676_b200 as P
    dy, h, w = make(4, 64, torch.bfloat16)
    got = P.rms_norm_backward(dy[:0].cuda(), h[:0].cuda(), w.cuda(), torch.empty(0, device="cuda"),
                              out=dict(dweight=torch.full((64,), 7.0, device="cuda")))
    assert got["dx"].shape == (0, 64) and (got["dweight"] == 0).all()


def test_norm_backward_against_differences():
    """dx and dweight along random directions against central differences of the definition in 64 bits."""
    import paper_2608_03676_b200 as P
    N, D = 6, 40
    x, r, w = (t.double() for t in make(N, D, torch.float32, seed=11))
    dy, dh, _ = make(N, D, torch.float32, seed=12)
    h = (x + r).float()
    rstd = (h.double().square().mean(1) + 1e-3).rsqrt().float()
    got = P.rms_norm_backward(dy.cuda(), h.cuda(), w.float().cuda(), rstd.cuda(), dh=dh.cuda())

    def value(hh, ww):                             # what the gradients are gradients of
        y = hh / torch.sqrt((hh * hh).mean(1, keepdim=True) + 1e-3) * ww
        return (y * dy.double()).sum() + (hh * dh.double()).sum()

    g = torch.Generator().manual_seed(13)
    for _ in range(8):
        a, b, step = torch.randn((N, D), generator=g).double(), torch.randn(D, generator=g).double(), 1e-5
        hd, wd = h.double(), w.float().double()
        along_h = (value(hd + step * a, wd) - value(hd - step * a, wd)) / (2 * step)
        along_w = (value(hd, wd + step * b) - value(hd, wd - step * b)) / (2 * step)
        # differences are off by step^2 times a third derivative of about a hundred terms; the kernel by fp32 roundings
        assert abs(float((got["dx"].double().cpu() * a).sum() - along_h)) < 1e-4
        assert abs(float((got["dweight"].double().cpu() * b).sum() - along_w)) < 1e-4


def test_norm_refuses():
    import paper_2608_03676_b200 as P
    x, r, w = (t.cuda() for t in make(8, 64, torch.bfloat16))
    bad = [lambda: P.rms_norm(x.cpu(), w), lambda: P.rms_norm(x, w.cpu()), lambda: P.rms_norm(x.double(), w.double()),
           lambda: P.rms_norm(x, w.float()), lambda: P.rms_norm(x, w[:63]), lambda: P.rms_norm(x, w, residual=r[:7]),
           lambda: P.rms_norm(x, w, residual=r.float()), lambda: P.rms_norm(x, w, group=48), lambda: P.rms_norm(x, w, group=-32),
           lambda: P.rms_norm(x, w, eps=-1.0), lambda: P.rms_norm(x, w, eps=float("nan")), lambda: P.rms_norm(x, w, want_y=False),
           lambda: P.rms_norm(x.t(), w[:8]), lambda: P.rms_norm(x, w, out=dict(y=x[:, :32])),
           lambda: P.rms_norm(x[:7], w, out=dict(y=x[1:])), lambda: P.rms_norm(x, w, residual=r, out=dict(y=r)),
           lambda: P.rms_norm(x, w, residual=r, out=dict(y=x, h=x)), lambda: P.rms_norm(x[0, 0], w),
           lambda: P.rms_norm_backward(x, r, w, torch.ones(7, device="cuda")),
           lambda: P.rms_norm_backward(x, r, w, torch.ones(8, device="cuda"), out=dict(dx=r)),
           lambda: P.rms_norm_backward(x, r, w, torch.ones(8, device="cuda"), dh=x[:7])]
    before = x.clone(), r.clone()
    for i, call in enumerate(bad):
        with pytest.raises(P.TaotError):
            call()
            print("not refused:", i)
    assert torch.equal(before[0], x) and torch.equal(before[1], r)
