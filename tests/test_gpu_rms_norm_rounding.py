"""The 8-bit rows of the norm to the bit: scales as the products and values as the quotients of the 32-bit y that they are defined by."""
import pytest
import torch

import layer_plain as plain

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def quotients(y, group):
    """Scales and 8-bit values of the fp32 rows y on the CPU: a product with the fp32 reciprocal, fp32 divisions (all rounded to nearest),
    then e4m3 (to nearest, ties to even)."""
    inverse = torch.tensor(1.0) / plain.E4M3_MAX
    scales, values = [], []
    for p in torch.split(y, group, dim=-1):
        s = (p.abs().amax(-1) * inverse).clamp(min=plain.LEAST_SCALE)
        scales.append(s)
        values.append((p / s[:, None]).clamp(-plain.E4M3_MAX, plain.E4M3_MAX).to(torch.float8_e4m3fn))
    return torch.stack(scales, -1), torch.cat([v.view(torch.uint8) for v in values], -1)


def check(x, w, group):
    """The 32-bit y is h * rstd * weight, two fp32 products (in fp32 rows it is also what is returned)."""
    import paper_2608_03676_b200 as P
    out = {name: t.cpu() for name, t in P.rms_norm(x.cuda(), w.cuda(), group=group).items()}
    y = x.float() * out["rstd"][:, None] * w.float()
    if x.dtype == torch.float32:
        assert torch.equal(out["y"], y)
    scales, q = quotients(y, group)
    assert torch.equal(out["scales"], scales), float(((out["scales"] - scales).abs() / scales).max())
    got = out["q"].view(torch.uint8)
    assert torch.equal(got, q), "%d of %d" % (int((got != q).sum()), q.numel())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,D,group", [(3000, 256, 64), (700, 1024, 128), (500, 1111, 32), (300, 4096, 128), (90, 8192, 256), (200, 5000, 64),
                                       (100, 4733, 256), (60, 12288, 128), (60, 12289, 32), (2000, 33, 32)])
def test_eight_bit_rows_are_the_quotients_rounded_once(dtype, N, D, group):
    g = torch.Generator().manual_seed(N + D)
    rand = lambda *s: torch.randn(s, generator=g)
    check(rand(N, D).to(dtype), (1 + 0.2 * rand(D)).to(dtype), group)
    # few different values: many quotients in the middle of two 8-bit values
    coarse = torch.randint(-32, 33, (N, D), generator=g).to(dtype)
    check(coarse, torch.ones(D, dtype=dtype), group)


@pytest.mark.parametrize("N,D,group", [(500, 1024, 128), (300, 1111, 32), (30, 12288, 128)])
@pytest.mark.parametrize("size", [1e-44, 1e-40, 3e-38, 1e-36, 1e-33, 1e-28, 1e-27, 1e-20, 1e20, 1e35])
def test_eight_bit_rows_of_tiny_and_huge_values(N, D, group, size):
    """From scales at their least value, with y below the smallest normal number, to scales near the largest."""
    g = torch.Generator().manual_seed(D)
    rand = lambda *s: torch.randn(s, generator=g)
    check(rand(N, D), size * (1 + 0.2 * rand(D)), group)


def test_eight_bit_rows_of_infinite_scales():
    """An infinite y: its group's scale is infinite, the quotients of the finite values are 0 and its own is not a number."""
    import paper_2608_03676_b200 as P
    for dtype, D in ((torch.float32, 512), (torch.float32, 511), (torch.bfloat16, 512), (torch.float32, 12288)):
        x, w = torch.ones((4, D), dtype=dtype), torch.ones(D, dtype=dtype)
        w[130] = float("inf")
        out = P.rms_norm(x.cuda(), w.cuda(), group=128)
        q, s = out["q"].float().cpu(), out["scales"].cpu()
        assert torch.isinf(s[:, 1]).all() and q[:, 130].isnan().all()
        assert (q[:, 128:130] == 0).all() and (q[:, 131:256] == 0).all()
        assert torch.isfinite(s[:, 0]).all() and (q[:, :128] == 448).all() and (q[:, 256:] == 448).all()
