"""rstd as the root and the division of its definition, each rounded to nearest, where the mean itself is exact."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [1, 2, 64, 256, 1024, 4096, 8192, 16384])
def test_the_root_and_the_division_are_rounded_to_nearest(D):
    """Rows of one value of at most 9 bits, D a power of two: squares (18 bits), sums of up to 64 of them in a
    thread, and by twos from there, and the mean are exact in fp32."""
    import paper_2608_03676_b200 as P
    g = torch.Generator().manual_seed(D)
    N = 200 if D > 2048 else 2000
    v = torch.randint(1, 512, (N,), generator=g).float() * 2.0 ** torch.randint(-30, 30, (N,), generator=g).float()
    x = v[:, None].expand(N, D).contiguous()
    out = P.rms_norm(x.cuda(), torch.ones(D, device="cuda"), eps=0.0)
    assert torch.equal(out["rstd"].cpu(), 1.0 / torch.sqrt(v * v))
