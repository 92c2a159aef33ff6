"""Rows of the largest values whose squares are said to be safe."""
import pytest
import torch

import test_gpu_rms_norm as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [1, 640, 4096, 8192, 8193, 16384, 65535, 65536])
def test_values_of_2_to_60(dtype, D):
    import paper_2608_03676_b200 as P
    x = torch.full((3, D), 2.0 ** 60, dtype=dtype)
    x[1] *= torch.where(torch.arange(D) % 2 == 0, 1.0, -1.0).to(dtype)
    x[2, : D // 2] = 1.0
    w = torch.ones(D, dtype=dtype)
    out = {name: t.cpu() for name, t in P.rms_norm(x.cuda(), w.cuda(), group=128).items()}
    assert torch.isfinite(out["y"].float()).all() and (out["rstd"] > 0).all()
    R.check_norm(out, x, w, 1e-6, None, 128)
    # as a sum of two that reaches it
    half = (x.float() / 2).to(dtype)
    both = {name: t.cpu() for name, t in P.rms_norm(half.cuda(), w.cuda(), residual=half.cuda(), group=128).items()}
    R.check_norm(both, half, w, 1e-6, half, 128)
