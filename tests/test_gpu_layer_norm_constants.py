"""Layer norm of constant rows.  The sum of d equal bf16 numbers is exact in fp32 (8 bits of the number and 14 of the count), and
so is the sum divided by d: the mean is the constant, the row's deviations are zeros, y is the bias rounded once, and the row
adds zeros to dgain.  All equal, without a tolerance."""
import pytest
import torch

import test_gpu_layer_norm as norm
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pool():
    return B.AdapterPool(64, 64, 8, norm.CAP)


@pytest.mark.parametrize("d", [8, 24, 200, 1000, 1032, 2040, 2056, 3584, 5000, 11008, 16376, 16384])
def test_constant_rows_are_their_bias(pool, d):
    c = torch.cat([torch.arange(1, 257).float(), -torch.arange(1, 257).float() / 64, torch.tensor([0.0, 1e-3, -3e4, 1e-30, 7e33])]).bfloat16().cuda()
    T = len(c)
    x = c[:, None].expand(T, d).contiguous()
    off, slot, rows = norm.batch(T, 9, d)
    gain, bias = norm.params(d, 1)
    seg = norm.segments(off, slot)
    y, mean, rstd = B.marlaas_layer_norm(pool, x, seg, gain, bias, eps=norm.EPS)
    assert torch.equal(mean, c.float())
    assert torch.equal(y, bias[torch.from_numpy(rows).cuda()].bfloat16())
    dy, _ = norm.rows_of(T, d, 2)
    dgain = torch.full_like(gain, 9.0)
    B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, mean, rstd, dgain=dgain)
    assert not dgain.any()
