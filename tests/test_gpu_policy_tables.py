"""Host tables: refused before anything is written, whatever they hold."""
import numpy as np
import pytest
import torch

from paper_2605_08527_b200 import binding as B

from test_gpu_policy import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pool():
    p = B.AdapterPool(64, 64, 8, 3)
    for t in range(3):
        B.marlaas_adapter_pool_register(p, t, 0, 8, 1.0, torch.zeros((64, 8), dtype=torch.bfloat16, device="cuda"),
                                        torch.zeros((8, 64), dtype=torch.bfloat16, device="cuda"))
    return p


@pytest.mark.parametrize("off", [[0, 9, 4], [0, 4, 1 << 30, 4], [0, -3, 4], [0, 2, 1, 4], [0, -(1 << 31), (1 << 31) - 1, 4], [1, 4], [0, 5], [0, 3]])
def test_offsets_outside_the_batch_are_refused(pool, off):
    T = 4
    table = torch.tensor(off, dtype=torch.int32)
    seg = B.Segments(table, torch.zeros(len(off) - 1, dtype=torch.int32))
    f, t = torch.zeros(T, device="cuda"), dev(np.zeros(T), torch.int32)
    x, W = torch.zeros((T, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((64, 64), dtype=torch.bfloat16, device="cuda")
    z = torch.zeros((T, 8), device="cuda")
    n0 = B.marlaas_kernel_launch_count()
    for call in (lambda: B.marlaas_group_advantages(pool, seg, f[:len(off) - 1].contiguous(), torch.tensor([0, len(off) - 1], dtype=torch.int32), t),
                 lambda: B.marlaas_policy_loss(pool, z, t, seg, f, f, f),
                 lambda: B.marlaas_lora_forward(pool, x, W, seg),
                 lambda: B.marlaas_lora_backward(pool, x, W, x, seg, dx=x.clone()),
                 lambda: B.marlaas_lora_build_index(pool, T, seg)):
        with pytest.raises(B.MarlaasError) as e:
            call()
        assert e.value.status == B.MARLAAS_ERR_BAD_SEGMENT_TABLE
    assert B.marlaas_kernel_launch_count() == n0
