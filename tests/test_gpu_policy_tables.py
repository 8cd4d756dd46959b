"""Host tables: refused before anything is written, whatever they hold, and read before the call returns."""
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


@pytest.mark.parametrize("S", [12, 3000])
def test_host_tables_may_be_overwritten_after_the_call(pool, S):
    # also where the device could read them by itself: page-locked memory
    r = np.random.RandomState(S)
    length = 20
    T = S * length
    off = torch.arange(0, T + 1, length, dtype=torch.int32)
    slot = torch.from_numpy(r.randint(-1, 3, S).astype(np.int32))
    groups = torch.arange(0, S + 1, 4, dtype=torch.int32)
    rewards, targets = dev(r.rand(S), torch.float32), dev(r.randint(-1, 8, T), torch.int32)
    z = torch.randn(T, 8, device="cuda")
    old = torch.full((T,), -2.0, device="cuda")
    seg = B.Segments(off.cuda(), slot.cuda())
    want = B.marlaas_group_advantages(pool, seg, rewards, groups.cuda(), targets)
    stats = B.marlaas_policy_loss(pool, z, targets, seg, old, want[1], want[2])
    torch.cuda.synchronize()
    for pinned in (False, True):
        tables = [t.pin_memory() if pinned else t.clone() for t in (off, slot, groups)]
        host = B.Segments(*tables[:2])
        torch.cuda._sleep(20_000_000)           # the stream is busy for some ten milliseconds
        got = B.marlaas_group_advantages(pool, host, rewards, tables[2], targets)
        for t in tables:
            t.zero_()
        torch.cuda.synchronize()
        tables[0].copy_(off), tables[1].copy_(slot)
        torch.cuda._sleep(20_000_000)
        more = B.marlaas_policy_loss(pool, z, targets, host, old, want[1], want[2])
        for t in tables:
            t.zero_()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), "pinned" if pinned else "pageable"
        assert torch.equal(more, stats), "pinned" if pinned else "pageable"
    B.marlaas_check_status(pool)
