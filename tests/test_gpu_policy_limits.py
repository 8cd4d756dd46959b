"""Batches at the limits of 32-bit counts."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2605_08527_b200 import binding as B

from test_gpu_policy import dev, segments

pytestmark = pytest.mark.gpu


def test_advantages_of_two_to_the_31_less_one_tokens():
    # the last tokens' numbers and a step beyond them pass 2^31: every sequence's count and every token's value, a part at a time
    pool = B.AdapterPool(64, 64, 8, 2)
    T = (1 << 31) - 1
    off = [0, 5, 1 << 30, T - 130, T]
    slot = [0, 1, 0, 1]
    targets = torch.zeros(T, dtype=torch.int32, device="cuda")
    targets[::3] = -1
    targets[T - 2:] = torch.tensor([-5, 7], dtype=torch.int32, device="cuda")
    rewards = dev([1.0, 0.0, 0.25, 2.0], torch.float32)
    seq_adv, adv, weight = B.marlaas_group_advantages(pool, segments(off, slot), rewards, dev([0, 2, 4], torch.int32), targets)
    B.marlaas_check_status(pool)
    # two of a group: one deviation to either side
    np.testing.assert_allclose(seq_adv.cpu().numpy(), [1, -1, -1, 1], atol=1e-5)
    step = 1 << 28
    for s in range(4):
        n = sum(int((targets[i:min(i + step, off[s + 1])] >= 0).sum()) for i in range(off[s], off[s + 1], step))
        w = np.float32(1.0) / np.float32(2.0 * np.float32(n))        # two sequences of either tenant
        for i in range(off[s], off[s + 1], step):
            part = slice(i, min(i + step, off[s + 1]))
            on = targets[part] >= 0
            assert torch.equal(adv[part], torch.where(on, seq_adv[s], 0.0))
            assert torch.all((weight[part] - torch.where(on, float(w), 0.0)).abs() <= 2e-7 * float(w))


def test_more_segments_or_groups_than_can_be_counted_are_refused():
    pool = B.AdapterPool(64, 64, 8, 2)
    L, many = B.load_library(), (1 << 30) + 1
    t = torch.zeros(64, dtype=torch.int32, device="cuda")
    f = torch.zeros(64, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    assert L.marlaas_policy_workspace_bytes(pool.handle, 4, many, 1) == 0 and L.marlaas_policy_workspace_bytes(pool.handle, 4, 1, many) == 0
    n0 = B.marlaas_kernel_launch_count()
    for host in (False, True):
        tables = t.cpu() if host else t
        flags = B.MARLAAS_FLAG_HOST_TABLE if host else 0
        for S, G in ((many, 1), ((1 << 31) - 1, 1), (1, many), (1, (1 << 31) - 1)):
            seg = B.marlaas_segments_t(S, tables.data_ptr(), tables.data_ptr())
            rc = L.marlaas_group_advantages(pool.handle, 0, ctypes.byref(seg), f.data_ptr(), G, tables.data_ptr(), t.data_ptr(), 1e-6,
                                            f.data_ptr(), None, None, ws.data_ptr(), ws.numel(), flags, B._stream(None))
            assert rc == B.MARLAAS_ERR_INVALID_ARG
        seg = B.marlaas_segments_t(many, tables.data_ptr(), tables.data_ptr())
        hp = B.marlaas_policy_loss_t(0.2, 0.2, 0.0, 0.0, 1.0, 1.0)
        z = torch.zeros((4, 8), device="cuda")
        rc = L.marlaas_policy_loss(pool.handle, 4, 8, z.data_ptr(), 8, B.MARLAAS_DTYPE_F32, t.data_ptr(), ctypes.byref(seg), f.data_ptr(), None,
                                   f.data_ptr(), f.data_ptr(), ctypes.byref(hp), None, 0, None, f.data_ptr(), ws.data_ptr(), ws.numel(), flags,
                                   B._stream(None))
        assert rc == B.MARLAAS_ERR_INVALID_ARG
    assert B.marlaas_kernel_launch_count() == n0


def test_a_target_outside_the_vocabulary_is_named_as_that():
    pool = B.AdapterPool(64, 64, 8, 2)
    B.marlaas_token_logprobs(pool, torch.zeros((4, 8), device="cuda"), dev([0, 1, 8, 2], torch.int32))
    with pytest.raises(B.MarlaasError, match="vocabulary.*2$") as e:
        B.marlaas_check_status(pool)
    assert e.value.status == B.MARLAAS_ERR_DEVICE_BAD_INDEX
