"""AdamW with 8-bit moments after a gradient whose square has left fp32's range.  The step itself leaves the master alone (its
second moment is infinite, as in the 32-bit form); afterwards the element's moments start anew, so that no master jumps.

Bound on a later step: for moments that began together, Cauchy's inequality gives |m| <= (1 - b1) / sqrt((1 - b2)
(1 - b1^2 / b2)) sqrt(v), with the corrections of step 2 and later and b1 = 0.9, b2 = 0.999 a step of 1.7 lr at most; codes
are within an eighth of the moments, 1.125 / sqrt(0.875) = 1.2 times that.  A neighbour in the block loses its m for a step
(it is below the block's range), never its v: 3 lr holds for all."""
import numpy as np
import pytest
import torch

from oracle import policy as op
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu

LR, SEED = 1e-3, 11


def moments_f32(m, v, g):
    f = np.float32
    b1, b2 = f(0.9), f(0.999)
    with np.errstate(over="ignore"):
        return b1 * m.astype(f) + (f(1) - b1) * g, b2 * v.astype(f) + ((f(1) - b2) * g) * g


def test_masters_stay_in_place_after_a_square_that_overflows():
    K, N, r = 64, 64, 8
    pool = B.AdapterPool(K, N, r, 1)
    rs = np.random.RandomState(3)
    n = K * r
    theta = {x: rs.randn(n).astype(np.float32) for x in "AB"}
    d = {x: torch.from_numpy(theta[x]).cuda() for x in "AB"}
    dg = {x: torch.empty(n, device="cuda") for x in "AB"}
    st = dict(zip("AB", B.compact_state(pool, r)))
    state = {x: np.zeros(n // 256 * 528, np.uint8) for x in "AB"}
    B.marlaas_adapter_pool_register(pool, 1, 0, r, 1.0, d["A"].bfloat16().view(K, r), d["B"].bfloat16().view(r, N))
    tables = B.CompactAdamWTables(pool, [1], [dg["A"]], [dg["B"]], [d["A"]], [d["B"]], [st["A"]], [st["B"]])
    huge = {0: 6.2e20, 5: -1e25, 130: 3e38, 255: -3e38, 256: 1e21, 511: 3.4e38}
    for step in range(1, 8):
        before = {x: d[x].cpu().numpy().copy() for x in "AB"}
        for k, x in enumerate("AB"):
            g = (1e-3 * rs.randn(n)).astype(np.float32)
            if step in (1, 5):
                for i, y in huge.items():
                    g[i] = y
            dg[x].copy_(torch.from_numpy(g))
            # the definition, from the device's masters
            bits = op.random_bits(n, SEED, step, 1, 0, k)
            m, v = moments_f32(*op.held_moments(state[x], n), g)
            c1, c2 = 1 / (1 - float(np.float32(0.9)) ** step), 1 / (1 - float(np.float32(0.999)) ** step)
            with np.errstate(invalid="ignore"):
                theta[x] = before[x] - np.float32(LR) * np.where(np.isinf(v), 0, c1 * m / (np.sqrt(c2 * v.astype(np.float64)) + 1e-8))
            state[x] = op.encode_state(m, v, bits)
        B.marlaas_adapter_pool_adamw_compact_commit(pool, tables, lr=LR, step=step, seed=SEED)
        for x in "AB":
            now = d[x].cpu().numpy()
            assert np.all(np.abs(now - before[x]) <= 3 * LR), f"step {step} {x}: {np.abs(now - before[x]).max() / LR} lr"
            np.testing.assert_allclose(now, theta[x], rtol=2e-5, atol=1e-7, err_msg=f"step {step} {x}")
            got, want = st[x].cpu().numpy().reshape(-1, 528)[:, :514], state[x].reshape(-1, 528)[:, :514]
            assert np.array_equal(got, want), f"step {step} {x}"
            if step in (1, 5):
                assert all(now[i] == before[x][i] for i in huge)


def test_small_first_moments_without_a_second_one_are_kept():
    # squares below the smallest number leave v at 0 as well: m stays and decays as it should
    K = N = 64
    pool = B.AdapterPool(K, N, 8, 1)
    z = lambda: torch.zeros(K * 8, device="cuda")       # noqa: E731
    g, gB, a, b = z(), z(), z(), z()
    g[:256] = 1e-25
    sA, sB = B.compact_state(pool, 8)
    B.marlaas_adapter_pool_register(pool, 1, 0, 8, 1.0, a.bfloat16().view(K, 8), b.bfloat16().view(8, N))
    tables = B.CompactAdamWTables(pool, [1], [g], [gB], [a], [b], [sA], [sB])
    for step in (1, 2):
        B.marlaas_adapter_pool_adamw_compact_commit(pool, tables, lr=LR, step=step, seed=SEED)
    m, v = B.marlaas_adamw_compact_state_export(pool, sA)
    # 1.9e-26 twice rounded to a code: within an eighth each time
    assert torch.all(v == 0) and torch.all((m[:256] - 1.9e-26).abs() <= 0.27 * 1.9e-26)
