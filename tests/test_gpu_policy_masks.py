"""Rows of logits with runs of -inf, as top-k filtering and constrained decoding make them, against the float64 definitions:
every warp has to count its finite logits also when the entries that it looks at first are all masked.

Vocabularies for every number of warps per row and of CTAs per row, in batches of a few rows (more CTAs each) and of more.
Tolerances as for any other row of logits (test_gpu_policy.py): a mask adds no rounding.
"""
import math

import numpy as np
import pytest
import torch

from oracle import policy as op
from paper_2605_08527_b200 import binding as B

from test_gpu_policy import dev, grad_bound, logp_close, loss_inputs, segments

pytestmark = pytest.mark.gpu

INF = math.inf


@pytest.fixture(scope="module")
def pool():
    return B.AdapterPool(64, 64, 8, 5)


def _keep_largest(z, k):
    cut = np.sort(z)[-k]
    z[z < cut] = -INF


def _first(n):
    def mask(z, r):
        z[:min(n, len(z) - 3)] = -INF
    return mask


def _part(parts, count):
    """The first `count` entries of the second of `parts` equal parts: one warp's first vectors in one CTA of a cluster."""
    def mask(z, r):
        begin = -(-len(z) // parts)
        z[max(begin - 8, 0):begin + 8 + count] = -INF
    return mask


def _window(z, r):
    a = len(z) // 2 + 3
    keep = z[a:a + 64].copy()
    z[:] = -INF
    z[a:a + 64] = keep


def _allowed(z, r):
    keep = r.choice(len(z), 64, replace=False)
    x = z[keep]
    z[:] = -INF
    z[keep] = x


def _last(z, r):
    z[:-5] = -INF


def _runs(z, r):
    for b in range(0, len(z), 128):
        if r.rand() < 0.7:
            z[b:b + 128] = -INF


def _far_below(z, r):       # all that is left is far from 0, on either side
    _first(2048)(z, r)
    z -= 80.0


def _far_above(z, r):
    _first(2048)(z, r)
    z += 80.0


MASKS = ([_first(128), _first(256), _first(2048), _first(4096), _window, _allowed, _last, _runs, _far_below, _far_above,
          lambda z, r: _keep_largest(z, 50), lambda z, r: _keep_largest(z, 1)] +
         [_part(c, n) for c in range(2, 9) for n in (128, 256)])

# warps per row (bf16): 1, 2, 4, 8, then clusters of 2 to 8; fp32 rows of half the length take the same
VOCABULARIES = [4000, 4104, 5003, 9001, 20011, 40003, 75001, 131080, 150001, 190003, 220009, 262144]


def masked_rows(T, V, dtype, seed):
    """[T][V] logits on the GPU and as float64, targets among the entries that are left."""
    r = np.random.RandomState(seed)
    z = torch.from_numpy(3 * r.randn(T, V)).to(dtype).double().numpy()
    tgt = np.zeros(T, dtype=np.int32)
    first = r.randint(len(MASKS))
    for i in range(T):
        MASKS[(first + i) % len(MASKS)](z[i], r)
        tgt[i] = r.choice(np.flatnonzero(z[i] > -INF))
    z = torch.from_numpy(z).to(dtype)
    z64 = z.double().numpy()
    unit = 4 if dtype == torch.float32 else 8
    buf = torch.full((T, -(-V // unit) * unit + unit), 777.0, dtype=dtype, device="cuda")
    buf[:, :V] = z.cuda()
    return buf, buf[:, :V], z64, tgt


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", VOCABULARIES)
@pytest.mark.parametrize("T", [1, 6, 20])
def test_rows_with_runs_of_minus_infinity(pool, T, V, dtype):
    if dtype == torch.float32:
        V = V // 2 + 1
    buf, z, z64, tgt = masked_rows(T, V, dtype, 13 * T + V)
    k = np.float64(np.float32(1 / 0.9))
    t = dev(tgt, torch.int32)
    ref_logp, ref_H = op.token_logprobs(z64, tgt, k)
    logp, H = B.marlaas_token_logprobs(pool, z, t, inv_temperature=1 / 0.9, with_entropy=True)
    logp_close(logp, ref_logp, "logp")
    logp_close(H, ref_H, "entropy")
    assert torch.equal(B.marlaas_token_logprobs(pool, z, t, inv_temperature=1 / 0.9), logp)

    old, ref, adv, w, off, slot = loss_inputs(T, z64, tgt, k, T + V, pool.capacity)
    args = (t, segments(off, slot), dev(old, torch.float32), dev(adv, torch.float32), dev(w, torch.float32))
    ts = np.repeat(slot, np.diff(off))
    for kl, ent in ((0.04, 0.0), (0.0, 0.02)):
        hp = dict(clip_low=0.2, clip_high=0.28, kl_coef=kl, entropy_coef=ent, inv_temperature=1 / 0.9)
        rs, rg, _ = op.policy_loss(z64, tgt, ts, pool.capacity, old, ref, adv, w, **{**hp, "inv_temperature": k})
        grad, lp = torch.empty_like(buf), torch.empty(T, device="cuda")
        more = dict(ref_logp=dev(ref, torch.float32) if kl else None, **hp)
        stats = B.marlaas_policy_loss(pool, z, *args, dlogits=grad[:, :V], logp=lp, **more)
        assert torch.equal(lp, logp)
        g = grad[:, :V].double().cpu().numpy()
        mag = grad_bound(z64, tgt, k, old, ref, adv, w, kl, ent, dtype)
        rel = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
        assert np.all(np.abs(g - rg) <= 3e-5 * mag + rel * np.abs(rg) + 1e-37)
        # softmax does not see a shift: a gradient's row sums to 0
        assert np.all(np.abs(g.sum(1)) <= 3e-5 * mag.sum(1) + rel * np.abs(rg).sum(1) + 1e-30)
        per = op.policy_loss(z64, tgt, np.zeros(T, dtype=int), pool.capacity, old, ref, np.abs(adv), w, **{**hp, "inv_temperature": k})[0][0]
        assert np.all(np.abs(stats.double().cpu().numpy() - rs) <= 4e-5 * (np.abs(rs) + np.abs(per).max()) + 1e-6)
        assert np.array_equal(stats[:, 7].cpu().numpy(), rs[:, 7].astype(np.float32))
        assert torch.equal(B.marlaas_policy_loss(pool, z, *args, **more), stats)
    # in place of the logits
    B.marlaas_policy_loss(pool, z, *args, dlogits=z, **more)
    assert torch.equal(z, grad[:, :V]) and torch.all(buf[:, V:] == 777.0)
    B.marlaas_check_status(pool)
