"""Columns of marlaas_policy_loss's stats that do not enter the loss.  Tolerances as in test_gpu_policy.py."""
import math

import numpy as np
import pytest
import torch

from oracle import policy as op
from paper_2605_08527_b200 import binding as B

from test_gpu_policy import dev, loss_inputs, make_logits, segments

pytestmark = pytest.mark.gpu


def test_the_kl_column_is_filled_whenever_there_is_a_reference():
    # a run without a KL term in its loss that watches the distance from its reference all the same
    pool = B.AdapterPool(64, 64, 8, 5)
    T, V = 40, 3001
    buf, z, z64, tgt = make_logits(T, V, torch.bfloat16, 77)
    old, ref, adv, w, off, slot = loss_inputs(T, z64, tgt, 1.0, 78, pool.capacity)
    ts = np.repeat(slot, np.diff(off))
    with_kl = op.policy_loss(z64, tgt, ts, pool.capacity, old, ref, adv, w, 0.2, 0.28, kl_coef=1.0)[0]
    without = op.policy_loss(z64, tgt, ts, pool.capacity, old, ref, adv, w, 0.2, 0.28)[0]
    want = without.copy()
    want[:, 2] = with_kl[:, 2]
    assert np.abs(want[:, 2]).max() > 0.01
    args = (dev(tgt, torch.int32), segments(off, slot), dev(old, torch.float32), dev(adv, torch.float32), dev(w, torch.float32))
    grad, plain = torch.empty_like(buf), torch.empty_like(buf)
    stats = B.marlaas_policy_loss(pool, z, *args, ref_logp=dev(ref, torch.float32), dlogits=grad[:, :V], clip_high=0.28)
    np.testing.assert_array_less(np.abs(stats.double().cpu().numpy() - want), 4e-5 * (np.abs(want) + T) + 1e-6)
    assert np.all(np.abs(stats[:, 2].double().cpu().numpy() - want[:, 2]) <= 4e-5 * np.abs(w).sum())
    # nothing else changes by it, a reference without a value included
    base = B.marlaas_policy_loss(pool, z, *args, dlogits=plain[:, :V], clip_high=0.28)
    keep = [0, 1, 3, 4, 5, 6, 7]
    assert torch.equal(grad[:, :V], plain[:, :V]) and torch.equal(stats[:, keep], base[:, keep]) and torch.all(base[:, 2] == 0)
    ref[np.flatnonzero(tgt >= 0)[:2]] = math.inf, math.nan
    bad = B.marlaas_policy_loss(pool, z, *args, ref_logp=dev(ref, torch.float32), dlogits=grad[:, :V], clip_high=0.28)
    assert torch.equal(grad[:, :V], plain[:, :V]) and torch.equal(bad[:, keep], base[:, keep]) and not torch.isfinite(bad[:, 2]).all()
