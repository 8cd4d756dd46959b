"""The float64 definitions of the policy update against facts they have to satisfy (CPU)."""
import math

import numpy as np
import pytest

from oracle import policy as op


def test_advantages_are_centred_scaled_and_weights_sum_to_one_per_tenant():
    off, slot = [0, 5, 9, 9, 14, 20], [1, 0, 1, -1, 0]
    tgt = np.array([-1, 3, 4, 5, 6] + [2, 2, -1, -1] + [1] * 5 + [-1, -1, 7, 7, 7, 0])
    for token_mean in (False, True):
        sa, adv, w = op.group_advantages(off, slot, [1.0, 0.0, 0.5, 2.0, 2.0], [0, 3, 5], tgt, 1e-6, token_mean)
        assert abs(sa[:3].sum()) < 1e-12 and np.all(sa[3:] == 0)
        assert np.std(sa[:3]) == pytest.approx(1, abs=1e-5)
        t = np.repeat(slot, np.diff(off))
        for b in (-1, 0, 1):
            assert w[t == b].sum() == pytest.approx(1)
        assert np.all(w[tgt < 0] == 0) and np.all(adv[tgt < 0] == 0)


@pytest.mark.parametrize("kl,ent,tau", [(0.0, 0.0, 1.0), (0.1, 0.0, 0.7), (0.05, 0.02, 1.3)])
def test_loss_gradient_agrees_with_differences(kl, ent, tau):
    r = np.random.RandomState(3)
    T, V = 6, 7
    z, tgt = r.randn(T, V), r.randint(0, V, T)
    tgt[2] = -1
    z[4, 3] = -math.inf if tgt[4] != 3 else z[4, 3]
    old = op.token_logprobs(z, tgt, tau)[0] + np.array([0.05, -0.05, 0, 0.6, -0.6, 0.1])
    ref, adv, w = old + 0.1 * r.randn(T), r.randn(T), r.rand(T)
    kw = dict(clip_low=0.2, clip_high=0.28, kl_coef=kl, entropy_coef=ent, inv_temperature=tau)
    ts = np.array([0, 1, 0, -1, 1, 0])
    stats, grad, _ = op.policy_loss(z, tgt, ts, 2, old, ref, adv, w, **kw)
    assert stats[:, 7].tolist() == [2, 2, 1]
    h = 1e-5
    for i in range(T):
        for j in range(V):
            if not np.isfinite(z[i, j]):
                assert grad[i, j] == 0
                continue
            zp, zm = z.copy(), z.copy()
            zp[i, j] += h
            zm[i, j] -= h
            f = [op.policy_loss(x, tgt, ts, 2, old, ref, adv, w, **kw)[0][:, 0].sum() for x in (zp, zm)]
            assert grad[i, j] == pytest.approx((f[0] - f[1]) / (2 * h), abs=2e-8)
    np.testing.assert_allclose(grad.sum(1), 0, atol=1e-12)      # softmax does not see a shift


def test_a_token_outside_the_clip_keeps_only_its_kl_gradient():
    z = np.array([[0.0, 1.0, 2.0]])
    lp = op.token_logprobs(z, [2], 1.0)[0]
    for delta, A, moves in ((0.5, 1.0, False), (0.5, -1.0, True), (-0.5, -1.0, False), (-0.5, 1.0, True)):
        _, g, _ = op.policy_loss(z, [2], [0], 1, lp - delta, None, [A], [1.0], 0.2, 0.2)
        assert np.any(g != 0) == moves


def test_eight_bit_moments_keep_their_expected_value_and_their_range():
    n = 256 * 40
    bits = op.random_bits(n, 5, 1, 77, 0, 1)
    # low and high halves are uniform and uncorrelated: mean and covariance within 5 standard errors
    lo, hi = (bits & np.uint64(0xFFFF)) / 65536.0, (bits >> np.uint64(16)) / 65536.0
    assert abs(lo.mean() - 0.5) < 5 / math.sqrt(12 * n) and abs(hi.mean() - 0.5) < 5 / math.sqrt(12 * n)
    assert abs(((lo - .5) * (hi - .5)).mean()) < 5 / (12 * math.sqrt(n))
    m, v = np.full(n, -0.3), np.full(n, 0.7)
    dm, dv = op.decode_state(op.encode_state(m, v, bits), n)
    # a step of the code is at most 1/8: the rounded values average to the value
    assert abs(dm.mean() + 0.3) < 5 * 0.3 / 8 / 2 / math.sqrt(n) and abs(dv.mean() - 0.7) < 5 * 0.7 / 8 / 2 / math.sqrt(n)
    assert np.all(np.abs(dm / m - 1) < 1 / 8) and np.all(np.abs(dv / v - 1) < 1 / 8)
    # values that are codes themselves survive; tiny m become 0, tiny positive v the smallest code
    m, v = np.zeros(256), np.zeros(256)
    m[:5], v[:5] = [1.0, -1.875, 2.0 ** -12, 2.0 ** -20, 0], [1.0, 1.875, 2.0 ** -28, 2.0 ** -40, 0]
    dm, dv = op.decode_state(op.encode_state(m, v, np.zeros(256, dtype=np.uint64)), 256)
    assert dm[:5].tolist() == [1.0, -1.875, 2.0 ** -12, 0, 0]
    assert dv[:3].tolist() == [1.0, 1.875, 2.0 ** -28] and 0 < dv[3] <= 2.0 ** -30 and dv[4] == 0


def test_compact_steps_follow_the_exact_moments_on_average():
    # 200 steps at beta2 = 0.999 from a large first gradient: v has to decay, which rounding to nearest would not do
    n = 256 * 8
    theta, state = np.zeros(n), op.encode_state(np.zeros(n), np.zeros(n), np.zeros(n, dtype=np.uint64))
    hp = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0)
    v_exact = 0.0
    for step in range(1, 201):
        g = np.full(n, 1.0 if step == 1 else 0.01)
        theta, _, _, state = op.adamw_compact_step(theta, g, state, op.random_bits(n, 9, step, 1, 0, 0), step=step, **hp)
        v_exact = 0.999 * v_exact + 0.001 * g[0] ** 2
    v = op.decode_state(state, n)[1]
    # variance of the rounding walk: at most step * value * change per step, relative 1/8 * 0.001 * 200 = 0.025
    assert abs(v.mean() / v_exact - 1) < 5 * math.sqrt(0.025 / n)
