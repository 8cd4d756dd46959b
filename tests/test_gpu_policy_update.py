"""The policy update's calls run together on the GPU, as the example does: rewards rise for every tenant, and one whole
iteration (forward, loss, backward, 8-bit AdamW commit) agrees with the same steps in float64."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import policy as op
from paper_2605_08527_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu


def _example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import policy_update
    return policy_update


def test_rewards_rise_for_every_tenant():
    history, stats, pool = _example().run(iterations=12, verbose=False)
    first, last = np.array(history[0]), np.mean(history[-3:], axis=0)
    # a quarter of the tokens is right by chance; 384 tokens per tenant and iteration: standard error 0.022
    assert np.all(np.abs(first - 0.25) < 5 * 0.022), first
    assert np.all(last > 0.25 + 10 * 0.022), last
    s = stats.cpu().numpy()
    assert np.all(s[-1] == 0) and np.all(s[:-1, 7] == 64 * 5) and np.allclose(s[:-1, 6], 1, atol=1e-5)
    for t in range(pool.capacity):
        assert B.marlaas_adapter_pool_lookup(pool, t)[3] == 24       # two commits per iteration


def test_one_update_matches_float64():
    K, V, r, tenants, L = 64, 136, 8, 3, 5
    g = torch.Generator().manual_seed(5)
    S = 6
    T = S * L
    W = (0.1 * torch.randn(K, V, generator=g)).bfloat16()
    x = torch.randn(T, K, generator=g).bfloat16()
    A = [torch.randn(K, r, generator=g).bfloat16().float() * 0.1 for _ in range(tenants)]
    Bm = [torch.randn(r, V, generator=g).bfloat16().float() * 0.1 for _ in range(tenants)]
    A, Bm = [a.bfloat16().float() for a in A], [b.bfloat16().float() for b in Bm]
    slot = np.array([0, 0, 1, 1, 2, 2])
    off, groups = np.arange(0, T + 1, L), np.array([0, 2, 4, 6])
    tgt = torch.randint(0, V, (T,), generator=g).numpy().astype(np.int32)
    tgt[::L] = -1
    rewards = np.array([1, 0, 0.5, 0.25, 0, 1], dtype=np.float32)
    hp = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.05, entropy_coef=0.01)
    adam = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.01, grad_scale=1.0, step=1)

    pool = B.AdapterPool(K, V, r, tenants)
    dev = lambda a: torch.as_tensor(a).cuda()       # noqa: E731
    dA, dB = [torch.empty(K, r, device="cuda") for _ in A], [torch.empty(r, V, device="cuda") for _ in Bm]
    mA, mB = [dev(a.clone()) for a in A], [dev(b.clone()) for b in Bm]
    for t in range(tenants):
        B.marlaas_adapter_pool_register(pool, t, 0, r, 2.0 * r, mA[t].bfloat16(), mB[t].bfloat16())
    st = [B.compact_state(pool, r) for _ in range(tenants)]
    tables = B.CompactAdamWTables(pool, range(tenants), dA, dB, mA, mB, [s[0] for s in st], [s[1] for s in st])
    seg = B.Segments(dev(off.astype(np.int32)), dev(slot.astype(np.int32)))
    targets = dev(tgt)
    _, adv, weight = B.marlaas_group_advantages(pool, seg, dev(rewards), dev(groups.astype(np.int32)), targets)
    h = torch.empty(T, pool.rank_stride, device="cuda")
    logits = B.marlaas_lora_forward(pool, dev(x), dev(W), seg, h_save=h)
    z64 = logits.double().cpu().numpy()             # the layer's own tests check it; here it is the loss's input
    old = B.marlaas_token_logprobs(pool, logits, targets)
    stats = B.marlaas_policy_loss(pool, logits, targets, seg, old, adv, weight, ref_logp=old - 0.1, dlogits=logits, **hp)
    dy64 = logits.double().cpu().numpy()
    B.marlaas_lora_backward(pool, dev(x), dev(W), logits, seg, dA=dA, dB=dB, h_saved=h)
    B.marlaas_adapter_pool_adamw_compact_commit(pool, tables, seed=3, **adam)
    B.marlaas_check_status(pool)

    ts = np.repeat(slot, L)
    _, radv, rw = op.group_advantages(off, slot, rewards, groups, tgt, 1e-6)
    rold = op.token_logprobs(z64, tgt, 1.0)[0]
    rs, rg, _ = op.policy_loss(z64, tgt, ts, tenants, rold, rold - 0.1, radv, rw, **hp)
    # advantages to 1e-5, log-probabilities to 1e-5, a bf16 result: see the loss's own test
    np.testing.assert_allclose(stats.cpu().numpy(), rs, rtol=1e-4, atol=1e-4)
    np.testing.assert_allclose(dy64, rg, rtol=2.0 ** -8, atol=2e-5 * np.abs(rg).max())
    x64 = x.double().numpy()
    for t in range(tenants):
        mine = ts == t
        gA = 2.0 * x64[mine].T @ (dy64[mine] @ Bm[t].double().numpy().T)
        gB = 2.0 * (x64[mine] @ A[t].double().numpy()).T @ dy64[mine]
        # the layer's gradients carry its split of fp32 vectors into two bf16 parts: 2^-16 of the magnitudes' sum
        for got, want, theta, master, k, state in ((dA[t], gA, A[t], mA[t], 0, st[t][0]), (dB[t], gB, Bm[t], mB[t], 1, st[t][1])):
            got = got.double().cpu().numpy()
            np.testing.assert_allclose(got, want, rtol=0, atol=1e-3 * np.abs(want).max())
            n = got.size
            th, _, _, _ = op.adamw_compact_step(theta.double().numpy().ravel(), got.ravel(), np.zeros(-(-n // 256) * 528, np.uint8),
                                                op.random_bits(n, 3, 1, t, 0, k), **adam)
            np.testing.assert_allclose(master.cpu().numpy().ravel(), th, rtol=2e-5, atol=1e-7)
            m, v = B.marlaas_adamw_compact_state_export(pool, state)
            # moments within a step of their code: an eighth
            np.testing.assert_allclose(m[:n].cpu().numpy(), 0.1 * got.ravel(), rtol=0.13, atol=0.1 * np.abs(got).max() * 2.0 ** -14)
        eA, eB = B.marlaas_adapter_pool_export(pool, t, r)
        assert torch.equal(eA, mA[t].bfloat16()) and torch.equal(eB, mB[t].bfloat16())
