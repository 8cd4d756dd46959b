"""The policy update's calls on the GPU against their float64 definitions (oracle/policy.py).

Tolerances, from the arithmetic: a log-probability is a difference of an exponent (two fp32 roundings, relative to its
size) and the logarithm of a sum whose terms carry those roundings and a two-ulp exponential, summed in chains of some
tens: 1e-5 absolute + 1e-6 relative.  A ratio carries that as a relative error, a probability the same: a gradient is
within 3e-5 of the sum of its terms' magnitudes, plus half an ulp of the output type (2^-8 relative for bf16, with room for
a value at a rounding boundary).  Sums over tokens: 4e-5 of the sum of the magnitudes.
"""
import math

import numpy as np
import pytest
import torch

from oracle import policy as op
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu

INF = math.inf


@pytest.fixture(scope="module")
def pool():
    return B.AdapterPool(64, 64, 8, 5)


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def segments(off, slot, on_host=False):
    t = [torch.tensor(x, dtype=torch.int32) for x in (off, slot)]
    return B.Segments(*(t if on_host else [x.cuda() for x in t]))


# ---- advantages ----

ADV_CASES = {
    "one token": ([0, 1], [0], [1.0], [0, 1], [3]),
    "a group of one and an empty group": ([0, 3, 5], [1, 1], [0.5, 2.0], [0, 1, 1, 2], [1, -1, 2, 3, 4]),
    "empty sequences, all inactive, slot -1": ([0, 0, 4, 4, 9, 9, 12], [0, 2, 2, -1, -1, 0], [1.0, 0.0, 0.3, 0.1, 0.1, 0.1],
                                               [0, 3, 6], [5, -1, 0, 7, -1, -1, -1, -1, -100, 2, -1, 2]),
    "no tokens at all": ([0, 0, 0], [0, 1], [1.0, 3.0], [0, 2], []),
}


def _ragged(seed, S, longest, slots):
    r = np.random.RandomState(seed)
    off = np.concatenate([[0], np.cumsum(r.randint(0, longest + 1, S))])
    cuts = np.unique(np.concatenate([[0, S], r.randint(0, S, max(1, S // 5))]))
    tgt = np.where(r.rand(off[-1]) < 0.3, -1, r.randint(0, 1000, off[-1]))
    return off.tolist(), r.randint(-1, slots, S).tolist(), (r.randint(0, 3, S) / 2).tolist(), cuts.tolist(), tgt.tolist()


ADV_CASES["ragged"] = _ragged(1, 61, 40, 5)
ADV_CASES["many short sequences"] = _ragged(2, 3001, 3, 5)
ADV_CASES["few long sequences"] = _ragged(3, 3, 30000, 2)
ADV_CASES["a thousand sequences"] = _ragged(4, 1500, 40, 5)
ADV_CASES["more sequences than fit shared memory"] = _ragged(5, 2500, 90, 3)


@pytest.mark.parametrize("name", ADV_CASES)
@pytest.mark.parametrize("token_mean,no_std", [(False, False), (True, False), (False, True)])
def test_group_advantages(pool, name, token_mean, no_std):
    off, slot, rewards, groups, tgt = ADV_CASES[name]
    tgt = np.array(tgt, dtype=np.int32)
    flags = (B.MARLAAS_FLAG_TOKEN_MEAN if token_mean else 0) | (B.MARLAAS_FLAG_NO_STD if no_std else 0)
    rewards = np.array(rewards, dtype=np.float32)
    ref = op.group_advantages(off, slot, rewards.astype(np.float64), groups, tgt, 1e-6, token_mean, no_std)
    got = B.marlaas_group_advantages(pool, segments(off, slot), dev(rewards, torch.float32), dev(groups, torch.int32),
                                     dev(tgt, torch.int32), flags=flags)
    B.marlaas_check_status(pool)
    for g, r, what in zip(got, ref, ("seq_adv", "adv", "weight")):
        # a few fp32 operations on values of order 1; groups all alike are exact zeros on both sides
        np.testing.assert_allclose(g.cpu().numpy(), r, rtol=1e-5, atol=2e-6 if what != "weight" else 0, err_msg=what)
        assert np.array_equal(g.cpu().numpy() == 0, r == 0) or what != "weight"


@pytest.mark.parametrize("name", ["ragged", "a thousand sequences", "more sequences than fit shared memory"])
def test_group_advantages_of_unaligned_and_absent_outputs(pool, name):
    off, slot, rewards, groups, tgt = ADV_CASES[name]
    T, S = len(tgt), len(slot)
    r, g = dev(np.array(rewards), torch.float32), dev(groups, torch.int32)
    want = B.marlaas_group_advantages(pool, segments(off, slot), r, g, dev(np.array(tgt), torch.int32))
    t = torch.zeros(T + 1, dtype=torch.int32, device="cuda")
    t[1:] = torch.tensor(tgt)
    out = [torch.full((n + 3,), 9.0, device="cuda") for n in (S, T, T)]
    B.marlaas_group_advantages(pool, segments(off, slot), r, g, t[1:], seq_adv=out[0][1:S + 1], adv=out[1][1:T + 1], weight=out[2][2:T + 2])
    assert torch.equal(out[0][1:S + 1], want[0]) and torch.equal(out[1][1:T + 1], want[1]) and torch.equal(out[2][2:T + 2], want[2])
    assert all((o[[0, -1]] == 9.0).all() for o in out)
    # an output that is not wanted is NULL at the C boundary
    ws = torch.empty(B.marlaas_policy_workspace_bytes(pool, T, S, len(groups) - 1), dtype=torch.uint8, device="cuda")
    seg = segments(off, slot)
    for keep in range(3):
        got = [torch.full((n,), 7.0, device="cuda") for n in (S, T, T)]
        ptr = [o.data_ptr() if k == keep else None for k, o in enumerate(got)]
        rc = B.load_library().marlaas_group_advantages(pool.handle, T, seg.ref, r.data_ptr(), len(groups) - 1, g.data_ptr(),
                                                       t[1:].data_ptr(), 1e-6, *ptr, ws.data_ptr(), ws.numel(), 0, B._stream(None))
        assert rc == B.MARLAAS_OK and torch.equal(got[keep], want[keep])
        assert all((o == 7.0).all() for k, o in enumerate(got) if k != keep)


def test_group_advantages_alike_rewards_host_tables_and_streams(pool):
    off, slot, _, groups, tgt = ADV_CASES["ragged"]
    rewards = dev(np.full(61, 0.1), torch.float32)
    t = dev(np.array(tgt), torch.int32)
    a = B.marlaas_group_advantages(pool, segments(off, slot), rewards, dev(groups, torch.int32), t, eps=0.0)
    assert torch.all(a[0] == 0)
    # a named slot has to hold an adapter when the table is on the host: only slot -1 here
    host = B.marlaas_group_advantages(pool, segments(off, [-1] * 61, True), rewards, torch.tensor(groups, dtype=torch.int32), t, eps=0.0)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        again = B.marlaas_group_advantages(pool, segments(off, [-1] * 61), rewards, dev(groups, torch.int32), t, eps=0.0)
    other.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(host, again))


def test_group_advantages_refusals(pool):
    ok = dict(rewards=dev(np.zeros(2), torch.float32), group_offsets=dev([0, 2], torch.int32), targets=dev(np.zeros(4), torch.int32))
    seg = segments([0, 2, 4], [0, 1])
    n0 = B.marlaas_kernel_launch_count()
    for kw, status in ((dict(eps=-1.0), B.MARLAAS_ERR_INVALID_ARG), (dict(eps=INF), B.MARLAAS_ERR_INVALID_ARG),
                       (dict(flags=B.MARLAAS_FLAG_ACCUMULATE), B.MARLAAS_ERR_INVALID_ARG),
                       (dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), B.MARLAAS_ERR_WORKSPACE_TOO_SMALL)):
        with pytest.raises(B.MarlaasError) as e:
            B.marlaas_group_advantages(pool, seg, **{**ok, **kw})
        assert e.value.status == status
    for groups in ([1, 2], [0, 1], [0, 3, 2]):
        with pytest.raises(B.MarlaasError) as e:
            B.marlaas_group_advantages(pool, segments([0, 2, 4], [-1, -1], True), ok["rewards"], torch.tensor(groups, dtype=torch.int32), ok["targets"])
        assert e.value.status == B.MARLAAS_ERR_BAD_SEGMENT_TABLE
    with pytest.raises(AssertionError):
        B.marlaas_group_advantages(pool, seg, ok["rewards"], torch.tensor([0, 2], dtype=torch.int32), ok["targets"])
    assert B.marlaas_kernel_launch_count() == n0
    # device tables: reported, nothing out of range is touched
    for off, slot, groups, status in (([0, 9, 4], [0, 1], [0, 2], B.MARLAAS_ERR_BAD_SEGMENT_TABLE), ([0, 2, 4], [0, 7], [0, 2], B.MARLAAS_ERR_DEVICE_BAD_INDEX),
                                      ([0, 2, 4], [0, 1], [0, 5], B.MARLAAS_ERR_BAD_SEGMENT_TABLE)):
        B.marlaas_group_advantages(pool, segments(off, slot), ok["rewards"], dev(groups, torch.int32), ok["targets"])
        with pytest.raises(B.MarlaasError) as e:
            B.marlaas_check_status(pool)
        assert e.value.status == status


# ---- rows of logits ----

def make_logits(T, V, dtype, seed, extra=0, mask=None):
    """[T][V] on the GPU inside rows with a padded leading dimension, and the same values as float64."""
    r = np.random.RandomState(seed)
    z = torch.from_numpy(3 * r.randn(T, V)).to(dtype)
    tgt = r.randint(0, V, T)
    tgt[r.rand(T) < 0.2] = -1
    if mask:
        mask(z, tgt, r)
    unit = 4 if dtype == torch.float32 else 8
    ld = -(-V // unit) * unit + extra
    buf = torch.full((T, ld), 777.0, dtype=dtype, device="cuda")
    buf[:, :V] = z.cuda()
    return buf, buf[:, :V], z.double().numpy(), tgt.astype(np.int32)


def _mask_inf(z, tgt, r):
    m = torch.from_numpy(r.rand(*z.shape) < 0.6)
    keep = torch.zeros_like(m)
    for i, a in enumerate(tgt):
        keep[i, max(a, 0)] = True
    z[m & ~keep] = -INF
    z[0] = -INF             # nothing left
    if z.shape[0] > 2:
        tgt[0], tgt[2] = 0, 0
        z[2] = -INF
        z[2, 0] = 5.0       # one entry left


def _mask_lowest(z, tgt, r):
    low = torch.finfo(z.dtype).min
    m = torch.from_numpy(r.rand(*z.shape) < 0.6)
    for i, a in enumerate(tgt):
        m[i, max(a, 0)] = False
    z[m] = low
    z[0] = low              # all alike: a uniform distribution
    tgt[0] = 0


def _large(z, tgt, r):
    z *= 300.0


MASKS = {"plain": None, "minus infinity": _mask_inf, "lowest": _mask_lowest, "large": _large}
SHAPES = [(1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (7, 255), (3, 1000), (6, 4099), (150, 515), (2, 33001), (3, 70001), (2, 131080), (700, 3001), (301, 40003)]


def logp_close(got, ref, what):
    got = got.double().cpu().numpy()
    same = np.isnan(got) & np.isnan(ref) | (got == ref)
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - ref) <= 1e-5 + 1e-6 * np.abs(ref)))
    assert not bad.any(), f"{what}: {got[bad][:4]} against {ref[bad][:4]}"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("T,V", SHAPES)
def test_token_logprobs(pool, T, V, mask, dtype):
    _, z, z64, tgt = make_logits(T, V, dtype, T * 1000 + V, extra=16, mask=MASKS[mask])
    for tau in (1.0, 0.6):
        k = np.float64(np.float32(1 / tau))
        ref = op.token_logprobs(z64, tgt, k)
        logp, H = B.marlaas_token_logprobs(pool, z, dev(tgt, torch.int32), inv_temperature=1 / tau, with_entropy=True)
        B.marlaas_check_status(pool)
        logp_close(logp, ref[0], "logp")
        logp_close(H, ref[1], "entropy")
        only = B.marlaas_token_logprobs(pool, z, dev(tgt, torch.int32), inv_temperature=1 / tau)
        assert torch.equal(only, logp)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_bad_logits_show_in_their_row_only(pool, dtype):
    _, z, z64, tgt = make_logits(6, 3001, dtype, 5)
    tgt[:] = [4, 4, 4, -1, 4, 3000]
    z[1, 2999], z[2, 17], z[3, 0], z[5, 3000] = math.nan, INF, math.nan, -INF
    z64[5, 3000] = -INF
    logp, H = B.marlaas_token_logprobs(pool, z, dev(tgt, torch.int32), with_entropy=True)
    ref = op.token_logprobs(np.where(np.isfinite(z64) | (z64 == -INF), z64, 0), tgt, 1.0)
    assert torch.isnan(logp[1:3]).all() and torch.isnan(H[1:3]).all()
    logp_close(logp[[0, 3, 4, 5]], ref[0][[0, 3, 4, 5]], "logp")       # a target of probability 0: -inf
    assert logp[5].item() == -INF


def loss_inputs(T, z64, tgt, k, seed, slots):
    r = np.random.RandomState(seed)
    base = op.token_logprobs(z64, tgt, k)[0]
    base = np.where(np.isfinite(base), base, 0)
    # ratios of all kinds, none nearer to the clip's edges than rounding
    delta = 0.3 * r.randn(T)
    for edge in (math.log(0.8), math.log(1.28)):
        delta = np.where(np.abs(delta - edge) < 1e-3, delta + 3e-3, delta)
    f = lambda x: x.astype(np.float32)      # noqa: E731
    adv = f(r.randn(T))
    adv[r.rand(T) < 0.1] = 0
    w = f(r.rand(T))
    off = np.unique(np.concatenate([[0, T], r.randint(0, T + 1, 4)]))
    slot = r.randint(-1, slots, len(off) - 1)
    return f(base - delta), f(base + 0.2 * r.randn(T)), adv, w, off.tolist(), slot.tolist()


def grad_bound(z64, tgt, k, old, ref, adv, w, kl, ent, dtype):
    """Sum of the magnitudes of a gradient's terms."""
    out = np.zeros_like(z64)
    for i in range(len(tgt)):
        y = op._distribution(z64[i], k) if tgt[i] >= 0 else None
        if y is None:
            continue
        p, lp = np.exp(y), y[tgt[i]]
        c = np.exp(lp - float(old[i])) * abs(float(adv[i])) + (kl * (1 + np.exp(float(ref[i]) - lp)) if kl else 0)
        H = -(p[p > 0] * y[p > 0]).sum()
        b = p * c
        b[p > 0] += ent * p[p > 0] * (np.abs(y[p > 0]) + H)
        b[tgt[i]] += c
        out[i] = abs(float(w[i])) * k * b
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mask,kl,ent", [("plain", 0.0, 0.0), ("minus infinity", 0.05, 0.0), ("lowest", 0.05, 0.02), ("plain", 0.0, 0.02)])
@pytest.mark.parametrize("T,V", SHAPES)
def test_policy_loss(pool, T, V, mask, kl, ent, dtype):
    buf, z, z64, tgt = make_logits(T, V, dtype, 7 * T + V, extra=8, mask=MASKS[mask])
    k = np.float64(np.float32(1 / 0.8))
    old, ref, adv, w, off, slot = loss_inputs(T, z64, tgt, k, T + V, pool.capacity)
    ts = np.repeat(slot, np.diff(off))
    hp = dict(clip_low=0.2, clip_high=0.28, kl_coef=kl, entropy_coef=ent, inv_temperature=1 / 0.8, grad_scale=3.0)
    rs, rg, rl = op.policy_loss(z64, tgt, ts, pool.capacity, old, ref, adv, w, **{**hp, "inv_temperature": k})
    args = (dev(tgt, torch.int32), segments(off, slot), dev(old, torch.float32), dev(adv, torch.float32), dev(w, torch.float32))
    refs = dev(ref, torch.float32) if kl else None
    grad = torch.full_like(buf, 55.0)
    logp = torch.empty(T, dtype=torch.float32, device="cuda")
    stats = B.marlaas_policy_loss(pool, z, *args, ref_logp=refs, dlogits=grad[:, :V], logp=logp, **hp)
    B.marlaas_check_status(pool)
    logp_close(logp, rl, "logp")
    assert torch.all(grad[:, V:] == 55.0) and torch.all(buf[:, V:] == 777.0)
    bound = 3.0 * 3e-5 * grad_bound(z64, tgt, k, old, ref, adv, w, kl, ent, dtype) + (2.0 ** -8 * np.abs(rg) if dtype == torch.bfloat16 else 0) + 1e-37
    err = np.abs(grad[:, :V].double().cpu().numpy() - rg)
    assert np.all(err <= bound), f"gradient: {(err / bound).max()} of the bound at {np.unravel_index(np.argmax(err / bound), err.shape)}"
    # the terms' magnitudes per slot: the stats of the absolute values
    mag = np.abs(rs) + 0.0
    per = op.policy_loss(z64, tgt, np.zeros(T, dtype=int), pool.capacity, old, ref, np.abs(adv), w, **{**hp, "inv_temperature": k})[0][0]
    np.testing.assert_array_less(np.abs(stats.double().cpu().numpy() - rs), 4e-5 * (mag + np.abs(per)[None, :].max()) + 1e-6)
    assert np.array_equal(stats[:, 7].cpu().numpy(), rs[:, 7].astype(np.float32))
    # without a gradient, without logp: the same stats; added to what is there
    more = B.marlaas_policy_loss(pool, z, *args, ref_logp=refs, **hp)
    assert torch.equal(more, stats)
    B.marlaas_policy_loss(pool, z, *args, ref_logp=refs, stats=more, flags=B.MARLAAS_FLAG_ACCUMULATE, **hp)
    assert torch.equal(more, 2 * stats)
    # the rollout's call on the same batch gives the same log-probabilities, bit for bit
    assert torch.equal(B.marlaas_token_logprobs(pool, z, args[0], inv_temperature=1 / 0.8), logp)
    # in place of the logits
    B.marlaas_policy_loss(pool, z, *args, ref_logp=refs, dlogits=z, **hp)
    assert torch.equal(z, grad[:, :V]) and torch.all(buf[:, V:] == 777.0)


def test_gradient_agrees_with_differences_of_the_loss(pool):
    # fp32, a small vocabulary: central differences of the GPU's own loss.  The loss is of order 1 with an error of some
    # 1e-6, so a difference over 2 * 0.02 is good to 1e-4; the third-order term is below h^2 = 4e-4 times the slope
    T, V, h = 5, 11, 0.02
    _, z, z64, tgt = make_logits(T, V, torch.float32, 31)
    tgt[:] = np.arange(T)
    old, ref, adv, w, off, slot = loss_inputs(T, z64, tgt, 1.0, 8, pool.capacity)
    old = (op.token_logprobs(z64, tgt, 1.0)[0] - np.array([0.05, -0.05, 0.6, -0.6, 0.1])).astype(np.float32)
    kw = dict(ref_logp=dev(ref, torch.float32), kl_coef=0.1, entropy_coef=0.05, clip_low=0.2, clip_high=0.2)
    args = (dev(tgt, torch.int32), segments(off, slot), dev(old, torch.float32), dev(adv, torch.float32), dev(w, torch.float32))
    grad = torch.empty((T, 12), device="cuda")[:, :V]
    B.marlaas_policy_loss(pool, z, *args, dlogits=grad, **kw)
    for i in range(T):
        for j in range(V):
            f = []
            for s in (h, -h):
                zz = torch.empty((T, 12), device="cuda")[:, :V].copy_(z)
                zz[i, j] += s
                f.append(B.marlaas_policy_loss(pool, zz, *args, **kw)[:, 0].double().sum().item())
            assert abs(grad[i, j].item() - (f[0] - f[1]) / (2 * h)) < 3e-3


def test_tokens_of_weight_zero_contribute_nothing_whatever_they_hold(pool):
    T, V = 4, 100
    _, z, _, tgt = make_logits(T, V, torch.bfloat16, 6)
    tgt[:] = 3
    nan = torch.full((T,), math.nan, device="cuda")
    nan[2] = -1.0
    w = torch.tensor([0.0, 0.0, 0.5, 0.0], device="cuda")
    z[0, 5] = math.nan
    grad = torch.full((T, 104), 9.0, dtype=torch.bfloat16, device="cuda")[:, :V]
    stats = B.marlaas_policy_loss(pool, z, dev(tgt, torch.int32), segments([0, 4], [1]), nan, nan, w, ref_logp=nan, dlogits=grad, kl_coef=0.1)
    assert torch.isfinite(stats).all() and stats[1, 7].item() == 1 and stats[1, 6].item() == 0.5
    assert torch.all(grad[[0, 1, 3]] == 0) and torch.isfinite(grad).all() and grad[2].abs().sum() > 0
    # a bad value of a token that counts shows in its tenant's row and its own gradient alone
    w[1] = 1.0
    stats = B.marlaas_policy_loss(pool, z, dev(tgt, torch.int32), segments([0, 2, 4], [0, 1]), nan, nan, w, ref_logp=nan, dlogits=grad, kl_coef=0.1)
    assert torch.isnan(stats[0, 0]) and torch.isfinite(stats[1:]).all()
    assert torch.isnan(grad[1]).all() and torch.isfinite(grad[[0, 2, 3]]).all()


def test_extreme_ratios(pool):
    # a ratio that overflows: clipped where the advantage is positive, 0 where it is 0, infinite where it is negative
    z = torch.zeros((3, 8), device="cuda")
    z[:, 1] = 2.0
    old = torch.full((3,), -200.0, device="cuda")
    stats = B.marlaas_policy_loss(pool, z, dev(np.ones(3), torch.int32), segments([0, 1, 2, 3], [0, 1, 2]), old,
                                  torch.tensor([1.5, 0.0, -1.0], device="cuda"), torch.ones(3, device="cuda"), dlogits=torch.empty_like(z))
    assert stats[0, 1].item() == pytest.approx(-1.2 * 1.5) and stats[0, 5].item() == 1
    assert stats[1, 1].item() == 0 and stats[2, 1].item() == INF


def test_a_target_without_probability_has_an_infinite_kl_and_leaves_the_other_rows_alone(pool):
    z = torch.zeros((3, 16), device="cuda")
    z[1, 4] = -INF
    f = torch.full((3,), -2.5, device="cuda")
    grad = torch.empty_like(z)
    stats = B.marlaas_policy_loss(pool, z, dev(np.full(3, 4), torch.int32), segments([0, 1, 2, 3], [0, 1, 2]), f, torch.ones(3, device="cuda"),
                                  torch.ones(3, device="cuda"), ref_logp=f, dlogits=grad, kl_coef=0.1)
    assert stats[1, 2].item() == INF and stats[1, 0].item() == INF and stats[1, 4].item() == 0
    assert torch.isfinite(stats[[0, 2]]).all() and torch.isfinite(grad[[0, 2]]).all()


def test_offsets_past_two_to_the_31(pool):
    V = 131072
    T = (1 << 31) // V + 40
    z = torch.empty((T, V), dtype=torch.bfloat16, device="cuda").normal_()
    grad = torch.full_like(z, 1.0)
    rows = [0, 7, T // 2, T - 2, T - 1]
    tgt = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    tgt[rows] = torch.tensor([0, 5, 131071, 3, 131070], dtype=torch.int32, device="cuda")
    one = torch.ones(T, device="cuda")
    logp = torch.empty(T, device="cuda")
    B.marlaas_policy_loss(pool, z, tgt, segments([0, T], [0]), one * -12.0, one, one, dlogits=grad, logp=logp, clip_high=1e9)
    ref = torch.log_softmax(z[rows].double(), 1)
    at = ref.gather(1, tgt[rows].long()[:, None])[:, 0]
    logp_close(logp[rows], at.cpu().numpy(), "logp")
    rho = torch.exp(at + 12.0)[:, None]
    want = rho * ref.exp()
    want[torch.arange(5), tgt[rows].long()] -= rho[:, 0]
    err = (grad[rows].double() - want).abs()
    assert torch.all(err <= 2.0 ** -8 * want.abs() + 6e-5 * rho)
    assert all((grad[i] == 0).all() for i in (1, 6, T // 2 + 1, T - 3)) and logp[1].item() == 0


@pytest.mark.parametrize("T,V,dtype", [(8300, 34001, torch.bfloat16), (9001, 8193, torch.float32), (1500, 33000, torch.float32)])
def test_more_rows_than_the_device_holds_at_once(pool, T, V, dtype):
    # rows of a quarter ignored tokens, in runs; torch's float64 log-softmax is the reference, a part of the rows at a time
    unit = 4 if dtype == torch.float32 else 8
    z = torch.empty((T, -(-V // unit) * unit), dtype=dtype, device="cuda").normal_(0, 3)[:, :V]
    tgt = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    tgt[(torch.arange(T, device="cuda") // 37) % 4 == 0] = -1
    old = torch.full((T,), -9.0, device="cuda")
    adv, w = torch.randn(T, device="cuda"), torch.rand(T, device="cuda")
    grad = torch.empty_strided(z.shape, z.stride(), dtype=dtype, device="cuda")
    logp = torch.empty(T, device="cuda")
    stats = B.marlaas_policy_loss(pool, z, tgt, segments([0, T // 3, T], [2, 0]), old, adv, w, dlogits=grad, logp=logp, clip_low=1e9, clip_high=1e9)
    B.marlaas_check_status(pool)
    assert torch.equal(B.marlaas_token_logprobs(pool, z, tgt), logp)
    total = torch.zeros(2, dtype=torch.float64, device="cuda")
    for i in range(0, T, 500):
        y = torch.log_softmax(z[i:i + 500].double(), 1)
        live = tgt[i:i + 500] >= 0
        a = tgt[i:i + 500].clamp(min=0).long()[:, None]
        lp = torch.where(live, y.gather(1, a)[:, 0], 0.0)
        assert torch.all((logp[i:i + 500].double() - lp).abs() <= 1e-5 + 1e-6 * lp.abs())
        c = torch.exp(lp + 9.0) * adv[i:i + 500].double() * w[i:i + 500].double() * live
        want = y.exp() * c[:, None]
        want.scatter_add_(1, a, -c[:, None])
        err, size = (grad[i:i + 500].double() - want).abs(), want.abs()
        assert torch.all(err <= (2.0 ** -8 if dtype == torch.bfloat16 else 0) * size + 6e-5 * (size + 1e-3 * c.abs()[:, None]) + 1e-37)
        rows = torch.arange(i, min(i + 500, T), device="cuda")
        total += torch.stack([(-c * (rows < T // 3)).sum(), (-c * (rows >= T // 3)).sum()])
    assert torch.allclose(stats[[2, 0], 1].double(), total, rtol=1e-4, atol=1e-4 * total.abs().max().item())
    assert stats[[2, 0], 7].sum().item() == (tgt >= 0).sum().item()


def test_stats_of_many_tenants_and_a_single_row_of_any_stride(pool):
    many = B.AdapterPool(64, 64, 1, 700)
    T, V = 200, 72
    z = torch.randn(T, V, device="cuda")
    slot = torch.randint(-1, 700, (T,)).tolist()
    one = torch.ones(T, device="cuda")
    stats = torch.full((701, 8), 5.0, device="cuda")
    B.marlaas_policy_loss(many, z, dev(np.zeros(T), torch.int32), segments(list(range(T + 1)), slot), one * -4, one, one, stats=stats)
    want = np.bincount([s if s >= 0 else 700 for s in slot], minlength=701)
    assert np.array_equal(stats[:, 7].cpu().numpy(), want) and torch.all(stats[torch.from_numpy(want == 0)] == 0)
    more = stats.clone()
    B.marlaas_policy_loss(many, z, dev(np.zeros(T), torch.int32), segments(list(range(T + 1)), slot), one * -4, one, one, stats=more,
                          flags=B.MARLAAS_FLAG_ACCUMULATE)
    assert torch.equal(more, 2 * stats)
    row = torch.randn(3 * 85, device="cuda").as_strided((1, V), (85, 1))
    logp = B.marlaas_token_logprobs(pool, row, dev(np.full(1, 7), torch.int32))
    logp_close(logp, torch.log_softmax(row.double(), 1)[:, 7].cpu().numpy(), "logp")


@pytest.mark.parametrize("T,V", [(500, 40003), (600, 100), (3, 100)])
def test_batches_without_a_row_to_read(pool, T, V):
    z = torch.full((T, -(-V // 8) * 8), math.nan, dtype=torch.bfloat16, device="cuda")[:, :V]
    grad = torch.full((T, -(-V // 8) * 8), 3.0, dtype=torch.bfloat16, device="cuda")[:, :V]
    f = torch.full((T,), math.nan, device="cuda")
    logp = torch.full((T,), 7.0, device="cuda")
    stats = B.marlaas_policy_loss(pool, z, dev(np.full(T, -1), torch.int32), segments([0, T], [1]), f, f, f, dlogits=grad, logp=logp)
    assert torch.all(grad == 0) and torch.all(logp == 0) and torch.all(stats == 0)
    B.marlaas_check_status(pool)


def test_a_call_on_a_stream_of_its_own(pool):
    # the stream is an argument, the outputs are allocated by the call while another stream is current
    _, z, z64, tgt = make_logits(40, 3001, torch.bfloat16, 12)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for st in (side, side.cuda_stream):
        logp, H = B.marlaas_token_logprobs(pool, z, dev(tgt, torch.int32), with_entropy=True, stream=st)
        side.synchronize()
        logp_close(logp, op.token_logprobs(z64, tgt, 1.0)[0], "logp")
        one = torch.ones(40, device="cuda")
        torch.cuda.synchronize()
        stats = B.marlaas_policy_loss(pool, z, dev(tgt, torch.int32), segments([0, 40], [0]), one, one, one, stream=st)
        side.synchronize()
        assert stats[0, 7].item() == (tgt >= 0).sum()


def test_calls_can_be_captured_and_run_on_another_stream(pool):
    _, z, _, tgt = make_logits(33, 5003, torch.bfloat16, 9)
    old, ref, adv, w = (torch.rand(33, device="cuda") - 3 for _ in range(4))
    t, seg = dev(tgt, torch.int32), segments([0, 20, 33], [0, 4])
    grad = torch.empty((33, 5008), dtype=torch.bfloat16, device="cuda")[:, :5003]
    stats = B.marlaas_policy_loss(pool, z, t, seg, old, adv, w, ref_logp=ref, dlogits=grad, kl_coef=0.1).clone()
    g0 = grad.clone()
    ws = torch.empty(B.marlaas_policy_workspace_bytes(pool, 33, 2), dtype=torch.uint8, device="cuda")
    st = torch.empty_like(stats)
    grad.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            B.marlaas_policy_loss(pool, z, t, seg, old, adv, w, ref_logp=ref, dlogits=grad, kl_coef=0.1, stats=st, workspace=ws)
    for _ in range(3):
        grad.zero_()
        st.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(st, stats) and torch.equal(grad, g0)


def test_row_calls_refuse(pool):
    z = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    t, seg, f = dev(np.zeros(4), torch.int32), segments([0, 4], [0]), torch.zeros(4, device="cuda")
    n0 = B.marlaas_kernel_launch_count()

    def refused(status, fn, *a, **kw):
        with pytest.raises(B.MarlaasError) as e:
            fn(pool, *a, **kw)
        assert e.value.status == status, e.value

    inv = B.MARLAAS_ERR_INVALID_ARG
    for bad in (0.0, -1.0, INF, math.nan, 3e38):
        refused(inv, B.marlaas_token_logprobs, z, t, inv_temperature=bad)
        refused(inv, B.marlaas_policy_loss, z, t, seg, f, f, f, inv_temperature=bad)
    refused(inv, B.marlaas_token_logprobs, z[:, 1:], t)                             # rows off their 16-byte boundary
    refused(inv, B.marlaas_token_logprobs, torch.zeros((4, 65), dtype=torch.bfloat16, device="cuda"), t)
    refused(inv, B.marlaas_token_logprobs, z, t, flags=B.MARLAAS_FLAG_ACCUMULATE)
    refused(inv, B.marlaas_policy_loss, z, t, seg, f, f, f, kl_coef=0.1)            # no reference
    refused(inv, B.marlaas_policy_loss, z, t, seg, f, f, f, clip_low=-0.1)
    refused(inv, B.marlaas_policy_loss, z, t, seg, f, f, f, clip_high=math.nan)
    refused(inv, B.marlaas_policy_loss, z, t, seg, f, f, f, entropy_coef=INF)
    refused(inv, B.marlaas_policy_loss, z, t, seg, f, f, f, dlogits=torch.zeros(5 * 64, dtype=torch.bfloat16, device="cuda")[1:257].view(4, 64))
    refused(inv, B.marlaas_policy_loss, z, t, seg, f, f, f, logp=f)                 # an input
    both = torch.zeros((5, 64), dtype=torch.bfloat16, device="cuda")
    refused(inv, B.marlaas_policy_loss, both[:4], t, seg, f, f, f, dlogits=both[1:])
    refused(inv, B.marlaas_policy_loss, z, t, seg, f, f, f, flags=B.MARLAAS_FLAG_REUSE_PLAN)
    refused(B.MARLAAS_ERR_WORKSPACE_TOO_SMALL, B.marlaas_policy_loss, z, t, seg, f, f, f, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    refused(B.MARLAAS_ERR_BAD_SEGMENT_TABLE, B.marlaas_policy_loss, z, t, segments([0, 3], [-1], True), f, f, f)
    for bad in (t.long(), t[:3], t[::2]):
        with pytest.raises(AssertionError):
            B.marlaas_token_logprobs(pool, z, bad)
    for args in ((z.half(), t), (z.cpu(), t), (z, t.cpu())):
        with pytest.raises(AssertionError):
            B.marlaas_token_logprobs(pool, *args)
    for k in range(3):
        with pytest.raises(AssertionError):
            B.marlaas_policy_loss(pool, z, t, seg, *[f.cpu() if i == k else f for i in range(3)])
    assert B.marlaas_kernel_launch_count() == n0
    # a target past the vocabulary: reported, its row ignored
    t[2] = 64
    logp = B.marlaas_token_logprobs(pool, z, t)
    assert logp[2].item() == 0 and logp[1].item() == pytest.approx(-math.log(64), abs=1e-5)
    with pytest.raises(B.MarlaasError) as e:
        B.marlaas_check_status(pool)
    assert e.value.status == B.MARLAAS_ERR_DEVICE_BAD_INDEX
    # no tokens
    e0 = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    f0 = torch.empty(0, device="cuda")
    assert B.marlaas_token_logprobs(pool, e0, t[:0]).numel() == 0
    assert torch.all(B.marlaas_policy_loss(pool, e0, t[:0], segments([0], []), f0, f0, f0) == 0)
