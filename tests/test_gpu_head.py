"""Cross entropy of the vocabulary head from hidden states, on the GPU against its definition in 64 bits.

Tolerances, from the arithmetic.  A logit is a sum of d products that the tensor cores add in steps of 16, each within 2^-23 of
the magnitudes added so far: it is within e_z = 2^-23 (d / 16 + 1) k sum |x w| (the largest over the vocabulary is taken), and a
log-probability within 2 e_z and, for its exponentials, sums and logarithm, 1e-5 + 1e-6 relative.  A probability of the
gradient's product carries that as a relative error and two roundings to bf16 (2^-8 each); the product's sum and the output
add 2^-23 (V / 16 + 40) of the magnitudes and half a step of bf16 (2^-8).
"""
import math

import numpy as np
import pytest
import torch

from oracle import training as ot
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu

CAP = 4


@pytest.fixture(scope="module")
def pool():
    pool = B.AdapterPool(64, 64, 8, CAP)
    for t in range(CAP):            # (tables in host memory may name registered tenants alone)
        B.marlaas_adapter_pool_register(pool, t, 0, 0, 1.0, None, None)
    return pool


def segments(off, slot, on_host=False):
    t = [torch.tensor(x, dtype=torch.int32) for x in (off, slot)]
    return B.Segments(*(t if on_host else [x.cuda() for x in t]))


def inputs(T, d, V, seed, ignored=0.2, zero=0.1, spread=2.0, ld=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ldw = ld or -(-V // 8) * 8
    W = torch.full((d, ldw), math.nan, dtype=torch.bfloat16, device="cuda")         # what lies behind the vocabulary is not read
    W[:, :V] = (spread / math.sqrt(d) * torch.randn((d, V), generator=g, device="cuda")).bfloat16()
    W = W[:, :V]
    tgt = torch.randint(0, V, (T,), generator=g, device="cuda")
    x = (torch.randn((T, d), generator=g, device="cuda") + 2 * torch.rand((T, 1), generator=g, device="cuda") * W[:, tgt].float().T).bfloat16()
    w = torch.randn(T, generator=g, device="cuda")
    w[torch.rand(T, generator=g, device="cuda") < zero] = 0.0
    tgt[torch.rand(T, generator=g, device="cuda") < ignored] = -1
    r = np.random.RandomState(seed)
    off = np.sort(np.concatenate([[0, T], r.randint(0, T + 1, 4)]))
    slot = r.randint(-1, CAP, 5)
    return x, W, tgt.int(), w, off.tolist(), slot.tolist()


def reference(x, W, targets, w, off, slot, k, scale, out_of_range=False):
    """(logp, its tolerance, stats, their tolerance, dx, its tolerance) as float64 tensors on the GPU."""
    X, Wd = x.double(), W.double()
    T, d = X.shape
    V = W.shape[1]
    on = (targets >= 0) & (targets < V) & (torch.ones_like(targets, dtype=torch.bool) if w is None else w != 0)
    wt = torch.where(on, torch.ones(T, device="cuda", dtype=torch.float64) if w is None else w.double(), 0.0)
    X = torch.where(on[:, None], X, 0.0)
    y = torch.where(on, targets, 0).long()[:, None]
    z = k * (X @ Wd)
    ez = 2.0 ** -23 * (d / 16 + 1) * k * (X.abs() @ Wd.abs()).amax(1)
    ls = torch.log_softmax(z, 1)
    logp = torch.where(on, torch.gather(ls, 1, y)[:, 0], 0.0)
    tol = torch.where(on, 2 * ez + 1e-5 + 1e-6 * logp.abs(), 0.0)
    p = torch.exp(ls)
    diff = p.clone()
    diff.scatter_add_(1, y, torch.full_like(y, -1.0, dtype=torch.float64))
    c = (scale * k * wt)[:, None]
    dx = c * (diff @ Wd.T)
    size = diff.abs() @ Wd.abs().T
    etol = c.abs() * (2.0 ** -7 * 1.01 * size + (2 * ez + 1e-5)[:, None] * 2 * (p @ Wd.abs().T) + 2.0 ** -23 * (V / 16 + 40) * size) * 1.01 + 2.0 ** -8 * dx.abs()
    slots = np.repeat(np.where(np.array(slot) < 0, CAP, slot), np.diff(off))
    to = torch.from_numpy(slots).cuda()
    stats, stol = (torch.zeros((CAP + 1, 4), dtype=torch.float64, device="cuda") for _ in range(2))
    stats.index_add_(0, to, torch.stack([-wt * logp, wt, -logp, on.double()], 1))
    stol.index_add_(0, to, torch.stack([wt.abs() * (tol + 1e-5 * logp.abs()), 1e-5 * wt.abs(), tol + 1e-5 * logp.abs(), 0 * wt], 1))
    return logp, tol, stats, stol, dx, etol


def check(got, ref, tol):
    err = (got.double() - ref).abs()
    assert torch.isfinite(got.double()).all()
    bad = err > tol
    assert not bad.any(), (int(bad.sum()), float((err - tol).max()), float(err.max()))


SIZES = [(1, 8, 1), (1, 64, 1000), (3, 72, 40), (5, 520, 257), (64, 512, 8000), (129, 136, 513), (256, 128, 256), (300, 256, 5003),
         (1000, 64, 3001), (2, 1024, 70001), (700, 320, 4096), (40, 4096, 2056)]


@pytest.mark.parametrize("T,d,V", SIZES)
def test_loss_and_gradient(pool, T, d, V):
    x, W, tgt, w, off, slot = inputs(T, d, V, T + d + V)
    k, scale = 0.8, 1.5
    seg = segments(off, slot)
    dx = torch.full_like(x, 9.0)
    logp, stats = B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=dx, inv_temperature=k, grad_scale=scale)
    B.marlaas_check_status(pool)
    rl, tl, rs, ts, rd, td = reference(x, W, tgt, w, off, slot, k, scale)
    check(logp, rl, tl)
    check(stats, rs, ts)
    check(dx, rd, td)
    off_ = (tgt < 0) | (w == 0)
    assert torch.all(dx[off_] == 0) and torch.all(logp[off_] == 0)
    # the log-probabilities alone, the same bits; and the same call the same bits
    assert torch.equal(B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, inv_temperature=k)[0], logp)
    again = torch.empty_like(x)
    l2, s2 = B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=again, inv_temperature=k, grad_scale=scale)
    assert torch.equal(again, dx) and torch.equal(l2, logp) and torch.equal(s2, stats)


def test_against_the_row_by_row_definition(pool):
    x, W, tgt, w, off, slot = inputs(6, 24, 50, 3)
    tok = np.repeat(slot, np.diff(off))
    dx = torch.empty_like(x)
    logp, stats = B.marlaas_head_cross_entropy(pool, x, W, tgt, segments(off, slot), weight=w, dx=dx, inv_temperature=1.25, grad_scale=-2.0)
    rl, rs, rd = ot.head_cross_entropy(x.double().cpu().numpy(), W.double().cpu().numpy(), tgt.tolist(), w.tolist(), tok, CAP, 1.25, -2.0)
    ref = reference(x, W, tgt, w, off, slot, 1.25, -2.0)
    for got, want, tol in ((logp, rl, ref[1]), (stats, rs, ref[3]), (dx, rd, ref[5])):
        check(got, torch.from_numpy(want).cuda(), tol)


def test_gradient_against_differences(pool):
    """dx along random directions against differences of the loss in 64 bits, for inputs that are exact in bf16."""
    x, W, tgt, w, off, slot = inputs(8, 64, 300, 5, ignored=0.0, zero=0.0)
    dx = torch.empty_like(x)
    B.marlaas_head_cross_entropy(pool, x, W, tgt, weight=w, dx=dx)
    tol = reference(x, W, tgt, w, off, slot, 1.0, 1.0)[5]
    g = torch.Generator(device="cuda").manual_seed(1)
    loss = lambda v: -(w.double() * torch.log_softmax(v @ W.double(), 1).gather(1, tgt.long()[:, None])[:, 0]).sum()     # noqa: E731
    for _ in range(5):
        u = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-5
        diff = (loss(x.double() + h * u) - loss(x.double() - h * u)) / (2 * h)
        assert abs(float((dx.double() * u).sum() - diff)) <= float((tol * u.abs()).sum()) + 1e-6


def test_pieces_of_rows(pool):
    """A vocabulary and a batch of more exponentials than one piece holds."""
    T, d, V = 2300, 64, 131072          # a piece: 2048 rows
    x, W, tgt, w, off, slot = inputs(T, d, V, 11, ignored=0.05)
    dx = torch.empty_like(x)
    logp, stats = B.marlaas_head_cross_entropy(pool, x, W, tgt, segments(off, slot), weight=w, dx=dx)
    rl, tl, rs, ts, rd, td = reference(x, W, tgt, w, off, slot, 1.0, 1.0)
    check(logp, rl, tl)
    check(stats, rs, ts)
    check(dx, rd, td)


def test_ignored_rows_may_hold_anything(pool):
    T, d, V = 300, 128, 1000
    x, W, tgt, w, off, slot = inputs(T, d, V, 12, ignored=0.4, zero=0.2)
    seg = segments(off, slot)
    a, b = torch.empty_like(x), torch.empty_like(x)
    l0, s0 = B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=a)
    ign = (tgt < 0) | (w == 0)
    x2, w2 = x.clone(), w.clone()
    x2[ign] = math.nan
    w2[tgt < 0] = math.inf
    l1, s1 = B.marlaas_head_cross_entropy(pool, x2, W, tgt, seg, weight=w2, dx=b)
    assert torch.equal(l0, l1) and torch.equal(s0, s1) and torch.equal(a, b)
    # everything ignored, and nothing at all
    none = torch.full_like(tgt, -100)
    l2, s2 = B.marlaas_head_cross_entropy(pool, x2, W, none, seg, weight=w, dx=b)
    assert not l2.any() and not s2.any() and not b.any()
    s3 = torch.full_like(s0, 5.0)
    B.marlaas_head_cross_entropy(pool, x[:0], W, tgt[:0], segments([0, 0], [1]), stats=s3, flags=B.MARLAAS_FLAG_ACCUMULATE)
    assert torch.all(s3 == 5)


def test_bad_rows_and_extreme_logits(pool):
    T, d, V = 7, 64, 700
    x, W, tgt, w, off, slot = inputs(T, d, V, 13, ignored=0.0, zero=0.0)
    x[2, 3], x[4, 0] = math.nan, math.inf
    dx = torch.empty_like(x)
    logp, _ = B.marlaas_head_cross_entropy(pool, x, W, tgt, weight=w, dx=dx)
    bad = torch.tensor([False, False, True, False, True, False, False], device="cuda")
    assert torch.isnan(logp[bad]).all() and torch.isnan(dx[bad]).all()
    rl, tl, _, _, rd, td = reference(torch.where(bad[:, None], 0.0, x.float()).bfloat16(), W, tgt, w, off, slot, 1.0, 1.0)
    check(logp[~bad], rl[~bad], tl[~bad])
    check(dx[~bad], rd[~bad], td[~bad])
    # entries of the vocabulary that are switched off by -inf, logits that differ by hundreds, one tile of -inf alone
    W = torch.zeros((64, 800), dtype=torch.bfloat16, device="cuda")
    W[0] = torch.linspace(-300, 300, 800, device="cuda").bfloat16()
    W[1, 256:512] = -math.inf
    x = torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda")
    x[:, 0] = torch.tensor([1.0, -1.0, 0.25], device="cuda")
    x[:, 1] = 1.0
    tgt = torch.tensor([799, 3, 700], dtype=torch.int32, device="cuda")
    # 0 times -inf is NaN in the product with x, so the columns are -inf through x[:, 1] = 1 alone
    logp, _ = B.marlaas_head_cross_entropy(pool, x, W, tgt)
    z = x.double()[:, :1] @ W.double()[:1]
    z[:, 256:512] = -math.inf
    ref = torch.log_softmax(z, 1).gather(1, tgt.long()[:, None])[:, 0]
    assert torch.all((logp.double() - ref).abs() <= 1e-5 + 1e-6 * z[:, [0, -1]].abs().amax(1))
    # nothing but -inf: no distribution
    W[1] = -math.inf
    logp, _ = B.marlaas_head_cross_entropy(pool, x, W, tgt)
    assert torch.all(logp == 0)


def test_targets_outside_the_vocabulary_are_reported(pool):
    x, W, tgt, w, off, slot = inputs(20, 64, 100, 14, ignored=0.0, zero=0.0)
    tgt[7] = 100
    dx = torch.empty_like(x)
    logp, _ = B.marlaas_head_cross_entropy(pool, x, W, tgt, weight=w, dx=dx)
    with pytest.raises(B.MarlaasError) as e:
        B.marlaas_check_status(pool)
    assert e.value.status == B.MARLAAS_ERR_DEVICE_BAD_INDEX
    rl, tl, _, _, rd, td = reference(x, W, tgt, w, off, slot, 1.0, 1.0)
    check(logp, rl, tl)
    check(dx, rd, td)
    assert logp[7] == 0 and not dx[7].any()


def test_pitches_host_tables_in_place_accumulation_and_no_weights(pool):
    T, d, V = 200, 136, 901
    x, W, tgt, _, off, slot = inputs(T, d, V, 15, ld=1024)
    full = torch.full((T, 200), 3.0, dtype=torch.bfloat16, device="cuda")
    full[:, :d] = x
    xv = full[:, :d]
    rl, tl, rs, ts, rd, td = reference(x, W, tgt, None, off, slot, 1.0, 1.0)
    stats = torch.full((CAP + 1, 4), 2.0, device="cuda")
    logp, stats = B.marlaas_head_cross_entropy(pool, xv, W, tgt, segments(off, slot, on_host=True), dx=xv, stats=stats,
                                               flags=B.MARLAAS_FLAG_ACCUMULATE)
    check(logp, rl, tl)
    check(stats, rs + 2, ts + 1e-6 * (rs.abs() + 2))
    check(xv, rd, td)
    assert torch.all(full[:, d:] == 3)


def test_same_as_the_calls_on_kept_logits(pool):
    """Against marlaas_lora_forward and marlaas_policy_loss, whose gradient at ratio 1 this is for weights w adv."""
    T, d, V = 260, 128, 1000
    x, W, tgt, w, off, slot = inputs(T, d, V, 16, zero=0.0)
    W = W.contiguous()
    head = B.AdapterPool(d, V, 8, CAP)
    seg = segments([0, T], [-1])
    z = B.marlaas_lora_forward(head, x, W, seg)
    adv = w
    weight = torch.full_like(w, 1.0 / T)
    old = B.marlaas_token_logprobs(head, z, tgt)
    dz = torch.empty_like(z)
    B.marlaas_policy_loss(head, z, tgt, seg, old, adv, weight, dlogits=dz)
    via = torch.empty_like(x)
    B.marlaas_lora_backward(head, x, W, dz, seg, dx=via)
    dx = torch.empty_like(x)
    logp, _ = B.marlaas_head_cross_entropy(pool, x, W, tgt, weight=weight * adv, dx=dx)
    on = tgt >= 0
    # the logits of the other way are rounded to bf16: 2^-8 of the largest, and a probability moves by that
    step = 2.0 ** -8 * z.float().abs().amax(1)
    assert torch.all((logp - old)[on].abs() <= 2 * step[on] + 1e-4)
    size = (weight * adv).abs()[:, None] * (2 * step + 2.0 ** -6)[:, None] * 2 * W.float().abs().amax(1)[None, :]
    assert torch.all((dx.float() - via.float()).abs() <= size + 2.0 ** -7 * via.float().abs())


def test_streams_and_graphs(pool):
    T, d, V = 500, 256, 3000
    x, W, tgt, w, off, slot = inputs(T, d, V, 17)
    seg = segments(off, slot)
    dx = torch.empty_like(x)
    logp, stats = B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=dx)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    d2 = torch.zeros_like(dx)
    l2, s2 = B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=d2, stream=side)
    side.synchronize()
    assert torch.equal(d2, dx) and torch.equal(l2, logp) and torch.equal(s2, stats)
    graphs, outs = [], []
    for _ in range(2):
        o = (torch.zeros_like(dx), torch.zeros_like(logp), torch.zeros_like(stats))
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=o[0], logp=o[1], stats=o[2])
        graphs.append(gr)
        outs.append(o)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graphs[0].replay()
        with torch.cuda.stream(other):
            graphs[1].replay()
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o[0], dx) and torch.equal(o[1], logp) and torch.equal(o[2], stats)
    # a replay follows what the device now holds: other tokens count
    tgt[:50] = -1
    graphs[0].replay()
    l3, s3 = B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=dx)
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], dx) and torch.equal(outs[0][1], l3) and torch.equal(outs[0][2], s3)
