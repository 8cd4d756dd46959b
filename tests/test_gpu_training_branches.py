"""Sizes that take the training-step operators down the ways that ordinary test sizes do not: batches whose counted tokens are put in
order by kernels of their own, several pieces of rows, pools of hundreds of slots, contractions that end inside a 64-deep panel."""
import numpy as np
import pytest
import torch

import test_gpu_dropout as drop
import test_gpu_head as head
import test_gpu_layer_norm as norm
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pool():
    return B.AdapterPool(64, 64, 8, head.CAP)


@pytest.mark.parametrize("T,d,V", [(4096, 64, 300), (4097, 64, 300), (9000, 72, 1001), (5000, 64, 131072)])
def test_head_of_a_batch(pool, T, d, V):
    """The last is three pieces of rows."""
    x, W, tgt, w, off, slot = head.inputs(T, d, V, T)
    seg = head.segments(off, slot)
    ref = head.reference(x, W, tgt, w, off, slot, 0.9, 1.5)
    dx = torch.full_like(x, 9.0)
    logp, stats = B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=dx, inv_temperature=0.9, grad_scale=1.5)
    B.marlaas_check_status(pool)
    for got, i in ((logp, 0), (stats, 2), (dx, 4)):
        head.check(got, ref[i], ref[i + 1])
    ign = (tgt < 0) | (w == 0)
    assert not dx[ign].any() and not logp[ign].any()
    # without the gradient, again, and in place: the same bits
    alone = B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, inv_temperature=0.9)
    assert torch.equal(alone[0], logp) and torch.equal(alone[1], stats)
    same = x.clone()
    same[ign] = float("nan")
    l2, s2 = B.marlaas_head_cross_entropy(pool, same, W, tgt, seg, weight=w, dx=same, inv_temperature=0.9, grad_scale=1.5)
    assert torch.equal(l2, logp) and torch.equal(s2, stats) and torch.equal(same, dx)


def test_head_of_a_batch_with_a_bad_target(pool):
    T, d, V = 4500, 64, 500
    x, W, tgt, w, off, slot = head.inputs(T, d, V, 3)
    seg = head.segments(off, slot)
    tgt[[0, 1023, 4499]] = -1
    dx, dx1 = torch.empty_like(x), torch.empty_like(x)
    logp, stats = B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=dx)
    B.marlaas_check_status(pool)
    tgt[1023] = V
    l1, s1 = B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=dx1)
    with pytest.raises(B.MarlaasError) as e:
        B.marlaas_check_status(pool)
    assert e.value.status == B.MARLAAS_ERR_DEVICE_BAD_INDEX
    assert torch.equal(l1, logp) and torch.equal(s1, stats) and torch.equal(dx1, dx)
    # everything ignored
    none = torch.full_like(tgt, -1)
    l2, s2 = B.marlaas_head_cross_entropy(pool, x, W, none, seg, weight=w, dx=dx1)
    assert not l2.any() and not s2.any() and not dx1.any()


def test_head_pieces_without_a_gradient(pool):
    """A piece without kept exponentials is 65536 rows at this vocabulary."""
    T, d, V = 70000, 8, 262144
    x, W, tgt, w, off, slot = head.inputs(T, d, V, 4, ignored=0.01, zero=0.01)
    assert int(((tgt >= 0) & (w != 0)).sum()) > 65536 + 256
    logp, stats = B.marlaas_head_cross_entropy(pool, x, W, tgt, head.segments(off, slot), weight=w)
    B.marlaas_check_status(pool)
    for part in (slice(0, 40000), slice(40000, T)):         # a row's result does not depend on the other rows
        assert torch.equal(B.marlaas_head_cross_entropy(pool, x[part], W, tgt[part], weight=w[part])[0], logp[part])
    rows = torch.cat([torch.arange(0, 300), torch.arange(66500, 67300), torch.arange(T - 300, T)]).cuda()
    ref = head.reference(x[rows], W, tgt[rows], w[rows], [0, len(rows)], [0], 1.0, 1.0)
    head.check(logp[rows], ref[0], ref[1])
    # sums of the log-probabilities as they are: up to T / 256 numbers in one chain and a tree of 256, 2^-24 each
    to = torch.from_numpy(np.repeat(np.where(np.array(slot) < 0, head.CAP, slot), np.diff(off))).cuda()
    on = ((tgt >= 0) & (w != 0)).double()
    terms = torch.stack([-w.double() * logp.double(), w.double() * on, -logp.double(), on], 1)
    want, size = (torch.zeros((head.CAP + 1, 4), dtype=torch.float64, device="cuda").index_add_(0, to, v) for v in (terms, terms.abs()))
    assert torch.all((stats.double() - want).abs() <= 2.0 ** -24 * (T / 256 + 16) * size)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("cap,T,d,S", [(400, 9001, 64, 8300), (1500, 9001, 72, 8300), (4096, 20000, 64, 9000), (4096, 3000, 2048, 2900), (700, 5, 64, 3)])
def test_norm_of_many_tenants(cap, T, d, S, rms):
    """Pools whose order counts in blocks of 256 tokens; all but the last are put in order."""
    pool = B.AdapterPool(64, 64, 8, cap)
    r = np.random.RandomState(cap + T)
    off = np.sort(np.concatenate([[0, T], r.randint(0, T + 1, S - 1)]))
    slot = r.randint(-1, cap, S)
    slot[:2] = cap - 1, 0
    rows = np.repeat(np.where(slot < 0, cap, slot), np.diff(off))
    g = torch.Generator(device="cuda").manual_seed(cap)
    gain, bias = 1 + 0.3 * torch.randn((cap + 1, d), generator=g, device="cuda"), torch.randn((cap + 1, d), generator=g, device="cuda")
    x, dy = norm.rows_of(T, d, 1, shift=0.5)[0], norm.rows_of(T, d, 2)[0]
    seg, fl = norm.segments(off.tolist(), slot.tolist()), B.MARLAAS_FLAG_RMS_NORM if rms else 0
    y, mean, rstd = B.marlaas_layer_norm(pool, x, seg, gain, bias, eps=norm.EPS, flags=fl)
    norm.check_forward(x, rows, gain, bias, rms, y, mean, rstd)
    dx, dgain, dbias = torch.empty_like(x), torch.full_like(gain, 9.0), torch.full_like(bias, 9.0)
    B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, mean, rstd, dx=dx, dgain=dgain, dbias=dbias, flags=fl)
    norm.check_backward(x, dy, rows, gain, mean, rstd, rms, dx, dgain, dbias)
    absent = np.setdiff1d(np.arange(cap + 1), rows)
    assert not dgain[absent].any() and not dbias[absent].any()
    B.marlaas_check_status(pool)
    add = torch.ones_like(gain)
    B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, mean, rstd, dgain=add, flags=fl | B.MARLAAS_FLAG_ACCUMULATE)
    assert torch.equal(add, dgain + 1)


@pytest.mark.parametrize("T,K,N,ranks,S,parts", [(600, 2056, 2120, [8, 16, 64], 7, None), (2100, 1032, 1096, [16] * 5, 11, None), (513, 2632, 72, [128, 5], 3, None),
                                                 (600, 2056, 768, [8, 24], 5, [512, 256]), (1100, 4104, 2056, [16, 16], 4, None)])
def test_dropout_of_widths_that_end_inside_a_panel(T, K, N, ranks, S, parts):
    c = drop.Case(T, K, N, ranks, S, T + K, parts=parts)
    drop.check_case(c, c.keep())
    y, h = c.forward()
    y1, h1 = c.forward()
    assert torch.equal(y1, y) and torch.equal(h1, h)
