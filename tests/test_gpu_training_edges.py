"""Calls of the training-step operators at the edges of what their documentation allows: offsets past 2^31 elements, sizes on both
sides of each change of kernel, outputs left out, and rows that hold what must not spread."""
import math

import pytest
import torch

import test_gpu_dropout as drop
import test_gpu_head as head
import test_gpu_layer_norm as norm
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pool():
    pool = B.AdapterPool(64, 64, 8, norm.CAP)
    for t in range(norm.CAP):
        B.marlaas_adapter_pool_register(pool, t, 0, 0, 1.0, None, None)
    return pool


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("T,d,S", [(148, 504, 4), (149, 512, 9), (593, 2040, 20), (592, 2048, 3), (1185, 2304, 50), (597, 3592, 60), (741, 6152, 11),
                                   (300, 16376, 25), (3000, 4096, 1000), (9000, 64, 8300), (9000, 72, 3000), (5000, 1600, 40), (4000, 520, 1)])
def test_norms_on_both_sides_of_each_change(pool, T, d, S, rms):
    norm.test_both_passes(pool, T, d, S, rms)


def test_norm_outputs_left_out(pool):
    T, d = 700, 2056
    off, slot, rows = norm.batch(T, 9, 3)
    x, dy = norm.rows_of(T, d, 4)[0], norm.rows_of(T, d, 5)[0]
    gain, bias = norm.params(d, 6)
    seg = norm.segments(off, slot)
    _, mean, rstd = B.marlaas_layer_norm(pool, x, seg, gain, bias, eps=norm.EPS)
    full = [torch.empty_like(x), torch.empty_like(gain), torch.empty_like(gain)]
    B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, mean, rstd, dx=full[0], dgain=full[1], dbias=full[2])
    for k in range(1, 8):
        got = [torch.full_like(v, 3.0) if k >> i & 1 else None for i, v in enumerate(full)]
        B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, mean, rstd, dx=got[0], dgain=got[1], dbias=got[2])
        assert all(g is None or torch.equal(g, v) for g, v in zip(got, full)), k


def test_norm_rows_far_apart(pool):
    """Rows 2^30 elements apart: the third begins at 2^31."""
    d, ld = 2048, 1 << 30
    buf = torch.zeros(2 * ld + d, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (3, d), (ld, 1))
    near = norm.rows_of(3, d, 8)[0]
    x.copy_(near)
    gain, bias = norm.params(d, 9)
    seg = norm.segments([0, 1, 3], [2, 0])
    y, mean, rstd = B.marlaas_layer_norm(pool, near, seg, gain, bias, eps=norm.EPS)
    assert torch.equal(B.marlaas_layer_norm(pool, x, seg, gain, bias, eps=norm.EPS)[0], y)
    dy = norm.rows_of(3, d, 10)[0]
    want = torch.empty_like(near)
    B.marlaas_layer_norm_backward(pool, near, dy, seg, gain, mean, rstd, dx=want)
    B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, mean, rstd, dx=x)         # in place
    assert torch.equal(x, want)


def test_head_rows_and_weights_far_apart(pool):
    T, d, V = 70, 96, 1000
    x, W, tgt, w, off, slot = head.inputs(T, d, V, 11)
    seg = head.segments(off, slot)
    dx = torch.empty_like(x)
    logp, stats = B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=dx)
    ld = 1 << 25                                        # row 64 begins at 2^31
    buf = torch.zeros((d - 1) * ld + V, dtype=torch.bfloat16, device="cuda")
    far = torch.as_strided(buf, (d, V), (ld, 1))
    far.copy_(W)
    dx1 = torch.empty_like(x)
    l1, s1 = B.marlaas_head_cross_entropy(pool, x, far, tgt, seg, weight=w, dx=dx1)
    assert torch.equal(l1, logp) and torch.equal(s1, stats) and torch.equal(dx1, dx)
    xf = torch.as_strided(buf, (T, d), (ld, 1))
    xf.copy_(x)
    l1, s1 = B.marlaas_head_cross_entropy(pool, xf, W, tgt, seg, weight=w, dx=xf)         # in place
    assert torch.equal(l1, logp) and torch.equal(s1, stats) and torch.equal(xf, dx)


@pytest.mark.parametrize("T", [100, 600])
def test_dropout_rows_far_apart(T):
    c = drop.Case(T, 128, 256, [8, 16], 5, 31)
    y, h = c.forward()
    dx, dA, dB = c.backward(h)
    ld = -(-(1 << 31) // (T - 1) // 8) * 8 + 8          # the last row begins past 2^31
    buf = torch.zeros((T - 1) * ld + 256, dtype=torch.bfloat16, device="cuda")
    near, c.x = c.x, torch.as_strided(buf, (T, 128), (ld, 1))
    c.x.copy_(near)
    y1, h1 = c.forward()
    assert torch.equal(y1, y) and torch.equal(h1, h)
    dA1, dB1 = c.grads()
    B.marlaas_lora_backward_dropout(c.pool, c.x, c.W, c.dy, c.seg, c.rates_dev, drop.SEED, drop.OFFSET, dA=dA1, dB=dB1, h_saved=h)
    assert all(torch.equal(a, b) for a, b in zip(dA1 + dB1, dA + dB))
    c.x = near
    near, c.dy = c.dy, torch.as_strided(buf, (T, 256), (ld, 1))
    c.dy.copy_(near)
    dx1, dA1, dB1 = c.backward(h)
    assert torch.equal(dx1, dx) and all(torch.equal(a, b) for a, b in zip(dA1 + dB1, dA + dB))


@pytest.mark.parametrize("parts", [None, [512, 256]])
@pytest.mark.parametrize("cap", [3, 70])
def test_dropout_gradients_on_their_own(parts, cap):
    c = drop.Case(900, 136 if parts is None else 128, sum(parts or [192]), [8, 16, 24], 40, 32, parts=parts, cap=cap)
    none = [None] * (cap - 3)
    y, h = c.forward()
    dx, dA, dB = c.backward(h)
    a, b = c.grads()
    B.marlaas_lora_backward_dropout(c.pool, c.x, c.W, c.dy, c.seg, c.rates_dev, drop.SEED, drop.OFFSET, dA=a + none)
    B.marlaas_lora_backward_dropout(c.pool, c.x, c.W, c.dy, c.seg, c.rates_dev, drop.SEED, drop.OFFSET, dB=b + none, h_saved=h)
    assert all(torch.equal(p, q) for p, q in zip(a + b, dA + dB))
    only = torch.empty_like(dx)
    B.marlaas_lora_backward_dropout(c.pool, None, c.W, c.dy, c.seg, c.rates_dev, drop.SEED, drop.OFFSET, dx=only)
    assert torch.equal(only, dx)


@pytest.mark.parametrize("T", [200, 1000])
def test_what_a_row_drops_reaches_no_other_tenant(T):
    """Blocks of tokens of several tenants: NaN where a row's own mask drops it."""
    c = drop.Case(T, 256, 128, [8, 16, 8, 24], T // 5, 33, rates=[0.5, 0.1, 0.0, 0.3])
    keep = c.keep()
    _, h = c.forward()
    dx, dA, dB = c.backward(None)
    c.x = torch.where(keep, c.x, torch.full_like(c.x, math.nan))
    assert torch.isnan(c.x).any()
    _, h1 = c.forward()
    dx1, dA1, dB1 = c.backward(None)
    assert torch.equal(h1, h) and torch.equal(dx1, dx)
    assert all(torch.equal(a, b) for a, b in zip(dA1 + dB1, dA + dB))


def test_everything_at_once_on_two_streams(pool):
    """The same pools from two streams at the same time: each has its own workspace."""
    c = drop.Case(700, 256, 384, [16, 8], 6, 34)
    x, W, tgt, w, off, slot = head.inputs(300, 256, 5003, 35)
    hseg, nseg = head.segments(off, slot), norm.segments(*norm.batch(300, 7, 36)[:2])
    gain, bias = norm.params(256, 37)

    def step():
        y, h = c.forward()
        dx, dA, dB = c.backward(h)
        hx = torch.empty_like(x)
        logp, stats = B.marlaas_head_cross_entropy(pool, x, W, tgt, hseg, weight=w, dx=hx)
        n, mean, rstd = B.marlaas_layer_norm(pool, x, nseg, gain, bias, eps=norm.EPS)
        nx, ng, nb = torch.empty_like(x), torch.empty_like(gain), torch.empty_like(gain)
        B.marlaas_layer_norm_backward(pool, x, hx, nseg, gain, mean, rstd, dx=nx, dgain=ng, dbias=nb)
        return [y, h, dx, *dA, *dB, hx, logp, stats, n, nx, ng, nb]

    want = step()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(step())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
    B.marlaas_check_status(pool)
    B.marlaas_check_status(c.pool)


@pytest.mark.parametrize("T,d,V", [(16, 200, 127), (17, 64, 128), (32, 72, 129), (33, 520, 20000), (63, 448, 191), (64, 456, 40000), (65, 456, 40000)])
def test_head_of_a_few_tokens(T, d, V):
    pool = B.AdapterPool(64, 64, 8, head.CAP)
    head.test_loss_and_gradient(pool, T, d, V)


@pytest.mark.parametrize("T,d,V", [(33, 65536, 264), (2, 64, B.MARLAAS_MAX_VOCABULARY), (260, 8, 9)])
def test_head_at_its_largest(T, d, V):
    pool = B.AdapterPool(64, 64, 8, head.CAP)
    head.test_loss_and_gradient(pool, T, d, V)


@pytest.mark.parametrize("T,K,N,ranks,S,cap", [(5, 98312, 64, [8, 16], 3, None), (600, 128, 256, [8, 16], 9, 300), (300, 128, 256, [8, 16], 9, 300),
                                               (515, 8, 8, [128], 4, None), (2, 4096, 16, [128, 1], 2, None)])
def test_dropout_at_its_largest(T, K, N, ranks, S, cap):
    c = drop.Case(T, K, N, ranks, S, T + K + N, cap=cap)
    drop.check_case(c, c.keep())


@pytest.mark.parametrize("T", [40, 700])
def test_dropout_without_any_adapter(T):
    """Slots of rank 0, and a batch of the base model alone: the plain layer's products, each a sum in its own order
    (2^-23 (n / 16 + 2) of the magnitudes) rounded once (2^-8)."""
    def near(a, b, x, W):
        size = x.double().abs() @ W.double().abs()
        assert torch.all((a.double() - b.double()).abs() <= 2 * (2.0 ** -23 * (x.shape[1] / 16 + 2) * size + 2.0 ** -8 * 1.01 * b.double().abs()))

    for ranks, on in (([0, 0], True), ([8, 16], False)):
        c = drop.Case(T, 128, 256, ranks, 4, 41)
        if not on:
            c.slot = [-1] * 4
            c.tok = [-1] * T
            c.seg = drop.segments(c.off, c.slot)
        y, h = c.forward()
        assert not h.any()
        plain = torch.empty_like(y)
        B.marlaas_lora_forward(c.pool, c.x, c.W, c.seg, y=plain)
        near(y, plain, c.x, c.W)
        dx, dA, dB = c.backward(h)
        back = torch.empty_like(dx)
        B.marlaas_lora_backward(c.pool, c.x, c.W, c.dy, c.seg, dx=back)
        near(dx, back, c.dy, c.W.T)
        assert all(g is None or not g.any() for g in dA + dB)
