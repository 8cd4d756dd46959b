"""Layer norm and RMS norm with parameters per tenant, on the GPU against their float64 definitions (oracle/training.py).

Tolerances, from the arithmetic: a row's sums run over at most 128 elements in one chain and a tree of the rest, fp32: the mean
and the variance are within 1e-5 of the sums of their terms' magnitudes.  An output carries that, and half a step of bf16
(2^-8 relative).  The gradients of the parameters are sums over up to a few hundred tokens in one chain and a tree: 2e-5 of
the sum of the magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import training as ot
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu

CAP, EPS = 5, 1e-5
HALF = 2.0 ** -8


@pytest.fixture(scope="module")
def pool():
    pool = B.AdapterPool(64, 64, 8, CAP)
    for t in range(CAP):            # (tables in host memory may name registered tenants alone)
        B.marlaas_adapter_pool_register(pool, t, 0, 0, 1.0, None, None)
    return pool


def segments(off, slot, on_host=False):
    t = [torch.tensor(x, dtype=torch.int32) for x in (off, slot)]
    return B.Segments(*(t if on_host else [x.cuda() for x in t]))


def batch(T, S, seed=0):
    """S segments over T tokens, some empty, slots -1 .. CAP - 1; the row of the parameters per token."""
    r = np.random.RandomState(seed)
    off = np.sort(np.concatenate([[0, T], r.randint(0, T + 1, S - 1)]))
    slot = r.randint(-1, CAP, S)
    return off.tolist(), slot.tolist(), np.repeat(np.where(slot < 0, CAP, slot), np.diff(off))


def rows_of(T, d, seed, ld=None, scale=1.0, shift=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    full = torch.full((T, ld or d), 7.0, dtype=torch.bfloat16, device="cuda")
    full[:, :d] = (scale * torch.randn((T, d), generator=g, device="cuda") + shift).bfloat16()
    return full[:, :d], full


def params(d, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return 1 + 0.3 * torch.randn((CAP + 1, d), generator=g, device="cuda"), torch.randn((CAP + 1, d), generator=g, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def check_forward(x, rows, gain, bias, rms, y, mean, rstd):
    xn, g = f64(x), f64(gain)[rows]
    ry, rm, rr = ot.layer_norm(xn, rows, f64(gain), None if bias is None else f64(bias), EPS, rms)
    size = np.abs(xn) + np.abs(xn).mean(1, keepdims=True)
    bound = HALF * np.abs(ry) + 1e-5 * ((size * rr[:, None] + np.abs(xn - rm[:, None]) * rr[:, None]) * np.abs(g) + np.abs(ry))
    assert np.all(np.abs(f64(y) - ry) <= bound)
    assert np.all(np.abs(f64(mean) - rm) <= 1e-5 * np.abs(xn).mean(1))
    assert np.all(np.abs(f64(rstd) - rr) <= 1e-5 * rr * (1 + np.abs(xn).mean(1) * np.abs(rm) * rr * rr))


def check_backward(x, dy, rows, gain, mean, rstd, rms, dx, dgain, dbias, add=0.0):
    xn, dn, g = f64(x), f64(dy), f64(gain)[rows]
    m, r = f64(mean), f64(rstd)
    rdx, rg, rb = ot.layer_norm_backward(xn, dn, rows, f64(gain), m, r, rms)
    xh = (xn if rms else xn - m[:, None]) * r[:, None]
    a = np.abs(dn * g)
    fuzz = 2.0 ** -22 * (np.abs(xn) + np.abs(m)[:, None]) * r[:, None]          # of xh
    if dx is not None:
        size = a + a.mean(1, keepdims=True) + (np.abs(xh) + fuzz) * (a * np.abs(xh)).mean(1, keepdims=True)
        assert np.all(np.abs(f64(dx) - rdx) <= HALF * np.abs(rdx) + 2e-5 * r[:, None] * size)
    for got, ref, terms in ((dgain, rg, np.abs(dn) * (np.abs(xh) + fuzz)), (dbias, rb, np.abs(dn))):
        if got is not None:
            size = np.zeros(ref.shape)
            np.add.at(size, rows, terms)
            assert np.all(np.abs(f64(got) - (ref + add)) <= 2e-5 * (size + abs(add)))


SIZES = [(1, 8, 1), (2, 64, 2), (7, 1000, 3), (64, 1024, 9), (33, 4096, 5), (300, 4104, 40), (1025, 264, 1025), (5000, 72, 3),
         (2500, 520, 30), (65, 8192, 4), (40, 8200, 6), (19, 16384, 2)]


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("T,d,S", SIZES)
def test_both_passes(pool, T, d, S, rms):
    off, slot, rows = batch(T, S, T + d)
    x, _ = rows_of(T, d, 1, shift=0.5)
    dy, _ = rows_of(T, d, 2, scale=0.1)
    gain, bias = params(d, 3)
    fl = B.MARLAAS_FLAG_RMS_NORM if rms else 0
    seg = segments(off, slot)
    y, mean, rstd = B.marlaas_layer_norm(pool, x, seg, gain, None if rms else bias, eps=EPS, flags=fl)
    check_forward(x, rows, gain, None if rms else bias, rms, y, mean, rstd)
    dx, dgain, dbias = torch.empty_like(x), torch.full_like(gain, 9.0), torch.full_like(bias, 9.0)
    B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, mean, rstd, dx=dx, dgain=dgain, dbias=dbias, flags=fl)
    check_backward(x, dy, rows, gain, mean, rstd, rms, dx, dgain, dbias)
    absent = sorted(set(range(CAP + 1)) - set(rows.tolist()))
    assert torch.all(dgain[absent] == 0) and torch.all(dbias[absent] == 0)
    B.marlaas_check_status(pool)
    # the same call gives the same bits
    again, g2, b2 = torch.empty_like(x), torch.empty_like(gain), torch.empty_like(bias)
    B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, mean, rstd, dx=again, dgain=g2, dbias=b2, flags=fl)
    assert torch.equal(again, dx) and torch.equal(g2, dgain) and torch.equal(b2, dbias)


def test_large_batch_of_one_tenant(pool):
    T, d = 30011, 256
    x, _ = rows_of(T, d, 4, scale=3.0, shift=-2.0)
    dy, _ = rows_of(T, d, 5)
    gain, bias = params(d, 6)
    seg, rows = segments([0, T], [2]), np.full(T, 2)
    y, mean, rstd = B.marlaas_layer_norm(pool, x, seg, gain, bias, eps=EPS)
    check_forward(x, rows, gain, bias, False, y, mean, rstd)
    dx, dgain, dbias = torch.empty_like(x), torch.empty_like(gain), torch.empty_like(bias)
    B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, mean, rstd, dx=dx, dgain=dgain, dbias=dbias)
    check_backward(x, dy, rows, gain, mean, rstd, False, dx, dgain, dbias)


def test_host_tables_pitches_in_place_and_accumulation(pool):
    T, d, ld = 77, 136, 160
    off, slot, rows = batch(T, 6, 8)
    x, xf = rows_of(T, d, 7, ld)
    dy, dyf = rows_of(T, d, 8, ld)
    gain, bias = params(d, 9)
    host, seg = segments(off, slot, on_host=True), segments(off, slot)
    y0, mean, rstd = B.marlaas_layer_norm(pool, x, seg, gain, bias, eps=EPS)
    y1, m1, r1 = B.marlaas_layer_norm(pool, x, host, gain, bias, eps=EPS)
    assert torch.equal(y0, y1) and torch.equal(mean, m1) and torch.equal(rstd, r1)
    x0, dy0 = x.clone(), dy.clone()
    dgain, dbias = torch.full_like(gain, 2.0), torch.full_like(bias, 2.0)
    B.marlaas_layer_norm_backward(pool, x, dy, host, gain, mean, rstd, dx=dy, dgain=dgain, dbias=dbias, flags=B.MARLAAS_FLAG_ACCUMULATE)
    check_backward(x0, dy0, rows, gain, mean, rstd, False, dy, dgain, dbias, add=2.0)
    assert torch.all(dyf[:, d:] == 7) and torch.equal(x, x0)
    only = torch.empty_like(bias)
    B.marlaas_layer_norm_backward(pool, x, dy0, seg, gain, mean, rstd, dbias=only)
    check_backward(x0, dy0, rows, gain, mean, rstd, False, None, None, only)
    just = torch.empty_like(dy0)
    B.marlaas_layer_norm_backward(pool, x, dy0, seg, gain, mean, rstd, dx=just)
    assert torch.equal(just, dy)
    B.marlaas_layer_norm(pool, x, seg, gain, bias, eps=EPS, y=x)
    assert torch.equal(x, y0) and torch.all(xf[:, d:] == 7)


def test_bad_rows_stay_alone_and_constant_rows_are_their_bias(pool):
    T, d = 9, 128
    x, _ = rows_of(T, d, 10)
    x[2, 5], x[4, 0] = float("nan"), float("inf")
    x[6] = 3.0
    gain, bias = params(d, 11)
    y, mean, rstd = B.marlaas_layer_norm(pool, x, segments([0, 4, 9], [1, -1]), gain, bias, eps=EPS)
    assert torch.isnan(y[2]).all() and torch.isnan(y[4]).all()
    good = [0, 1, 3, 5, 6, 7, 8]
    assert torch.isfinite(y[good].float()).all()
    assert torch.equal(y[6], bias[CAP].bfloat16())


def test_no_tokens(pool):
    gain, bias = params(64, 12)
    x = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    seg = segments([0, 0], [1])
    y, mean, rstd = B.marlaas_layer_norm(pool, x, seg, gain, bias)
    assert y.shape == (0, 64)
    dg, db = torch.full_like(gain, 3.0), torch.full_like(gain, 3.0)
    B.marlaas_layer_norm_backward(pool, x, x, seg, gain, mean, rstd, dgain=dg, flags=B.MARLAAS_FLAG_ACCUMULATE)
    B.marlaas_layer_norm_backward(pool, x, x, seg, gain, mean, rstd, dbias=db)
    assert torch.all(dg == 3) and torch.all(db == 0)


def test_ill_formed_device_tables_are_reported(pool):
    x, _ = rows_of(40, 64, 13)
    gain, bias = params(64, 14)
    for off, slot, status in (([0, 30, 20, 40], [0, 1, 2], B.MARLAAS_ERR_BAD_SEGMENT_TABLE), ([0, 39], [0], B.MARLAAS_ERR_BAD_SEGMENT_TABLE),
                              ([0, 20, 40], [0, CAP], B.MARLAAS_ERR_DEVICE_BAD_INDEX)):
        seg = segments(off, slot)
        _, mean, rstd = B.marlaas_layer_norm(pool, x, seg, gain, bias)
        with pytest.raises(B.MarlaasError) as e:
            B.marlaas_check_status(pool)
        assert e.value.status == status
        B.marlaas_layer_norm_backward(pool, x, x, seg, gain, mean, rstd, dgain=torch.empty_like(gain))
        with pytest.raises(B.MarlaasError) as e:
            B.marlaas_check_status(pool)
        assert e.value.status == status


def test_streams_and_graphs(pool):
    T, d = 700, 512
    off, slot, rows = batch(T, 20, 15)
    x, _ = rows_of(T, d, 16)
    dy, _ = rows_of(T, d, 17)
    gain, bias = params(d, 18)
    seg = segments(off, slot)
    y, mean, rstd = B.marlaas_layer_norm(pool, x, seg, gain, bias)
    dx, dgain, dbias = torch.empty_like(x), torch.empty_like(gain), torch.empty_like(bias)
    B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, mean, rstd, dx=dx, dgain=dgain, dbias=dbias)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = [torch.zeros_like(v) for v in (dx, dgain, dbias)]
    ys = B.marlaas_layer_norm(pool, x, seg, gain, bias, stream=side)
    B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, mean, rstd, dx=out[0], dgain=out[1], dbias=out[2], stream=side)
    side.synchronize()
    assert torch.equal(ys[0], y) and all(torch.equal(a, b) for a, b in zip(out, (dx, dgain, dbias)))
    graphs, outs = [], []
    for _ in range(2):                  # two graphs, each with a workspace of its own
        o = [torch.zeros_like(v) for v in (y, mean, rstd, dx, dgain, dbias)]
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            B.marlaas_layer_norm(pool, x, seg, gain, bias, y=o[0], mean=o[1], rstd=o[2])
            B.marlaas_layer_norm_backward(pool, x, dy, seg, gain, o[1], o[2], dx=o[3], dgain=o[4], dbias=o[5])
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
        assert all(torch.equal(a, b) for a, b in zip(o, (y, mean, rstd, dx, dgain, dbias)))
