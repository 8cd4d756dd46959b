"""The adapters' gradients of the layer with dropout hold what their own tenant's tokens hold, and nothing of the others': tenants
that share blocks of 64 tokens, in batches that each form of the reductions takes (`fits`: the masked blocks certainly fit the
workspace, cdiv(T, 64) + segments <= 3 cdiv(T, 64) + 2 capacity; otherwise the device decides between the tensor cores and the
sums over ordered tokens)."""
import math

import pytest
import torch

import test_gpu_dropout as drop
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu

RANKS, RATES = [8, 16, 8, 24], [0.5, 0.1, 0.0, 0.3]


def mixed(T, S, kind, seed):
    """A batch of S segments.  "fits": of any slots; "device decides": S - 1 empty or one-token segments of one tenant, so that the
    bound by the segments is missed though few tenants share a block; "too many": tokens of all tenants in turn and a small pool."""
    c = drop.Case(T, 256, 128, RANKS, S, seed, rates=RATES)
    if kind == "device decides":
        half = T // 2
        c.off = [0, half] + [half + 1 + i for i in range(S - 2)] + [T]
        c.slot = [0] + [1] * (S - 2) + [2]
        c.tok = [s for s, a, b in zip(c.slot, c.off, c.off[1:]) for _ in range(b - a)]
        c.seg = drop.segments(c.off, c.slot)
    elif kind == "too many":
        c.off, c.slot = list(range(T + 1)), [i % 4 for i in range(T)]
        c.tok = list(c.slot)
        c.seg = drop.segments(c.off, c.slot)
    nblk = -(-T // 64)
    assert (nblk + len(c.slot) <= 3 * nblk + 2 * c.cap) == (kind == "fits")
    tok = torch.tensor([int(t) for t in c.tok])
    present = sum(len([t for t in tok[i:i + 64].unique() if t >= 0]) for i in range(0, T, 64))
    assert (present > 3 * nblk + 2 * c.cap) == (kind == "too many")
    return c, tok.cuda()


FORMS = [(200, 12, "fits"), (600, 25, "fits"), (1000, 30, "fits"), (1000, 60, "device decides"), (2000, 2000, "too many")]


@pytest.mark.parametrize("saved", [True, False])
@pytest.mark.parametrize("T,S,kind", FORMS)
def test_what_a_row_of_dy_holds_reaches_no_other_tenant(T, S, kind, saved):
    c, tok = mixed(T, S, kind, 41)
    _, h = c.forward()
    h = h if saved else None
    dx, dA, dB = c.backward(h)
    for bad, value in ((1, math.inf), (2, math.nan), (-1, math.nan)):
        dy = c.dy
        rows = tok == bad
        assert rows.any() or bad == -1
        c.dy = torch.where(rows[:, None], torch.full_like(dy, value), dy)
        dx1, dA1, dB1 = c.backward(h)
        c.dy = dy
        assert torch.equal(dx1[~rows], dx[~rows])
        for t in range(len(RANKS)):
            if t != bad:
                assert torch.equal(dA1[t], dA[t]) and torch.equal(dB1[t], dB[t]), (bad, t)
    B.marlaas_check_status(c.pool)


@pytest.mark.parametrize("T,S,kind", FORMS)
def test_what_a_row_of_x_holds_reaches_no_other_tenant(T, S, kind):
    c, tok = mixed(T, S, kind, 42)
    y, h = c.forward()
    dx, dA, dB = c.backward(None)
    for bad in (0, 1, 2, -1):
        x = c.x
        rows = tok == bad
        c.x = torch.where(rows[:, None], torch.full_like(x, math.nan), x)
        y1, h1 = c.forward()
        dx1, dA1, dB1 = c.backward(None)
        c.x = x
        assert torch.equal(y1[~rows], y[~rows]) and torch.equal(h1[:, ~rows], h[:, ~rows]) and torch.equal(dx1, dx)
        for t in range(len(RANKS)):
            if t != bad:
                assert torch.equal(dA1[t], dA[t]) and torch.equal(dB1[t], dB[t]), (bad, t)


@pytest.mark.parametrize("T,S,kind", FORMS)
def test_what_a_row_drops_does_not_matter(T, S, kind):
    c, tok = mixed(T, S, kind, 43)
    keep = c.keep()
    _, h = c.forward()
    dx, dA, dB = c.backward(None)
    c.x = torch.where(keep, c.x, torch.full_like(c.x, math.nan))
    assert torch.isnan(c.x).any()
    _, h1 = c.forward()
    dx1, dA1, dB1 = c.backward(None)
    assert torch.equal(h1, h) and torch.equal(dx1, dx)
    assert all(torch.equal(a, b) for a, b in zip(dA1 + dB1, dA + dB))
