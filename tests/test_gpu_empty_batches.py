"""Batches without tokens, with each set of outputs: nothing to do is not an error."""
import pytest
import torch

import test_gpu_dropout as drop
import test_gpu_head as head
import test_gpu_layer_norm as norm
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu


def test_head():
    pool = B.AdapterPool(64, 64, 8, head.CAP)
    x, W, tgt, w, _, _ = head.inputs(4, 64, 100, 1)
    for dx in (None, x[:0]):
        logp, stats = B.marlaas_head_cross_entropy(pool, x[:0], W, tgt[:0], weight=w[:0], dx=dx)
        assert logp.shape == (0,) and stats is None
        for seg in (head.segments([0], []), head.segments([0, 0], [1])):
            logp, stats = B.marlaas_head_cross_entropy(pool, x[:0], W, tgt[:0], seg, dx=dx)
            assert logp.shape == (0,) and not stats.any()


def test_norms():
    pool = B.AdapterPool(64, 64, 8, norm.CAP)
    x = torch.zeros((0, 64), dtype=torch.bfloat16, device="cuda")
    gain, bias = norm.params(64, 1)
    for seg in (norm.segments([0], []), norm.segments([0, 0], [1])):
        y, mean, rstd = B.marlaas_layer_norm(pool, x, seg, gain, bias)
        assert y.shape == x.shape and mean.shape == rstd.shape == (0,)
        B.marlaas_layer_norm_backward(pool, x, x, seg, gain, mean, rstd, dx=torch.empty_like(x))
        dgain = torch.ones_like(gain)
        B.marlaas_layer_norm_backward(pool, x, x, seg, gain, mean, rstd, dx=torch.empty_like(x), dgain=dgain, flags=B.MARLAAS_FLAG_ACCUMULATE)
        assert torch.all(dgain == 1)
        B.marlaas_layer_norm_backward(pool, x, x, seg, gain, mean, rstd, dgain=dgain)
        assert not dgain.any()


def test_dropout():
    c = drop.Case(0, 64, 128, [8, 16], 1)
    y, h = c.forward()
    assert y.shape == (0, 128)
    dx, dA, dB = c.backward(h)
    assert dx.shape == (0, 64) and not any(g.any() for g in dA + dB)
    dx, dA, dB = c.backward(h, flags=B.MARLAAS_FLAG_ACCUMULATE)
    assert all(torch.all(g == 5) for g in dA + dB)
