"""The head's outputs may not lie over its inputs, but for dx over the whole of x."""
import pytest
import torch

import test_gpu_training_refusals as refusals
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu

T, D, V = refusals.T, refusals.D, refusals.V


@pytest.fixture(scope="module")
def env():
    return refusals.Env()


def spans(env):
    """First and last byte but three of each input."""
    a = env.args["head_cross_entropy"]
    off, slot = env.seg.seg_offsets, env.seg.seg_slot
    return {"x": (a["x"], 2 * T * D), "W": (a["W"], 2 * D * V), "targets": (a["targets"], 4 * T), "weight": (env.rates.data_ptr(), 4 * T),
            "the segment table": (off.data_ptr(), 4 * off.numel()), "the table's slots": (slot.data_ptr(), 4 * slot.numel())}


@pytest.mark.parametrize("out", ["dx", "logp", "stats"])
@pytest.mark.parametrize("inp", ["x", "W", "targets", "weight", "the segment table", "the table's slots"])
def test_an_output_over_an_input(env, out, inp):
    env.rates = torch.ones(T, device="cuda") if env.rates.numel() < T else env.rates
    at, n = spans(env)[inp]
    size = {"dx": 2 * ((T - 1) * V + D), "logp": 4 * T, "stats": 4 * 4 * (refusals.CAP + 1)}[out]
    step = 16 if out == "dx" else 4
    first, last = -(-(at - size + 1) // step) * step, (at + n - 1) // step * step        # overlaps of a few bytes at either end
    for p in (first, last, -(-at // step) * step):
        if out == "dx" and inp == "x" and p == at:
            continue        # (another leading dimension: refused as well, below)
        env.refused("head_cross_entropy", B.MARLAAS_ERR_INVALID_ARG, weight=env.rates.data_ptr(), **{out: p})
        assert "overlaps" in B.marlaas_last_error()


def test_dx_over_x_with_another_leading_dimension(env):
    env.refused("head_cross_entropy", B.MARLAAS_ERR_INVALID_ARG, dx=env.args["head_cross_entropy"]["x"])


def test_beside_one_another(env):
    """Outputs that end where inputs begin, and the other way round, are fine."""
    buf = torch.zeros(64 * T, device="cuda")
    p = buf.data_ptr()
    x = torch.zeros((T, D), dtype=torch.bfloat16, device="cuda")
    a = dict(weight=p + 4 * T, logp=p, stats=p + 8 * T, targets=p + 8 * T + 16 * (refusals.CAP + 1), dx=x.data_ptr(), lddx=D, x=x.data_ptr())
    assert env.call("head_cross_entropy", **a) == B.MARLAAS_OK, B.marlaas_last_error()
    torch.cuda.synchronize()
