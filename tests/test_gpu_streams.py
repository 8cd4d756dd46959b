"""Calls that are given a stream while another one is current: memory that they allocate is not still in use there, and what
they return may be let go."""
import numpy as np
import pytest
import torch

from paper_2605_08527_b200 import binding as B

from test_gpu_policy import dev, segments

pytestmark = pytest.mark.gpu

T, V, K, N = 1 << 15, 8, 64, 64


@pytest.fixture(scope="module")
def setting():
    pool = B.AdapterPool(K, N, 8, 2)
    for t in range(2):
        B.marlaas_adapter_pool_register(pool, t, 0, 8, 8.0, torch.randn(K, 8, device="cuda").bfloat16(), torch.randn(8, N, device="cuda").bfloat16())
    r = np.random.RandomState(2)
    s = dict(pool=pool, seg=segments([0, T // 2, T], [0, 1]), groups=dev([0, 2], torch.int32), rewards=dev([1.0, 0.0], torch.float32),
             targets=dev(r.randint(0, V, T), torch.int32), z=torch.randn(T, V, device="cuda"), f=torch.rand(T, device="cuda") - 2,
             x=torch.randn(T, K, device="cuda").bfloat16(), W=torch.randn(K, N, device="cuda").bfloat16(),
             state=torch.randint(0, 100, (512 * 528,), device="cuda").to(torch.uint8))
    torch.cuda.synchronize()
    return s


CALLS = {
    "advantages": (lambda s, **kw: B.marlaas_group_advantages(s["pool"], s["seg"], s["rewards"], s["groups"], s["targets"], **kw), 4 * T),
    "log-probabilities": (lambda s, **kw: B.marlaas_token_logprobs(s["pool"], s["z"], s["targets"], with_entropy=True, **kw), 4 * T),
    "loss": (lambda s, **kw: B.marlaas_policy_loss(s["pool"], s["z"], s["targets"], s["seg"], s["f"], s["f"], s["f"], **kw), 32 * T),
    "moments": (lambda s, **kw: B.marlaas_adamw_compact_state_export(s["pool"], s["state"], **kw), 4 * 512 * 256),
    "forward": (lambda s, **kw: B.marlaas_lora_forward(s["pool"], s["x"], s["W"], s["seg"], **kw), 2 * T * N),
    "forward of several": (lambda s, **kw: B.marlaas_lora_forward_multi([dict(pool=s["pool"], x=s["x"], W=s["W"], seg=s["seg"])], **kw), 2 * T * N),
    "index": (lambda s, **kw: B.marlaas_lora_build_index(s["pool"], T, s["seg"], **kw), 4 * T),
    "export": (lambda s, **kw: B.marlaas_adapter_pool_export(s["pool"], 1, 8, **kw), 2 * K * 8),
}


def flat(out):
    return [out] if isinstance(out, torch.Tensor) else [t for o in out for t in flat(o)]


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("by_handle", [False, True])
def test_allocations_on_a_given_stream(setting, name, by_handle):
    call, nbytes = CALLS[name]
    want = [t.clone() for t in flat(call(setting))]
    B.marlaas_check_status(setting["pool"])
    side = torch.cuda.Stream()
    stream = side.cuda_stream if by_handle else side
    # blocks of the outputs' and the workspace's size that are free to the allocator, but read by work that has yet to run here
    held = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in (nbytes, nbytes, nbytes, 32 * T, 40 * T)]
    copies = [torch.zeros_like(h) for h in held]
    torch.cuda.synchronize()
    torch.cuda._sleep(40_000_000)
    for c, h in zip(copies, held):
        c.copy_(h)
    del held, h
    got = flat(call(setting, stream=stream))
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.all(c == 7) for c in copies)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    # let go here while work on it is under way here, then the same call again: its memory is not taken for the new outputs
    torch.cuda._sleep(40_000_000)
    copies = [t.clone() for t in got]
    del got
    again = [t.fill_(1) for t in flat(call(setting, stream=stream)) if t.dtype != torch.int32]
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(copies, want))
    del again
