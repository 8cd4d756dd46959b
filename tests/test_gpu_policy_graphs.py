"""Captured calls without a workspace of the caller's: replays neither write into memory that has been given to something else
nor share scratch with another graph."""
import numpy as np
import pytest
import torch

from paper_2605_08527_b200 import binding as B

from test_gpu_policy import dev, segments

pytestmark = pytest.mark.gpu


class Batch:
    def __init__(self, pool, S, length, V, seed):
        r = np.random.RandomState(seed)
        self.pool, self.T, self.V = pool, S * length, V
        self.seg = segments(np.arange(0, self.T + 1, length).tolist(), r.randint(-1, pool.capacity, S).tolist())
        self.groups = dev(np.arange(0, S + 1, 4), torch.int32)
        self.rewards, self.targets = dev(r.rand(S), torch.float32), dev(r.randint(-1, V, self.T), torch.int32)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.z = torch.randn(self.T, V, generator=g, device="cuda").bfloat16()
        self.old = torch.full((self.T,), -5.0, device="cuda")
        self.out = None

    def __call__(self):
        seq_adv, adv, weight = B.marlaas_group_advantages(self.pool, self.seg, self.rewards, self.groups, self.targets)
        grad = torch.empty_like(self.z)
        stats = B.marlaas_policy_loss(self.pool, self.z, self.targets, self.seg, self.old, adv, weight, dlogits=grad)
        self.out = (seq_adv, adv, weight, grad, stats)
        return self.out


def capture(call, stream=None):
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=stream):
        call()
    return g


@pytest.mark.parametrize("S", [40, 2600])       # one kernel for the advantages; three with totals in the workspace
def test_a_replay_after_a_larger_batch(S):
    pool = B.AdapterPool(64, 64, 8, 5)
    side = torch.cuda.Stream()
    small, large = Batch(pool, S, 5, 256, 1), Batch(pool, 8 * S, 20, 256, 2)
    with torch.cuda.stream(side):
        want = [t.clone() for t in small()]
    g = capture(small, side)
    with torch.cuda.stream(side):
        large()
        # memory that a replaced workspace would have left free
        sizes = [B.marlaas_policy_workspace_bytes(pool, small.T, S, G) for G in (0, S // 4)]
        full = [torch.full((max(n, 256),), 77, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
    torch.cuda.synchronize()
    for t in small.out:
        t.zero_()
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(small.out, want))
    assert all(torch.all(t == 77) for t in full)
    B.marlaas_check_status(pool)


def test_two_graphs_at_the_same_time():
    pool = B.AdapterPool(64, 64, 8, 5)
    batches = [Batch(pool, 2400, 5, 512, 3), Batch(pool, 2400, 5, 512, 4)]
    want = [[t.clone() for t in b()] for b in batches]
    graphs = [capture(b) for b in batches]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for b in batches:
            for t in b.out:
                t.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                for _ in range(4):
                    g.replay()
        torch.cuda.synchronize()
        for b, w in zip(batches, want):
            assert all(torch.equal(x, y) for x, y in zip(b.out, w))
    B.marlaas_check_status(pool)


def test_a_capture_on_a_stream_of_its_own():
    # the stream is an argument of the calls, another one is current: it takes part in the capture by events
    pool = B.AdapterPool(64, 64, 8, 5)
    b = Batch(pool, 2400, 5, 256, 5)
    want = [t.clone() for t in b()]
    other = torch.cuda.Stream()
    out = []

    def call():
        adv, weight = torch.empty(b.T, device="cuda"), torch.empty(b.T, device="cuda")
        other.wait_stream(torch.cuda.current_stream())
        out.append(B.marlaas_group_advantages(pool, b.seg, b.rewards, b.groups, b.targets, adv=adv, weight=weight, stream=other))
        torch.cuda.current_stream().wait_stream(other)

    g = capture(call)
    b()         # the cached workspace of the current stream is not the graph's
    for t in out[0]:
        t.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(out[0], want))


def test_a_replay_of_the_layer_after_a_larger_batch():
    pool = B.AdapterPool(256, 512, 16, 2)
    for t in range(2):
        B.marlaas_adapter_pool_register(pool, t, 0, 16, 16.0, torch.randn(256, 16, device="cuda").bfloat16() / 16,
                                        torch.randn(16, 512, device="cuda").bfloat16())
    W = torch.randn(256, 512, device="cuda").bfloat16() / 16
    side = torch.cuda.Stream()

    def forward(T, y):
        B.marlaas_lora_forward(pool, xs[T], W, segs[T], y=y)

    xs = {T: torch.randn(T, 256, device="cuda").bfloat16() for T in (1500, 9000)}
    segs = {T: segments([0, T // 3, T], [0, 1]) for T in xs}
    y = {T: torch.empty((T, 512), dtype=torch.bfloat16, device="cuda") for T in xs}
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        forward(1500, y[1500])
    torch.cuda.synchronize()
    want = y[1500].clone()
    n = B.marlaas_lora_workspace_bytes(pool, 1500)
    g = capture(lambda: forward(1500, y[1500]), side)
    with torch.cuda.stream(side):
        forward(9000, y[9000])
        full = [torch.full((n,), 77, dtype=torch.uint8, device="cuda") for _ in range(4)]
    y[1500].zero_()
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y[1500], want) and all(torch.all(t == 77) for t in full)
    B.marlaas_check_status(pool)
