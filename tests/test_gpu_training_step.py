"""The calls around a training step's layers in a row, as they are used: an adapted projection with dropout, a norm with its
tenants' parameters, the vocabulary head's loss, and all the way back, against 64-bit automatic differentiation of the same step.

Tolerance: eight tensors on the way are rounded to bf16 (the projection's and the norm's outputs and their gradients, the
products' operands s' h, s' g and the probabilities twice), each by at most 2^-8 of its size; what a layer passes on grows by
no more than half: in the 2-norm the step's gradients are within 8 x 1.5 x 2^-8 = 4.7 %.
"""
import numpy as np
import pytest
import torch

from oracle import training as ot
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu

CAP, EPS = 3, 1e-5


class Step:
    def __init__(self, T=600, K=256, d=512, V=1000, ranks=(8, 16, 5), seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rn = lambda *s: torch.randn(s, generator=g, device="cuda")       # noqa: E731
        r = np.random.RandomState(seed)
        self.T, self.K, self.d, self.V, self.ranks = T, K, d, V, ranks
        self.pool = B.AdapterPool(K, d, max(ranks), CAP)
        self.x, self.W = rn(T, K).bfloat16(), (rn(K, d) / K ** 0.5).bfloat16()
        self.A = [(rn(K, q) / K ** 0.5).bfloat16() for q in ranks]
        self.Bm = [(0.3 * rn(q, d)).bfloat16() for q in ranks]
        for t, q in enumerate(ranks):
            B.marlaas_adapter_pool_register(self.pool, t, 0, q, 8.0, self.A[t], self.Bm[t])
        self.gain, self.bias = 1 + 0.2 * rn(CAP + 1, d), 0.2 * rn(CAP + 1, d)
        self.head = (2 * rn(d, V) / d ** 0.5).bfloat16()
        off = np.unique(np.concatenate([[0, T], r.randint(0, T, 6)]))
        slot = r.randint(-1, CAP, len(off) - 1)
        self.tok = np.repeat(slot, np.diff(off))
        self.seg = B.Segments(*(torch.tensor(a, dtype=torch.int32, device="cuda") for a in (off, slot)))
        self.targets = torch.randint(0, V, (T,), generator=g, device="cuda").int()
        self.targets[torch.rand(T, generator=g, device="cuda") < 0.3] = -1
        self.weight = rn(T) / T
        self.rates = [0.1, 0.3, 0.0]
        self.rates_dev = torch.tensor(self.rates, device="cuda")

    def run(self, flags=0, dA=None, dB=None, dgain=None, dbias=None):
        T, p = self.T, self.pool
        h = torch.empty((T, p.rank_stride), device="cuda")
        y = B.marlaas_lora_forward_dropout(p, self.x, self.W, self.seg, self.rates_dev, 11, 3, h_save=h)
        n, mean, rstd = B.marlaas_layer_norm(p, y, self.seg, self.gain, self.bias, eps=EPS)
        dn = torch.empty_like(n)
        logp, stats = B.marlaas_head_cross_entropy(p, n, self.head, self.targets, self.seg, weight=self.weight, dx=dn)
        dgain = torch.empty_like(self.gain) if dgain is None else dgain
        dbias = torch.empty_like(self.bias) if dbias is None else dbias
        B.marlaas_layer_norm_backward(p, y, dn, self.seg, self.gain, mean, rstd, dx=dn, dgain=dgain, dbias=dbias, flags=flags)
        dx = torch.empty_like(self.x)
        dA = [torch.empty(a.shape, device="cuda") for a in self.A] if dA is None else dA
        dB = [torch.empty(b.shape, device="cuda") for b in self.Bm] if dB is None else dB
        B.marlaas_lora_backward_dropout(p, self.x, self.W, dn, self.seg, self.rates_dev, 11, 3, dx=dx, dA=dA, dB=dB, h_saved=h, flags=flags)
        return dict(logp=logp, stats=stats, dx=dx, dgain=dgain, dbias=dbias, dA=dA, dB=dB)

    def reference(self):
        leaf = lambda t: t.double().requires_grad_()      # noqa: E731
        x, A, Bm, gain, bias = leaf(self.x), [leaf(a) for a in self.A], [leaf(b) for b in self.Bm], leaf(self.gain), leaf(self.bias)
        keep = torch.from_numpy(ot.dropout_keep(self.tok, self.K, self.rates, 11, 3)).cuda()
        y = x @ self.W.double()
        for t, q in enumerate(self.ranks):
            mine = torch.from_numpy(self.tok == t).cuda()[:, None]
            y = y + torch.where(mine, ot.dropout_factor(8.0 / q, self.rates[t]) * ((x * keep) @ A[t]) @ Bm[t], 0.0)
        rows = torch.from_numpy(np.where(self.tok < 0, CAP, self.tok)).cuda()
        c = y - y.mean(1, keepdim=True)
        n = c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) * gain[rows] + bias[rows]
        on = self.targets >= 0
        ls = torch.log_softmax(n @ self.head.double(), 1)
        logp = torch.where(on, ls.gather(1, self.targets.clamp(min=0).long()[:, None])[:, 0], 0.0)
        loss = -(self.weight.double() * logp).sum()
        loss.backward()
        return dict(logp=logp.detach(), loss=loss.detach(), dx=x.grad, dgain=gain.grad, dbias=bias.grad, dA=[a.grad for a in A], dB=[b.grad for b in Bm])


def near(got, ref, bound=8 * 1.5 * 2.0 ** -8):
    err, size = float((got.double() - ref).norm()), float(ref.norm())       # (both 0 for a tenant without tokens)
    assert err <= bound * size, (err, size)


@pytest.mark.parametrize("T", [64, 600, 1500])
def test_a_whole_step(T):
    s = Step(T)
    out, ref = s.run(), s.reference()
    B.marlaas_check_status(s.pool)
    near(out["logp"], ref["logp"])
    assert abs(float(out["stats"][:, 0].double().sum() - ref["loss"])) <= 0.047 * float((s.weight.double() * ref["logp"]).abs().sum())
    near(out["dx"], ref["dx"])
    near(out["dgain"], ref["dgain"])
    near(out["dbias"], ref["dbias"])
    for k in ("dA", "dB"):
        for a, b in zip(out[k], ref[k]):
            near(a, b)


def test_two_micro_batches_accumulate():
    s = Step()
    once = s.run()
    acc = {k: ([v.clone() for v in once[k]] if isinstance(once[k], list) else once[k].clone()) for k in ("dA", "dB", "dgain", "dbias")}
    s.run(flags=B.MARLAAS_FLAG_ACCUMULATE, **acc)
    for k in ("dgain", "dbias"):
        assert torch.allclose(acc[k], 2 * once[k], rtol=1e-6, atol=0)
    for k in ("dA", "dB"):
        assert all(torch.allclose(a, 2 * b, rtol=1e-6, atol=0) for a, b in zip(acc[k], once[k]))


def test_a_captured_step_while_eager_ones_run():
    """A step captured into a graph and replayed beside eager steps of the same pool on another stream: the same bits."""
    s = Step()
    ref = s.run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cap = s.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    eager = []
    for _ in range(3):
        g.replay()
        with torch.cuda.stream(side):
            eager.append(s.run())
    torch.cuda.synchronize()
    for out in [cap] + eager:
        for k in ("logp", "stats", "dx", "dgain", "dbias"):
            assert torch.equal(out[k], ref[k]), k
        for k in ("dA", "dB"):
            assert all(torch.equal(a, b) for a, b in zip(out[k], ref[k])), k
    # new inputs, the same graph
    s.x.copy_(torch.randn(s.x.shape, device="cuda").bfloat16())
    g.replay()
    again = s.run()
    torch.cuda.synchronize()
    assert torch.equal(again["dx"], cap["dx"]) and torch.equal(again["logp"], cap["logp"])
