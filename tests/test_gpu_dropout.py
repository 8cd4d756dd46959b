"""The layer with dropout in its adapters, on the GPU against its definition in 64 bits with the same masks.

Tolerances, from the arithmetic.  Products of bf16 numbers are summed in fp32 in steps of 16: 2^-23 (n / 16 + 2) of the sum of
magnitudes for n products.  s' h and s' g enter the second product rounded to bf16 (2^-8 relative each), so y and dx are off
by that part of the low-rank term's magnitudes, and by half a step of bf16 (2^-8) once or, for dx, twice.  The adapters'
gradients take h and g split in two bf16 numbers: 2^-16 of the magnitudes, and the sums' part.
"""
import numpy as np
import pytest
import torch

from oracle import training as ot
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu

SEED, OFFSET = 0x123456789ABCDEF0, (7 << 32) + 5


def segments(off, slot, on_host=False):
    t = [torch.tensor(x, dtype=torch.int32) for x in (off, slot)]
    return B.Segments(*(t if on_host else [x.cuda() for x in t]))


def masks(tok, width, rates, seed, offset):
    """oracle.training.dropout_keep for whole arrays."""
    T, n = len(tok), -(-width // 8)
    m, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [np.tile(np.arange(n, dtype=np.uint64), (T, 1)), np.repeat(np.arange(T, dtype=np.uint64)[:, None], n, 1),
         np.full((T, n), offset & 0xFFFFFFFF, dtype=np.uint64), np.full((T, n), offset >> 32, dtype=np.uint64)]
    for i in range(7):
        k0, k1 = np.uint64(((seed & 0xFFFFFFFF) + i * 0x9E3779B9) & 0xFFFFFFFF), np.uint64(((seed >> 32) + i * 0xBB67AE85) & 0xFFFFFFFF)
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> sh) ^ c[1] ^ k0, b & m, (a >> sh) ^ c[3] ^ k1, a & m]
    bits = np.stack([w for v in c for w in (v & np.uint64(0xFFFF), v >> np.uint64(16))], 2).reshape(T, -1)[:, :width]
    limit = np.array([0 if t < 0 else ot.threshold(rates[t]) for t in tok], dtype=np.uint64)
    return bits >= limit[:, None]


class Case:
    def __init__(self, T, K, N, ranks, S, seed=0, parts=None, rates=None, alpha=12.0, cap=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rn = lambda *s: torch.randn(s, generator=g, device="cuda")       # noqa: E731
        r = np.random.RandomState(seed)
        self.T, self.K, self.N, self.ranks, self.n = T, K, N, ranks, len(ranks)
        self.parts = parts or [N]
        self.cap = cap or self.n
        self.pool = B.AdapterPool(K, N, max(ranks + [1]), self.cap, parts=parts)
        self.x, self.dy = rn(T, K).bfloat16(), rn(T, N).bfloat16()
        self.W = (rn(K, N) / K ** 0.5).bfloat16()
        self.A = [[(rn(K, q) / K ** 0.5).bfloat16() for _ in self.parts] if q else None for q in ranks]
        self.Bm = [[(0.3 * rn(q, w)).bfloat16() for w in self.parts] if q else None for q in ranks]
        for t, q in enumerate(ranks):
            a, b = (self.A[t], self.Bm[t]) if parts or not q else (self.A[t][0], self.Bm[t][0])
            B.marlaas_adapter_pool_register(self.pool, 100 + t, 0, q, alpha if q else 1.0, a if q else None, b if q else None)
        self.scale = [alpha / q if q else 0.0 for q in ranks]
        self.off = np.sort(np.concatenate([[0, T], r.randint(0, T + 1, S - 1)])).tolist()
        self.slot = r.randint(-1, self.n, S).tolist()
        self.tok = np.repeat(self.slot, np.diff(self.off))
        self.rates = list(rates) if rates else [[0.1, 0.5, 0.0, 0.05][t % 4] for t in range(self.n)]
        self.rates_dev = torch.tensor(self.rates + [0.0] * (self.cap - self.n), device="cuda")
        self.seg = segments(self.off, self.slot)

    def keep(self, seed=SEED, offset=OFFSET):
        return torch.from_numpy(masks(self.tok, self.K, self.rates, seed, offset)).cuda()

    def grads(self, fill=5.0):
        P = len(self.parts)
        return ([torch.full((P * self.K * q,), fill, device="cuda") if q else None for q in self.ranks],
                [torch.full((q * self.N,), fill, device="cuda") if q else None for q in self.ranks])

    def reference(self, keep, h_given=None):
        """y, dx, dA, dB with their tolerances; h."""
        K, N, T = self.K, self.N, self.T
        x, W, dy = self.x.double(), self.W.double(), self.dy.double()
        y, dx = x @ W, dy @ W.T
        ytol = 2.0 ** -23 * (K / 16 + 2) * (x.abs() @ W.abs())
        dtol = 2.0 ** -23 * (N / 16 + 2) * (dy.abs() @ W.abs().T)
        P, RP = len(self.parts), self.pool.rank_stride
        h, htol = (torch.zeros((P, T, RP), dtype=torch.float64, device="cuda") for _ in range(2))
        dA, dB, atol, btol = [], [], [], []
        cut = np.concatenate([[0], np.cumsum(self.parts)])
        for t, q in enumerate(self.ranks):
            if not q:
                dA.append(None), dB.append(None), atol.append(None), btol.append(None)
                continue
            f = ot.dropout_factor(self.scale[t], self.rates[t])
            i = torch.from_numpy(np.nonzero(self.tok == t)[0]).cuda()
            xd = torch.where(keep[i], x[i], 0.0)
            ga, gb, ta, tb = [], [], [], []
            for p in range(P):
                c = slice(int(cut[p]), int(cut[p + 1]))
                A, Bm = self.A[t][p].double(), self.Bm[t][p].double()
                hp = xd @ A
                he = 2.0 ** -23 * (K / 16 + 2) * (xd.abs() @ A.abs())
                h[p, i, :q], htol[p, i, :q] = hp, he
                y[i, c] += f * hp @ Bm
                ytol[i, c] += f * (2.0 ** -8 * 1.02 * hp.abs() + he) @ Bm.abs() + 2.0 ** -20 * f * hp.abs() @ Bm.abs()
                g = dy[i, c] @ Bm.T
                ge = 2.0 ** -23 * ((cut[p + 1] - cut[p]) / 16 + 2) * (dy[i, c].abs() @ Bm.abs().T)
                low = f * g @ A.T
                dx[i] += torch.where(keep[i], low, 0.0)
                dtol[i] += f * (2.0 ** -8 * 1.02 * g.abs() + ge) @ A.abs().T + 2.0 ** -20 * f * g.abs() @ A.abs().T
                n = 2.0 ** -16 + 2.0 ** -23 * (len(i) / 16 + 8)
                ga.append((f * xd.T @ g).reshape(-1)), ta.append((f * (n * xd.abs().T @ g.abs() + xd.abs().T @ ge)).reshape(-1))
                hs = hp if h_given is None else h_given[p, i, :q].double()
                gb.append((f * hs.T @ dy[i, c]).reshape(-1)), tb.append((f * (n * hs.abs().T @ dy[i, c].abs() + he.T @ dy[i, c].abs())).reshape(-1))
            dA.append(torch.cat(ga)), dB.append(torch.cat(gb)), atol.append(torch.cat(ta)), btol.append(torch.cat(tb))
        ytol += 2.0 ** -8 * 1.01 * (y.abs() + ytol)
        dtol += 2.0 ** -7 * 1.01 * (dx.abs() + dtol) + 2.0 ** -8 * 1.01 * (dx - dy @ W.T).abs()
        return dict(y=y, dx=dx, dA=dA, dB=dB, h=h), dict(y=ytol, dx=dtol, dA=atol, dB=btol, h=htol + 1e-30)

    def forward(self, **kw):
        h = torch.full((len(self.parts), self.T, self.pool.rank_stride), 3.0, device="cuda")
        y = B.marlaas_lora_forward_dropout(self.pool, self.x, self.W, kw.pop("seg", self.seg), self.rates_dev, SEED, OFFSET, h_save=h, **kw)
        return y, h

    def backward(self, h=None, fill=5.0, **kw):
        dA, dB = self.grads(fill)
        dx = torch.full_like(self.x, 9.0)
        full = lambda g: g + [None] * (self.cap - self.n)        # noqa: E731
        B.marlaas_lora_backward_dropout(self.pool, self.x, self.W, self.dy, kw.pop("seg", self.seg), self.rates_dev, SEED, OFFSET, dx=dx, dA=full(dA),
                                        dB=full(dB), h_saved=h, **kw)
        return dx, dA, dB


def check(got, ref, tol, what):
    err = (got.double() - ref).abs()
    assert torch.isfinite(got.double()).all(), what
    bad = err > tol
    assert not bad.any(), (what, int(bad.sum()), float((err - tol).max()), float(err.max()))


def check_case(c, keep, add=0.0):
    ref, tol = c.reference(keep)
    y, h = c.forward()
    check(y, ref["y"], tol["y"], "y")
    check(h, ref["h"], tol["h"], "h")
    for saved in (h, None):
        dx, dA, dB = c.backward(saved)
        check(dx, ref["dx"], tol["dx"], "dx")
        for t, q in enumerate(c.ranks):
            if q:
                check(dA[t], ref["dA"][t], tol["dA"][t] + 1e-30, "dA")
                check(dB[t], ref["dB"][t], tol["dB"][t] + 1e-30, "dB")
    B.marlaas_check_status(c.pool)


SIZES = [(1, 8, 8, [4], 1), (5, 64, 72, [8, 1], 2), (100, 512, 512, [8], 1), (130, 136, 264, [5, 16, 0], 7), (300, 1000, 520, [16, 32, 64, 8], 12),
         (513, 128, 128, [16, 16], 5), (1000, 200, 648, [8, 16, 32, 64, 128], 9), (1030, 256, 256, [16] * 9, 40), (2100, 512, 384, [16, 8, 64], 6),
         (1024, 72, 1024, [24], 2)]


@pytest.mark.parametrize("T,K,N,ranks,S", SIZES)
def test_both_passes(T, K, N, ranks, S):
    c = Case(T, K, N, ranks, S, T + K)
    check_case(c, c.keep())


def test_masks_are_the_definition():
    tok, rates = [0, 1, -1, 0, 2], [0.3, 1.0, 0.0]
    a = ot.dropout_keep(tok, 40, rates, SEED, OFFSET)
    assert np.array_equal(a, masks(np.array(tok), 40, rates, SEED, OFFSET))
    # through the layer: x of ones, A = e_j, so that h is the mask's first columns, for the largest counters too
    K, r = 64, 8
    for seed, offset in ((SEED, OFFSET), (0, 0), (2 ** 64 - 1, 2 ** 64 - 1)):
        pool = B.AdapterPool(K, 64, r, 1)
        for j0 in range(0, K, r):
            A = torch.zeros((K, r), dtype=torch.bfloat16, device="cuda")
            A[j0:j0 + r] = torch.eye(r, dtype=torch.bfloat16)
            B.marlaas_adapter_pool_register(pool, 1, 0, r, 8.0, A, torch.zeros((r, 64), dtype=torch.bfloat16, device="cuda"))
            T = 70
            h = torch.empty((T, pool.rank_stride), device="cuda")
            B.marlaas_lora_forward_dropout(pool, torch.ones((T, K), dtype=torch.bfloat16, device="cuda"), torch.zeros((K, 64), dtype=torch.bfloat16, device="cuda"),
                                           segments([0, T], [0]), torch.tensor([0.37], device="cuda"), seed, offset, h_save=h)
            want = masks(np.zeros(T, dtype=int), K, [0.37], seed, offset)
            assert np.array_equal(h[:, :r].cpu().numpy() == 1.0, want[:, j0:j0 + r])


def test_several_projections():
    for T in (90, 1100):
        c = Case(T, 256, 256 + 512 + 256, [8, 16, 64], 6, 21, parts=[256, 512, 256])
        check_case(c, c.keep())


def test_rates_at_their_ends():
    nan, inf = float("nan"), float("inf")
    c = Case(600, 128, 256, [8] * 8, 12, 22, rates=[0.0, 1.0, nan, -0.5, 2.0, 1e-6, 0.99999, inf])
    check_case(c, c.keep())
    y, h = c.forward()
    gone = torch.from_numpy((c.tok == 1) | (c.tok == 4) | (c.tok == 7)).cuda()
    assert not h[0][gone].any()
    dx, dA, dB = c.backward(h)
    assert not any(g[t].any() for g in (dA, dB) for t in (1, 4, 7))


def test_rate_zero_is_the_plain_layer():
    c = Case(700, 256, 512, [16, 8], 5, 23, rates=[0.0, 0.0])
    y, h = c.forward()
    h2 = torch.empty_like(h)
    y2 = B.marlaas_lora_forward(c.pool, c.x, c.W, c.seg, h_save=h2)
    assert torch.all((y.float() - y2.float()).abs() <= 2.0 ** -7 * y2.float().abs() + 1e-3)
    assert torch.all((h - h2).abs() <= 1e-5 * (1 + h2.abs()))


def test_dropped_elements_may_hold_anything():
    c = Case(200, 128, 256, [8, 16], 3, 24, rates=[0.5, 0.25])
    keep = c.keep()
    _, h0 = c.forward()
    _, a0, b0 = c.backward(None)
    c.x[~keep] = float("inf")
    c.x[0][~keep[0]] = float("nan")
    _, h = c.forward()
    assert torch.equal(h, h0)
    _, a, b = c.backward(None)
    assert all(torch.equal(p, q) for p, q in zip(a + b, a0 + b0))


def test_host_tables_accumulation_pitches_and_absent_outputs():
    c = Case(333, 136, 264, [8, 16, 24], 8, 25, cap=5)
    keep = c.keep()
    ref, tol = c.reference(keep)
    # tables in host memory may name registered tenants alone
    host = segments(c.off, c.slot, on_host=True)
    y, h = c.forward(seg=host)
    y1, h1 = c.forward()
    assert torch.equal(y, y1) and torch.equal(h, h1)
    dx, dA, dB = c.backward(h, fill=0.5, seg=host, flags=B.MARLAAS_FLAG_ACCUMULATE)
    for t in range(3):
        check(dA[t], ref["dA"][t] + 0.5, tol["dA"][t] + 1e-6 * (1 + ref["dA"][t].abs()), "dA")
        check(dB[t], ref["dB"][t] + 0.5, tol["dB"][t] + 1e-6 * (1 + ref["dB"][t].abs()), "dB")
    full = torch.full((c.T, 200), 4.0, dtype=torch.bfloat16, device="cuda")
    full[:, :136] = c.x
    out = torch.full((c.T, 320), 6.0, dtype=torch.bfloat16, device="cuda")
    B.marlaas_lora_forward_dropout(c.pool, full[:, :136], c.W, c.seg, c.rates_dev, SEED, OFFSET, y=out[:, :264])
    assert torch.equal(out[:, :264], y) and torch.all(out[:, 264:] == 6)
    only = torch.full_like(full, 2.0)
    B.marlaas_lora_backward_dropout(c.pool, None, c.W, c.dy, c.seg, c.rates_dev, SEED, OFFSET, dx=only[:, :136])
    assert torch.equal(only[:, :136], dx) and torch.all(only[:, 136:] == 2)
    a1 = [torch.zeros_like(g) if t != 1 else None for t, g in enumerate(dA)] + [None, None]
    B.marlaas_lora_backward_dropout(c.pool, full[:, :136], c.W, c.dy, c.seg, c.rates_dev, SEED, OFFSET, dA=a1)
    for t in (0, 2):
        check(a1[t], ref["dA"][t], tol["dA"][t] + 1e-30, "dA")
    # a batch without tokens
    z = torch.empty((0, 136), dtype=torch.bfloat16, device="cuda")
    B.marlaas_lora_backward_dropout(c.pool, z, c.W, c.dy[:0], segments([0, 0], [0]), c.rates_dev, SEED, OFFSET, dA=dA + [None, None])
    assert not any(g.any() for g in dA)


def test_finely_mixed_tenants():
    """A tenant per token: the copies of the gradient's blocks do not fit and the plain reduction runs."""
    c = Case(640, 64, 128, [8] * 40, 640, 26)
    check_case(c, c.keep())


def test_streams_and_graphs():
    c = Case(1200, 256, 384, [16, 8], 6, 27)
    y, h = c.forward()
    dx, dA, dB = c.backward(h)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y1 = B.marlaas_lora_forward_dropout(c.pool, c.x, c.W, c.seg, c.rates_dev, SEED, OFFSET, stream=side)
    dx1 = torch.empty_like(dx)
    B.marlaas_lora_backward_dropout(c.pool, c.x, c.W, c.dy, c.seg, c.rates_dev, SEED, OFFSET, dx=dx1, stream=side)
    side.synchronize()
    assert torch.equal(y1, y) and torch.equal(dx1, dx)
    graphs, outs = [], []
    for _ in range(2):
        o = [torch.zeros_like(v) for v in (y, h, dx)] + [[torch.zeros_like(v) for v in g] for g in (dA, dB)]
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            B.marlaas_lora_forward_dropout(c.pool, c.x, c.W, c.seg, c.rates_dev, SEED, OFFSET, y=o[0], h_save=o[1])
            B.marlaas_lora_backward_dropout(c.pool, c.x, c.W, c.dy, c.seg, c.rates_dev, SEED, OFFSET, dx=o[2], dA=o[3], dB=o[4], h_saved=o[1])
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
        assert torch.equal(o[0], y) and torch.equal(o[1], h) and torch.equal(o[2], dx)
        assert all(torch.equal(a, b) for a, b in zip(o[3] + o[4], dA + dB))
