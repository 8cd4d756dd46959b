"""AdamW with 8-bit moments on the GPU: masters against float64, codes bit for bit against the format's definition applied
to moments computed in numpy's fp32 with the same separate roundings, the pool's rows against the rounded masters.

A master differs from float64 by the few fp32 roundings of one update of size lr: 2e-5 relative / 1e-7 absolute, as for the
32-bit form."""
import math

import numpy as np
import pytest
import torch

from oracle import policy as op
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu

HP = dict(lr=2e-2, beta1=0.9, beta2=0.98, eps=1e-6, weight_decay=0.05, grad_scale=0.5)


def moments_f32(m, v, g):
    f = np.float32
    b1, b2, gs = f(HP["beta1"]), f(HP["beta2"]), f(HP["grad_scale"])
    g = gs * g.astype(f)
    m = b1 * m.astype(f) + (f(1) - b1) * g
    return m, b2 * v.astype(f) + ((f(1) - b2) * g) * g


class Tenant:
    def __init__(self, pool, tid, rank, seed):
        self.rank, self.tid = rank, tid
        r = np.random.RandomState(seed)
        widths = pool.parts or [pool.d_out]
        self.sizes = {"A": [pool.d_in * rank] * pool.n_parts, "B": [rank * w for w in widths]}
        self.theta = {x: [(0.05 * r.randn(n)).astype(np.float32) for n in s] for x, s in self.sizes.items()}
        self.state = {x: [np.zeros(B.marlaas_adamw_compact_state_bytes(n), np.uint8) for n in s] for x, s in self.sizes.items()}
        self.r = r

    def put(self, offset=0):
        """Device buffers; `offset` floats before each gradient and master, so that they are not 16-byte aligned."""
        def up(parts):
            a = np.concatenate([np.zeros(offset, np.float32)] + parts)
            return torch.from_numpy(a).cuda()[offset:]
        self.d = {x: up(self.theta[x]) for x in "AB"}
        self.dst = dict(zip("AB", B.compact_state(self.pool, self.rank)))
        self.dg = {x: torch.empty_like(self.d[x]) if offset == 0 else up([np.zeros_like(p) for p in self.theta[x]]) for x in "AB"}

    def new_grads(self, scale=1.0):
        self.g = {x: [(scale * self.r.randn(n) * np.exp(2 * self.r.randn(n))).astype(np.float32) for n in s] for x, s in self.sizes.items()}
        for x in "AB":
            self.dg[x].copy_(torch.from_numpy(np.concatenate(self.g[x])))

    def host_step(self, step, seed):
        for x, k in (("A", 0), ("B", 1)):
            for p, n in enumerate(self.sizes[x]):
                bits = op.random_bits(n, seed, step, self.tid, p, k)
                m0, v0 = op.decode_state(self.state[x][p], n)
                th, _, _, _ = op.adamw_compact_step(self.theta[x][p], self.g[x][p], self.state[x][p], bits, step=step, **HP)
                m, v = moments_f32(m0, v0, self.g[x][p])
                self.state[x][p] = op.encode_state(m, v, bits)
                self.theta[x][p] = th


CASES = {
    "one tenant": (64, 64, None, (8,), 0),
    "odd ranks, odd widths": (200, 136, None, (5, 1, 64, 127, 33), 0),
    "not 16-byte aligned": (72, 88, None, (16, 3), 1),
    "wide": (4096, 320, None, (16, 96), 0),
    "three projections": (264, 1024, (512, 256, 256), (16, 5), 0),
    "more tenants than a small table": (64, 72, None, (4,) * 60, 0),
}


@pytest.mark.parametrize("name", CASES)
def test_compact_commit_matches_the_definition(name):
    K, N, parts, ranks, offset = CASES[name]
    pool = B.AdapterPool(K, N, max(ranks), len(ranks) + 1, parts=list(parts) if parts else None)
    seed = (3 << 32) + 17
    ten = []
    for i, r in enumerate(ranks):
        tid = 10 + i + (7 << 33)
        t = Tenant(pool, tid, r, 100 + i)
        t.pool = pool
        t.put(offset)
        w = parts or (N,)
        As = [torch.from_numpy(a.astype(np.float32)).bfloat16().view(K, r).cuda() for a in t.theta["A"]]
        Bs = [torch.from_numpy(b.astype(np.float32)).bfloat16().view(r, w[p]).cuda() for p, b in enumerate(t.theta["B"])]
        B.marlaas_adapter_pool_register(pool, tid, 0, r, 16.0, As if parts else As[0], Bs if parts else Bs[0])
        ten.append(t)
    col = lambda f: [f(t) for t in ten]     # noqa: E731
    tables = B.CompactAdamWTables(pool, col(lambda t: t.tid), *(col(lambda t, x=x, a=a: getattr(t, a)[x]) for a, x in
                                  (("dg", "A"), ("dg", "B"), ("d", "A"), ("d", "B"), ("dst", "A"), ("dst", "B"))))
    for step in range(1, 4):
        for t in ten:
            t.new_grads(10.0 ** (1 - step))
        B.marlaas_adapter_pool_adamw_compact_commit(pool, tables, step=step, seed=seed, **HP)
        for t in ten:
            t.host_step(step, seed)
    B.marlaas_check_status(pool)
    At, Bs = pool.store()
    for i, t in enumerate(ten):
        for x in "AB":
            np.testing.assert_allclose(t.d[x].cpu().numpy(), np.concatenate(t.theta[x]), rtol=2e-5, atol=1e-7, err_msg=f"{i} {x}")
            # (the unused bytes of a block are not part of the state)
            got, want = t.dst[x].cpu().numpy().reshape(-1, 528)[:, :514], np.concatenate(t.state[x]).reshape(-1, 528)[:, :514]
            assert np.array_equal(got, want), f"tenant {i} {x}: {(got != want).sum()} of {got.size} bytes differ"
            m, v = B.marlaas_adamw_compact_state_export(pool, t.dst[x])
            at = 0
            for p, n in enumerate(t.sizes[x]):
                rm, rv = op.decode_state(t.state[x][p], n)
                assert np.array_equal(m[at:at + n].cpu().numpy(), rm.astype(np.float32)) and np.array_equal(v[at:at + n].cpu().numpy(), rv.astype(np.float32))
                at += -(-n // 256) * 256
        slot, rank, _, version = B.marlaas_adapter_pool_lookup(pool, t.tid)
        assert (slot, rank, version) == (i, ranks[i], 3)
        at0, c0, RP = 0, 0, pool.rank_stride
        for p in range(pool.n_parts):
            wp = (parts or (N,))[p]
            a = t.d["A"][p * K * rank:(p + 1) * K * rank].view(K, rank).bfloat16()
            b = t.d["B"][at0:at0 + rank * wp].view(rank, wp).bfloat16()
            assert torch.equal(At[p, i * RP:i * RP + rank], a.t()) and torch.equal(Bs[i * RP:i * RP + rank, c0:c0 + wp], b)
            assert torch.all(At[p, i * RP + rank:(i + 1) * RP] == 0) and torch.all(Bs[i * RP + rank:(i + 1) * RP] == 0)
            at0, c0 = at0 + rank * wp, c0 + wp
    # the same call on the same buffers gives the same bits; another seed does not
    state = [t.dst["A"].clone() for t in ten]
    keep = [(t.d["A"].clone(), t.d["B"].clone(), t.dst["B"].clone()) for t in ten]
    after = []
    for s in (seed, seed, seed + 1):
        for t, st, (a, b, sb) in zip(ten, state, keep):
            t.dst["A"].copy_(st), t.dst["B"].copy_(sb), t.d["A"].copy_(a), t.d["B"].copy_(b)
        B.marlaas_adapter_pool_adamw_compact_commit(pool, tables, step=4, seed=s, **HP)
        after.append([t.dst["A"].clone() for t in ten])
    assert all(torch.equal(x, y) for x, y in zip(after[0], after[1]))
    assert not all(torch.equal(x, y) for x, y in zip(after[0], after[2]))


def test_codes_are_those_of_separately_rounded_operations_over_millions_of_elements():
    # a product and a sum fused into one rounding move about one code in a million: 16 million elements, two steps, all
    # bytes equal to the same fp32 operations done one by one with torch
    K, N, r, T = 4096, 4096, 64, 32
    pool = B.AdapterPool(K, N, r, T)
    g = torch.Generator(device="cuda").manual_seed(4)
    for t in range(T):
        B.marlaas_adapter_pool_register(pool, t, 0, r, 1.0, torch.zeros(K, r, dtype=torch.bfloat16, device="cuda"),
                                        torch.zeros(r, N, dtype=torch.bfloat16, device="cuda"))
    n = K * r
    grad = torch.randn(2 * T, n, generator=g, device="cuda") * torch.exp(2 * torch.randn(2 * T, n, generator=g, device="cuda"))
    theta, state = torch.zeros_like(grad), torch.zeros(2 * T, n // 256 * 528, dtype=torch.uint8, device="cuda")
    part = lambda x, k: [x[2 * t + k] for t in range(T)]        # noqa: E731
    tables = B.CompactAdamWTables(pool, range(T), part(grad, 0), part(grad, 1), part(theta, 0), part(theta, 1), part(state, 0), part(state, 1))
    f = lambda x: float(np.float32(x))      # noqa: E731
    ref = state.clone()
    bits = [torch.from_numpy(op.random_bits(n, 6, s, t, 0, k).astype(np.int64)) for s in (1, 2) for t in range(T) for k in (0, 1)]
    for step in (1, 2):
        B.marlaas_adapter_pool_adamw_compact_commit(pool, tables, step=step, seed=6, **HP)
        blk = ref.view(-1, 528)
        rnd = torch.stack(bits[(step - 1) * 2 * T:step * 2 * T]).cuda().view(-1, 256)
        new = {}
        gr = (grad * f(HP["grad_scale"])).view(-1, 256)
        for name, at, orders, beta in (("m", 0, 15, HP["beta1"]), ("v", 256, 31, HP["beta2"])):
            code = blk[:, at:at + 256].int()
            base = ((blk[:, 512 + at // 256].int() - orders) * 8).clamp(min=0)[:, None]
            mag = code & 127 if name == "m" else code
            old = torch.where(mag > 0, (mag + base) << 20, torch.zeros_like(mag)).view(torch.float32)
            old = torch.where(code > 127, -old, old) if name == "m" else old
            one = float(np.float32(1) - np.float32(beta))
            new[name] = old * f(beta) + (gr * one if name == "m" else (gr * one) * gr)
        for name, at, orders, half in (("m", 0, 15, rnd & 0xFFFF), ("v", 256, 31, rnd >> 16)):
            x = new[name]
            b = x.view(torch.int32) & 0x7FFFFFFF
            E = (b.amax(1) + 0xFFFFF) >> 23
            code = ((b + (half.int() << 4)) >> 20) - ((E - orders) * 8).clamp(min=0)[:, None]
            code = code.clamp(min=0) + torch.where(x < 0, 128, 0) if name == "m" else torch.where(b > 0, code.clamp(min=1), torch.zeros_like(code))
            blk[:, at:at + 256], blk[:, 512 + at // 256] = code.to(torch.uint8), E.to(torch.uint8)
        got = state.view(-1, 528)[:, :514]
        assert torch.equal(got, blk[:, :514]), f"step {step}: {(got != blk[:, :514]).sum().item()} bytes differ"


def _small_pool(ranks=(8, 4)):
    pool = B.AdapterPool(64, 64, 8, 3)
    bufs = []
    for i, r in enumerate(ranks):
        a, b = torch.zeros((64, r), device="cuda"), torch.zeros((r, 64), device="cuda")
        B.marlaas_adapter_pool_register(pool, i + 1, 0, r, 1.0, a.bfloat16(), b.bfloat16())
        bufs.append((torch.zeros_like(a), torch.zeros_like(b), a, b, *B.compact_state(pool, r)))
    return pool, bufs


def _tables(pool, ids, bufs):
    return B.CompactAdamWTables(pool, ids, *zip(*bufs))


def test_moments_out_of_range_and_not_finite():
    pool, bufs = _small_pool((8,))
    g = bufs[0][0].view(-1)
    g[0], g[1], g[2], g[3], g[4] = math.nan, math.inf, 3e38, 1e-30, -1e-18
    g[256:512] = 1e-25 * torch.randn(256, device="cuda")          # a block of squares below the smallest number
    tables = _tables(pool, [1], bufs)
    B.marlaas_adapter_pool_adamw_compact_commit(pool, tables, lr=1e-3, step=1)
    m, v = B.marlaas_adamw_compact_state_export(pool, bufs[0][4])
    assert torch.isfinite(m).all() and torch.isfinite(v).all()
    A = bufs[0][2].view(-1)
    assert torch.isnan(A[0]) and not torch.isfinite(A[1]) and m[0] == 0 and m[1] == 0
    assert m[2] > 2.6e37 and v[2] == 0               # (its square is not finite)
    assert torch.isfinite(A[3:]).all() and torch.all(v[256:512] == 0) and m[256:512].abs().max() > 0
    # zero gradients on zero moments change nothing
    pool2, b2 = _small_pool((4,))
    b2[0][2].fill_(0.5)
    B.marlaas_adapter_pool_adamw_compact_commit(pool2, _tables(pool2, [1], b2), lr=1e-3, step=1)
    assert torch.all(b2[0][2] == 0.5) and torch.all(b2[0][4] == 0)


def test_compact_commit_refuses():
    pool, bufs = _small_pool()
    tables = _tables(pool, [1, 2], bufs)
    L, n0 = B.load_library(), B.marlaas_kernel_launch_count()

    def call(ids, rows, status, **kw):
        t = _tables(pool, [1, 2], bufs)
        t.n, t.ids = len(ids), (B.ctypes.c_uint64 * max(len(ids), 1))(*ids)
        for tab, k in rows:
            t.tables[tab][k] = None
        with pytest.raises(B.MarlaasError) as e:
            B.marlaas_adapter_pool_adamw_compact_commit(pool, t, lr=1e-3, **kw)
        assert e.value.status == status, e.value

    call([1, 99], [], B.MARLAAS_ERR_UNKNOWN_TENANT)
    call([1, 1], [], B.MARLAAS_ERR_INVALID_ARG)
    call([1, 2], [], B.MARLAAS_ERR_INVALID_ARG, step=0)
    call([1, 2], [], B.MARLAAS_ERR_INVALID_ARG, beta1=1.0)
    call([1, 2], [], B.MARLAAS_ERR_INVALID_ARG, beta2=-0.1)
    for k in range(6):
        call([1, 2], [(k, 1)], B.MARLAAS_ERR_INVALID_ARG)
    call([2, 1], [], B.MARLAAS_ERR_INVALID_ARG)                          # each with the other's buffers: other ranks
    with pytest.raises(AssertionError):
        _tables(pool, [2, 1], bufs)
    with pytest.raises(AssertionError):
        _tables(pool, [1], [(bufs[0][0].double(),) + bufs[0][1:]])
    assert L.marlaas_adamw_compact_state_export(pool.handle, -1, None, None, None, None) == B.MARLAAS_ERR_INVALID_ARG
    odd = torch.zeros(528 + 8, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.MarlaasError):
        B.marlaas_adamw_compact_state_export(pool, odd[8:])
    assert B.marlaas_kernel_launch_count() == n0
    # a tenant that has been registered anew with another rank
    B.marlaas_adapter_pool_register(pool, 2, 5, 8, 1.0, torch.zeros((64, 8), device="cuda").bfloat16(), torch.zeros((8, 64), device="cuda").bfloat16())
    with pytest.raises(B.MarlaasError) as e:
        B.marlaas_adapter_pool_adamw_compact_commit(pool, tables, lr=1e-3)
    assert e.value.status == B.MARLAAS_ERR_INVALID_ARG
    assert B.marlaas_adapter_pool_lookup(pool, 1)[3] == 0
    B.marlaas_adapter_pool_register(pool, 2, 5, 4, 1.0, torch.zeros((64, 4), device="cuda").bfloat16(), torch.zeros((4, 64), device="cuda").bfloat16())
    B.marlaas_adapter_pool_adamw_compact_commit(pool, tables, lr=1e-3, new_versions=[9, 8])
    assert B.marlaas_adapter_pool_lookup(pool, 1)[3] == 9 and B.marlaas_adapter_pool_lookup(pool, 2)[3] == 8
