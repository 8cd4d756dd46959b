"""AdamW with 8-bit moments: a commit of many tenants in one call is that of each by itself, whatever length of units the number
of elements calls for."""
import pytest
import torch

from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K,N,parts,ranks", [(1304, 1432, None, (8, 16, 32, 64, 5) * 8), (1024, 768, [256, 256, 256], (16, 33) * 16),
                                             (2048, 2048, None, (32,) * 24)])
def test_one_call_for_many_tenants_gives_the_bits_of_one_call_each(K, N, parts, ranks):
    n = len(ranks)
    elements = sum(ranks) * (K * len(parts or [N]) + N)
    assert 2.4e6 < elements < 9.7e6
    pool = B.AdapterPool(K, N, max(ranks), n, parts=parts)
    P = pool.n_parts
    g = torch.Generator(device="cuda").manual_seed(n)
    rand = lambda *shape: 1e-2 * torch.randn(*shape, generator=g, device="cuda")      # noqa: E731
    grads = [(rand(P * K * r), rand(r * N)) for r in ranks]
    start = [(rand(P * K * r), rand(r * N)) for r in ranks]
    for t, r in enumerate(ranks):
        a, b = start[t][0].bfloat16().view(P, K, r), start[t][1].bfloat16()
        B.marlaas_adapter_pool_register(pool, t, 0, r, 1.0, list(a) if parts else a[0], list(b.view(P, r, N // P)) if parts else b.view(r, N))
    out = []
    for together in (True, False):
        masters = [(a.clone(), b.clone()) for a, b in start]
        states = [B.compact_state(pool, r) for r in ranks]
        rows = [(*grads[t], *masters[t], *states[t]) for t in range(n)]
        for step in (1, 2):
            for ids in ([list(range(n))] if together else [[t] for t in range(n)]):
                tables = B.CompactAdamWTables(pool, ids, *zip(*(rows[t] for t in ids)))
                B.marlaas_adapter_pool_adamw_compact_commit(pool, tables, lr=1e-3, step=step, seed=5)
        used = [s.view(-1, 528)[:, :514] for pair in states for s in pair]
        out.append([x for pair in masters for x in pair] + used + [v.clone() for v in pool.store()])
    assert all(torch.equal(x, y) for x, y in zip(*out))
