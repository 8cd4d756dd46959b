"""Measured cases of the policy-update operators: group advantages, token log-probabilities, the clipped policy loss with
its gradient, and AdamW with 8-bit moments committed into the adapter store.

`run` computes a case either in its plain form (elementary torch operations in 32 bits, `own = False`) or through the
library's calls (`own = True`) on the same inputs.  `exact` gives the definition's values in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
CLIP_LOW, CLIP_HIGH, INV_TEMPERATURE, GRAD_SCALE = 0.2, 0.28, 1.0 / 0.9, 1.0
ADV_EPS = 1e-6
ADAM = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.01, grad_scale=0.5, step=7)
ADAM_SEED = 20240229
BLOCK, STATE_BLOCK = 256, 528               # elements of a block of 8-bit moments, and its bytes
RANKS = (8, 16, 32, 64)


def listed():
    return [
        # one small task's rollouts of one prompt set: a launch-bound call between two decode steps
        dict(name="advantages, 1 task", op="advantages", tenants=1, groups=4, group=8, median=64, longest=256, token_mean=False, std=True),
        # 32 concurrent tasks, all their groups in one training batch of about two million tokens
        dict(name="advantages, 32 tasks", op="advantages", tenants=32, groups=256, group=8, median=1024, longest=4096, token_mean=True, std=True),
        # behaviour log-probabilities of one decode step of a rollout batch
        dict(name="logprobs, decode", op="logprobs", T=32, V=32768, dtype="bf16", entropy=False, ignored=0.0, masked=False),
        # fp32 logits of an odd vocabulary, entropy wanted, a quarter of the rows prompt tokens
        dict(name="logprobs, fp32 odd", op="logprobs", T=1021, V=50001, dtype="f32", entropy=True, ignored=0.25, masked=True),
        # reference-policy pass over a training batch
        dict(name="logprobs, prefill", op="logprobs", T=4096, V=131072, dtype="bf16", entropy=False, ignored=0.0, masked=False),
        # the loss of a single token: latency
        dict(name="loss, 1 token", op="loss", T=1, V=32768, dtype="bf16", tenants=1, kl=0.04, entropy=0.0, ignored=0.0, masked=False),
        # an odd vocabulary with masked entries, prompt tokens, KL and entropy terms
        dict(name="loss, bf16 odd", op="loss", T=1000, V=100003, dtype="bf16", tenants=8, kl=0.04, entropy=0.003, ignored=0.25, masked=True),
        # fp32 logits
        dict(name="loss, fp32", op="loss", T=1024, V=32768, dtype="f32", tenants=4, kl=0.0, entropy=0.0, ignored=0.1, masked=False),
        # a training batch over a large vocabulary
        dict(name="loss, bf16 large", op="loss", T=4096, V=131072, dtype="bf16", tenants=10, kl=0.04, entropy=0.0, ignored=0.1, masked=False),
        # one small adapter: latency
        dict(name="adamw, 1 adapter", op="adamw", d_in=512, d_out=512, parts=1, tenants=1, rank=8),
        # heterogeneous tenants over one square projection
        dict(name="adamw, 32 ranks 8-64", op="adamw", d_in=5120, d_out=5120, parts=1, tenants=32, rank=0),
        # q, k, v of a 7B-shaped decoder layer through one pool
        dict(name="adamw, q k v rank 32", op="adamw", d_in=4096, d_out=12288, parts=3, tenants=32, rank=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["advantages", "logprobs", "loss", "loss", "adamw"])
    if op == "advantages":
        return dict(op=op, tenants=rng.randint(1, 32), groups=_log_int(rng, 2, 256), group=rng.randint(2, 8), median=_log_int(rng, 16, 1024),
                    longest=rng.randint(1024, 4096), token_mean=rng.random() < 0.5, std=rng.random() < 0.8)
    if op in ("logprobs", "loss"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        T, V = _log_int(rng, 1, 4096), _log_int(rng, 1000, 131072)
        while T * V * (4 if dtype == "f32" else 2) > 4096 * 131072 * 2:
            T = _log_int(rng, 1, 4096)
        ignored, masked = rng.choice([0.0, 0.1, 0.25]), rng.random() < 0.4
        if op == "logprobs":
            return dict(op=op, T=T, V=V, dtype=dtype, entropy=rng.random() < 0.5, ignored=ignored, masked=masked)
        return dict(op=op, T=T, V=V, dtype=dtype, tenants=rng.randint(1, 32), kl=rng.choice([0.0, 0.04]), entropy=rng.choice([0.0, 0.003]),
                    ignored=ignored, masked=masked)
    if rng.random() < 0.33:     # q, k, v: three projections of one width
        return dict(op=op, d_in=256 * _log_int(rng, 1, 16), d_out=768 * _log_int(rng, 1, 16), parts=3, tenants=_log_int(rng, 1, 32),
                    rank=rng.choice([5, 8, 16, 32]))
    return dict(op=op, d_in=8 * _log_int(rng, 16, 640), d_out=8 * _log_int(rng, 16, 640), parts=1, tenants=_log_int(rng, 1, 32),
                rank=rng.choice([0, 5, 8, 16, 32, 64]))


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _pool(d_in, d_out, max_rank, capacity, parts=None):
    from paper_2605_08527_b200 import binding
    return binding.AdapterPool(d_in, d_out, max_rank, capacity, device=DEV, parts=parts)


def _segments(off, slot):
    from paper_2605_08527_b200 import binding
    return binding.Segments(off, slot)


def _lengths(case):
    """The sequence lengths of an advantages case: lognormal, the same for every seed but in another order."""
    r = np.random.RandomState(11)
    n = case["groups"] * case["group"] - case["groups"] // 3        # ragged groups
    return np.clip(np.round(np.exp(r.normal(math.log(case["median"]), 0.6, n))), 1, case["longest"]).astype(np.int64)


def _prepare_advantages(case, seed):
    r = np.random.RandomState(seed % (1 << 31))
    lens = r.permutation(_lengths(case))
    S, G = len(lens), case["groups"]
    sizes = np.full(G, S // G) + (np.arange(G) < S % G)
    off = np.concatenate([[0], np.cumsum(lens)])
    T = int(off[-1])
    group_off = np.concatenate([[0], np.cumsum(sizes)])
    group_of = np.repeat(np.arange(G), sizes)
    slot = (np.sort(r.randint(0, case["tenants"], G)))[group_of]
    # verifiable rewards: 0 or 1 with a success rate of the prompt's own (some groups all alike), a few partial ones
    p = r.rand(G)[group_of]
    rewards = np.where(r.rand(S) < 0.1, 0.1, r.rand(S) < p).astype(np.float32)
    g = _gen(seed)
    targets = torch.randint(0, 32000, (T,), generator=g, device=DEV, dtype=torch.int32)
    # the first quarter of every sequence is its prompt; one sequence in 50 was cut off and trains on nothing
    seq = torch.repeat_interleave(torch.arange(S, device=DEV), torch.from_numpy(lens).to(DEV))
    pos = torch.arange(T, device=DEV) - torch.from_numpy(off[:-1]).to(DEV)[seq]
    cut = torch.from_numpy(np.where(r.rand(S) < 0.02, lens, lens // 4)).to(DEV)
    targets[pos < cut[seq]] = -1
    s = dict(case=case, T=T, cap=case["tenants"], off=_i32(off), slot=_i32(slot), group_off=_i32(group_off), targets=targets,
             rewards=torch.from_numpy(rewards).to(DEV))
    if own:
        s["pool"], s["seg"] = _pool(64, 64, 8, s["cap"]), _segments(s["off"], s["slot"])
    return s


def _logits(case, seed):
    """[T][V] logits inside rows padded to 16 bytes, and targets: normal, the sampled token raised by up to 10."""
    T, V = case["T"], case["V"]
    dt, pad = (torch.float32, 4) if case["dtype"] == "f32" else (torch.bfloat16, 8)
    ld = -(-V // pad) * pad
    g = _gen(seed)
    z = torch.empty((T, ld), dtype=dt, device=DEV).normal_(0.0, 2.0, generator=g)[:, :V]
    head = max(1, V // 8)
    tgt = torch.randint(0, head, (T,), generator=g, device=DEV)
    rows = torch.arange(T, device=DEV)
    if case["masked"]:
        z[:, V - max(1, V // 512):] = -math.inf                     # entries that only pad the embedding table
        z[3::16, head:] = torch.finfo(dt).min                       # constrained decoding
    z[rows, tgt] += (10 * torch.rand(T, generator=g, device=DEV)).to(dt)
    ignored = torch.rand(T, generator=g, device=DEV) < case["ignored"]
    return z, torch.where(ignored, -1, tgt).to(torch.int32), g


def _prepare_logprobs(case, seed):
    z, targets, _ = _logits(case, seed)
    s = dict(case=case, z=z, targets=targets)
    if own:
        s["pool"] = _pool(64, 64, 8, 1)
    return s


def _prepare_loss(case, seed):
    z, targets, g = _logits(case, seed)
    T, cap = case["T"], case["tenants"]
    # sequences of about 128 tokens, tenants in any order, some on the base weight alone
    r = np.random.RandomState(seed % (1 << 31))
    n = max(1, T // 128)
    off = np.unique(np.concatenate([[0], r.randint(0, T + 1, n - 1), [T]]))
    slot = r.randint(0 if len(off) < 4 else -1, cap, len(off) - 1)
    # the behaviour policy is near the current one; ratios keep clear of the clip's edges by more than rounding
    old = torch.empty(T, device=DEV)
    a = targets.clamp(min=0).long()
    for i in range(0, T, 256):
        zz = z[i:i + 256].float() * INV_TEMPERATURE
        old[i:i + 256] = torch.gather(zz, 1, a[i:i + 256, None])[:, 0] - torch.logsumexp(zz, 1)
    delta = 0.15 * torch.randn(T, generator=g, device=DEV)
    for edge in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH)):
        delta = torch.where((delta - edge).abs() < 1e-3, delta + 4e-3, delta)
    ref = old + 0.1 * torch.randn(T, generator=g, device=DEV)
    adv = torch.randn(T, generator=g, device=DEV)
    w = torch.rand(T, generator=g, device=DEV) * (2.0 / T)
    s = dict(case=case, z=z, targets=targets, cap=cap, off=_i32(off), slot=_i32(slot), old=old - delta, ref=ref if case["kl"] else None, adv=adv, w=w)
    if own:
        s["pool"], s["seg"] = _pool(64, 64, 8, cap), _segments(s["off"], s["slot"])
    return s


def _ranks(case):
    return [case["rank"] or RANKS[t % 4] for t in range(case["tenants"])]


def _matrices(case):
    """(part, 0 for A / 1 for B, tenant, rows, columns) in the order of the flat buffers, A's first; every matrix of a part
    starts on a block of its own."""
    P, K, N = case["parts"], case["d_in"], case["d_out"] // case["parts"]
    ranks = _ranks(case)
    return ([(p, 0, t, K, r) for t, r in enumerate(ranks) for p in range(P)],
            [(p, 1, t, r, N) for t, r in enumerate(ranks) for p in range(P)])


def _mix(x):
    """The 32-bit mixing function that turns an element's number into its random bits (definition of the rounding)."""
    x &= 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xB504F333) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _key(step, tenant, part, matrix):
    k = 0
    for word in (ADAM_SEED & 0xFFFFFFFF, ADAM_SEED >> 32, step & 0xFFFFFFFF, step >> 32, tenant & 0xFFFFFFFF, tenant >> 32, 2 * part + matrix):
        k = _mix((k + 0x9E3779B9) ^ word)
    return k


def _prepare_adamw(case, seed):
    g = _gen(seed)
    P, K, N, cap = case["parts"], case["d_in"], case["d_out"], case["tenants"]
    RP = -(-max(_ranks(case)) // 16) * 16
    s = dict(case=case)
    for x, mats in zip("AB", _matrices(case)):
        sizes = np.array([rows * cols for _, _, _, rows, cols in mats], dtype=np.int64)
        blocks = -(-sizes // BLOCK)
        first = np.concatenate([[0], np.cumsum(blocks)])
        nb = int(first[-1])
        of = np.repeat(np.arange(len(mats)), blocks)
        e0 = (np.arange(nb) - first[of]) * BLOCK
        e = (torch.from_numpy(e0).to(DEV)[:, None] + torch.arange(BLOCK, device=DEV)).view(-1)      # an element's number in its matrix
        m = torch.from_numpy(of).to(DEV).repeat_interleave(BLOCK)
        live = e < torch.from_numpy(sizes).to(DEV)[m]
        col = lambda i: torch.tensor([int(mat[i]) for mat in mats], device=DEV)[m]      # noqa: E731
        p, t, rows, cols = col(0), col(2), col(3), col(4)
        i, j = e // cols, e % cols
        if x == "A":       # row (slot RP + j) of A block p holds column j of A_t,p
            at = ((p * cap + t) * RP + j) * K + i
        else:              # row (slot RP + i), the projection's columns
            at = (t * RP + i) * N + p * (N // P) + j
        s["at" + x] = torch.where(live, at, cap * RP * (P * K if x == "A" else N))
        keys = torch.tensor([_key(ADAM["step"], 1000 + mat[2], mat[0], mat[1]) for mat in mats], device=DEV)
        s["e" + x] = (e + keys[m]) & 0xFFFFFFFF
        s["theta" + x] = 0.02 * torch.randn(nb * BLOCK, generator=g, device=DEV) * live
        # gradients whose scale varies from block to block, as it does between layers and tenants
        scale = torch.exp(torch.randn(nb, generator=g, device=DEV) - 9).repeat_interleave(BLOCK)
        s["grad" + x] = torch.randn(nb * BLOCK, generator=g, device=DEV) * scale * live
        # moments of earlier steps: m of either sign within 2^-4 of the block's largest, v within 2^-8
        st = torch.zeros((nb, STATE_BLOCK), dtype=torch.uint8, device=DEV)
        lv = live.view(nb, BLOCK)
        sign = 128 * torch.randint(0, 2, (nb, BLOCK), generator=g, device=DEV)
        st[:, :BLOCK] = ((sign + torch.randint(88, 128, (nb, BLOCK), generator=g, device=DEV)) * lv).to(torch.uint8)
        st[:, BLOCK:2 * BLOCK] = (torch.randint(184, 256, (nb, BLOCK), generator=g, device=DEV) * lv).to(torch.uint8)
        st[:, 2 * BLOCK] = torch.randint(110, 116, (nb,), generator=g, device=DEV).to(torch.uint8)
        st[:, 2 * BLOCK + 1] = torch.randint(94, 102, (nb,), generator=g, device=DEV).to(torch.uint8)
        s["state" + x] = st
        s["store" + x] = torch.zeros(cap * RP * (P * K if x == "A" else N) + 1, dtype=torch.bfloat16, device=DEV)
        s["split" + x] = (mats, sizes, first)
    if own:
        _own_adamw(s, case, RP)
    return s


def _own_adamw(s, case, RP):
    """The pool with its tenants registered, and the table of the tenants' tensors: views of the flat buffers, in which a
    tenant's projections lie one after another (the cases with several have whole blocks in each)."""
    from paper_2605_08527_b200 import binding as B
    P, K, N = case["parts"], case["d_in"], case["d_out"]
    pool = _pool(K, N, max(_ranks(case)), case["tenants"], None if P == 1 else [N // P] * P)
    cols = {}
    for x in "AB":
        mats, sizes, first = s["split" + x]
        for kind in ("grad", "theta", "state"):
            cols[kind + x] = []
            for t in range(case["tenants"]):
                k = [n for n, mat in enumerate(mats) if mat[2] == t]
                lo, hi = int(first[k[0]]), int(first[k[-1] + 1])
                if kind == "state":
                    cols[kind + x].append(s["state" + x][lo:hi])
                    continue
                v = s[kind + x][lo * BLOCK:hi * BLOCK]
                size = int(sizes[k].sum())
                assert P == 1 or size == v.numel()
                cols[kind + x].append(v[:size])
    for t, r in enumerate(_ranks(case)):
        a, b = cols["thetaA"][t].bfloat16(), cols["thetaB"][t].bfloat16()
        if P == 1:
            a, b = a.view(K, r), b.view(r, N)
        else:
            a, b = list(a.view(P, K, r)), list(b.view(P, r, N // P))
        B.marlaas_adapter_pool_register(pool, 1000 + t, 0, r, 2.0 * r, a, b)
    s["pool"] = pool
    s["tables"] = B.CompactAdamWTables(pool, [1000 + t for t in range(case["tenants"])], cols["gradA"], cols["gradB"], cols["thetaA"],
                                       cols["thetaB"], cols["stateA"], cols["stateB"])


def prepare(case, seed):
    case = dict(case)
    return {"advantages": _prepare_advantages, "logprobs": _prepare_logprobs, "loss": _prepare_loss, "adamw": _prepare_adamw}[case["op"]](case, seed)


# ---- one pass ----------------------------------------------------------------------------------------------------------

def _plain_advantages(s):
    c, T, S = s["case"], s["T"], s["rewards"].numel()
    go, off = s["group_off"].long(), s["off"].long()
    G, dev = go.numel() - 1, s["rewards"].device
    group = torch.repeat_interleave(torch.arange(G, device=dev), go[1:] - go[:-1], output_size=S)
    n = (go[1:] - go[:-1]).float()
    d = s["rewards"] - s["rewards"][go[:-1].clamp(max=S - 1)][group]
    mean = torch.zeros(G, device=dev).index_add_(0, group, d) / n
    c0 = d - mean[group]
    seq_adv = c0
    if c["std"]:
        var = torch.zeros(G, device=dev).index_add_(0, group, c0 * c0) / n
        seq_adv = c0 / (torch.sqrt(var)[group] + ADV_EPS)
    seq = torch.repeat_interleave(torch.arange(S, device=dev), off[1:] - off[:-1], output_size=T)
    active = s["targets"] >= 0
    length = torch.zeros(S, dtype=torch.int64, device=dev).index_add_(0, seq, active.long())
    bucket = torch.where(s["slot"] < 0, s["cap"], s["slot"]).long()
    per = length if c["token_mean"] else (length > 0).long()
    total = torch.zeros(s["cap"] + 1, dtype=torch.int64, device=dev).index_add_(0, bucket, per)
    w = total[bucket].float() if c["token_mean"] else total[bucket].float() * length.float()
    weight = torch.where(active, 1.0 / w[seq], torch.zeros((), device=dev))
    return dict(seq_adv=seq_adv, adv=torch.where(active, seq_adv[seq], torch.zeros((), device=dev)), weight=weight)


def _plain_rows(z, targets, inv_temperature):
    """Per row: e = exp((z - m)/tau), (z - m)/tau, log of the sum, log-probability of the target, entropy, and whether the
    row counts (it has a target and a finite logit)."""
    z = z.float()
    m = z.amax(1, keepdim=True)
    t = (z - torch.where(m == -math.inf, torch.zeros_like(m), m)) * inv_temperature
    e = torch.exp(t)
    total = e.sum(1)
    live = (targets >= 0) & (total > 0)
    total = torch.where(live, total, torch.ones_like(total))
    log_s = torch.log(total)
    a = targets.clamp(min=0).long()
    logp = torch.where(live, torch.gather(t, 1, a[:, None])[:, 0] - log_s, torch.zeros_like(log_s))
    p = e / total[:, None]
    H = log_s - torch.where(e > 0, p * t, torch.zeros_like(t)).sum(1)
    return p, t, log_s, logp, torch.where(live, H, torch.zeros_like(H)), live, a


def _plain_logprobs(s):
    _, _, _, logp, H, _, _ = _plain_rows(s["z"], s["targets"], INV_TEMPERATURE)
    return dict(logp=logp, entropy=H) if s["case"]["entropy"] else dict(logp=logp)


def _plain_loss(s):
    c, T = s["case"], s["targets"].numel()
    p, t, log_s, logp, H, live, a = _plain_rows(s["z"], s["targets"], INV_TEMPERATURE)
    zero = torch.zeros_like(logp)
    rho = torch.exp(logp - s["old"])
    plain, clipped = rho * s["adv"], rho.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * s["adv"]
    free = plain <= clipped
    pg = -torch.minimum(plain, clipped)
    coef = torch.where(free, -plain, zero)
    kl = zero
    if c["kl"]:
        d = s["ref"] - logp
        kl = torch.expm1(d) - d
        coef = coef - c["kl"] * torch.expm1(d)
    w = torch.where(live, s["w"], zero)
    loss = pg + c["kl"] * kl - c["entropy"] * H
    k = w * (GRAD_SCALE * INV_TEMPERATURE)
    grad = p * (-coef[:, None])
    if c["entropy"]:
        grad = grad + torch.where(p > 0, p * (c["entropy"] * (t - log_s[:, None] + H[:, None])), torch.zeros_like(p))
    grad[torch.arange(T, device=grad.device), a] += coef
    grad = torch.where(live[:, None], grad * k[:, None], torch.zeros_like(grad))
    one = torch.ones_like(w)
    terms = torch.stack([w * loss, w * pg, w * kl, w * H, w * rho, torch.where(free, zero, w), w, one], 1)
    terms = torch.where(live[:, None], terms, torch.zeros_like(terms))
    off = s["off"].long()
    bucket = torch.where(s["slot"] < 0, s["cap"], s["slot"]).long()
    bucket = torch.repeat_interleave(bucket, off[1:] - off[:-1], output_size=T)
    stats = torch.zeros((s["cap"] + 1, 8), device=w.device).index_add_(0, bucket, terms)
    return dict(dlogits=grad.to(s["z"].dtype), logp=logp, stats=stats)


def _bits(x):
    return x.view(torch.int32)


def _mix_tensor(x):
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xB504F333) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _decode(code, expo, signed):
    """The values that 8-bit codes of [blocks][256] stand for."""
    code = code.int()
    base = ((expo.int() - (15 if signed else 31)) * 8).clamp(min=0)[:, None]
    mag = code & 127 if signed else code
    v = torch.where(mag > 0, (mag + base) << 20, torch.zeros_like(mag)).view(torch.float32)
    return torch.where(code > 127, -v, v) if signed else v


def _encode(x, rnd, signed):
    """Codes and block exponents of [blocks][256] values; `rnd`: 16 random bits for each."""
    b = _bits(x) & 0x7FFFFFFF
    b = torch.where(b >= 0x7F800000, torch.zeros_like(b), b.clamp(max=0x7F700000))
    expo = (b.amax(1) + 0xFFFFF) >> 23
    base = ((expo - (15 if signed else 31)) * 8).clamp(min=0)[:, None]
    q = ((b + (rnd << 4)) >> 20) - base
    if signed:
        return q.clamp(min=0) + torch.where(x < 0, 128, 0), expo
    return torch.where(b > 0, q.clamp(min=1), torch.zeros_like(q)), expo


def _plain_adamw(s):
    h = ADAM
    f = np.float32
    one_b1, one_b2 = float(f(1) - f(h["beta1"])), float(f(1) - f(h["beta2"]))
    c1, c2 = 1 / (1 - float(f(h["beta1"])) ** h["step"]), 1 / (1 - float(f(h["beta2"])) ** h["step"])
    out = {}
    for x in ("A", "B"):
        st, nb = s["state" + x], s["state" + x].shape[0]
        grad = s["grad" + x].view(nb, BLOCK) * h["grad_scale"]
        m = _decode(st[:, :BLOCK], st[:, 2 * BLOCK], True) * h["beta1"] + grad * one_b1
        v = _decode(st[:, BLOCK:2 * BLOCK], st[:, 2 * BLOCK + 1], False) * h["beta2"] + (grad * one_b2) * grad
        theta = s["theta" + x].view(nb, BLOCK)
        theta -= h["lr"] * ((m * c1) / (torch.sqrt(v * c2) + h["eps"]) + h["weight_decay"] * theta)
        rnd = _mix_tensor(s["e" + x]).view(nb, BLOCK)
        mc, me = _encode(m, (rnd & 0xFFFF).int(), True)
        vc, ve = _encode(v, (rnd >> 16).int(), False)
        st[:, :BLOCK], st[:, BLOCK:2 * BLOCK], st[:, 2 * BLOCK], st[:, 2 * BLOCK + 1] = mc, vc, me, ve
        s["store" + x][s["at" + x]] = theta.view(-1).bfloat16()
        out["theta" + x] = s["theta" + x]
        out["m" + x] = _decode(st[:, :BLOCK], st[:, 2 * BLOCK], True).view(-1)
        out["v" + x] = _decode(st[:, BLOCK:2 * BLOCK], st[:, 2 * BLOCK + 1], False).view(-1)
        out["store" + x] = s["store" + x][:-1]
    return out


def _own_run(s):
    from paper_2605_08527_b200 import binding as B
    c = s["case"]
    if c["op"] == "advantages":
        seq_adv, adv, weight = B.marlaas_group_advantages(
            s["pool"], s["seg"], s["rewards"], s["group_off"], s["targets"], eps=ADV_EPS,
            flags=(B.MARLAAS_FLAG_TOKEN_MEAN if c["token_mean"] else 0) | (0 if c["std"] else B.MARLAAS_FLAG_NO_STD))
        return dict(seq_adv=seq_adv, adv=adv, weight=weight)
    if c["op"] == "logprobs":
        if not c["entropy"]:
            return dict(logp=B.marlaas_token_logprobs(s["pool"], s["z"], s["targets"], inv_temperature=INV_TEMPERATURE))
        logp, entropy = B.marlaas_token_logprobs(s["pool"], s["z"], s["targets"], inv_temperature=INV_TEMPERATURE, with_entropy=True)
        return dict(logp=logp, entropy=entropy)
    if c["op"] == "loss":
        dlogits = torch.empty_strided(s["z"].shape, s["z"].stride(), dtype=s["z"].dtype, device=s["z"].device)
        logp = torch.empty_like(s["old"])
        stats = B.marlaas_policy_loss(s["pool"], s["z"], s["targets"], s["seg"], s["old"], s["adv"], s["w"], ref_logp=s["ref"], dlogits=dlogits,
                                      logp=logp, clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=c["kl"], entropy_coef=c["entropy"],
                                      inv_temperature=INV_TEMPERATURE, grad_scale=GRAD_SCALE)
        return dict(dlogits=dlogits, logp=logp, stats=stats)
    B.marlaas_adapter_pool_adamw_compact_commit(s["pool"], s["tables"], seed=ADAM_SEED, **ADAM)
    out = {}
    for x, store in zip("AB", s["pool"].store()):
        m, v = B.marlaas_adamw_compact_state_export(s["pool"], s["state" + x])
        out.update({"theta" + x: s["theta" + x], "m" + x: m, "v" + x: v, "store" + x: store.view(-1)})
    return out


def run(state):
    if own:
        return _own_run(state)
    return {"advantages": _plain_advantages, "logprobs": _plain_logprobs, "loss": _plain_loss, "adamw": _plain_adamw}[state["case"]["op"]](state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "advantages":
        lens = _lengths(case)
        T, S = int(lens.sum()), len(lens)
        return dict(bytes=12 * T + 16 * S + 4 * case["groups"], flops=4 * T + 8 * S)
    if op in ("logprobs", "loss"):
        T, V, e = case["T"], case["V"], 4 if case["dtype"] == "f32" else 2
        read = (1 - case["ignored"]) * T
        if op == "logprobs":
            return dict(bytes=read * V * e + T * (8 + 4 * case["entropy"]), flops=read * V * (4 + 2 * case["entropy"]))
        return dict(bytes=read * V * e + T * V * e + T * (24 if case["kl"] else 20), flops=read * V * (9 + 3 * (case["entropy"] != 0)))
    n = sum(rows * cols for mats in _matrices(case) for _, _, _, rows, cols in mats)
    # gradient, master in and out, moments in and out, the store's bf16, and the moments' values
    return dict(bytes=n * (4 + 8 + 2 * 2 * (1 + 1 / 256) + 2 + 8), flops=16 * n)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _exact_advantages(s, case):
    r = s["rewards"].double().cpu().numpy()
    go, off = s["group_off"].cpu().numpy().astype(np.int64), s["off"].cpu().numpy().astype(np.int64)
    active = s["targets"].cpu().numpy() >= 0
    slot = s["slot"].cpu().numpy()
    seq_adv = np.zeros(len(r))
    for a, b in zip(go[:-1], go[1:]):
        if b > a:
            x = r[a:b]
            alike = np.all(x == x[0])
            mean = x[0] if alike else x.mean()
            sd = 0.0 if alike else np.sqrt(np.mean((x - mean) ** 2))
            seq_adv[a:b] = (x - mean) / (sd + ADV_EPS) if case["std"] else x - mean
    count = np.add.reduceat(active, off[:-1]).astype(np.float64) * (off[1:] > off[:-1])
    adv, weight = np.zeros(s["T"]), np.zeros(s["T"])
    for b in np.unique(slot):
        mine = np.flatnonzero(slot == b)
        tokens, used = count[mine].sum(), (count[mine] > 0).sum()
        for q in mine:
            if count[q]:
                weight[off[q]:off[q + 1]] = 1 / tokens if case["token_mean"] else 1 / (used * count[q])
                adv[off[q]:off[q + 1]] = seq_adv[q]
    put = lambda a: torch.from_numpy(a).to(DEV)     # noqa: E731
    return dict(seq_adv=put(seq_adv), adv=put(adv * active), weight=put(weight * active))


def _exact_rows(s, case, want_grad):
    z, tgt = s["z"], s["targets"]
    T, V = z.shape
    logp, H = torch.zeros(T, dtype=torch.float64, device=DEV), torch.zeros(T, dtype=torch.float64, device=DEV)
    grad = torch.zeros((T, V), dtype=torch.float64, device=DEV) if want_grad else None
    terms = torch.zeros((T, 8), dtype=torch.float64, device=DEV)
    tau = 1 / INV_TEMPERATURE
    for i in range(0, T, 128):
        rows = torch.arange(i, min(i + 128, T), device=DEV)
        rows = rows[tgt[rows] >= 0]
        if not len(rows):
            continue
        y = z[rows].double()
        # a mask of the type's lowest value times 1/tau leaves no probability, as minus infinity does
        y = torch.log_softmax((y - y.amax(1, keepdim=True)) / tau, 1)
        p = y.exp()
        a = tgt[rows].long()[:, None]
        lp = y.gather(1, a)[:, 0]
        h = -torch.special.xlogy(p, p).sum(1)
        logp[rows], H[rows] = lp, h
        if not want_grad:
            continue
        A, w = s["adv"][rows].double(), s["w"][rows].double()
        ratio = (lp - s["old"][rows].double()).exp()
        inside = torch.where(A >= 0, ratio <= 1 + CLIP_HIGH, ratio >= 1 - CLIP_LOW)
        pg = torch.where(inside, -ratio * A, -torch.where(A >= 0, 1 + CLIP_HIGH, 1 - CLIP_LOW) * A)
        slope = torch.where(inside, -ratio * A, torch.zeros_like(A))
        kl = torch.zeros_like(A)
        if case["kl"]:
            d = s["ref"][rows].double() - lp
            kl = d.exp() - d - 1
            slope = slope + case["kl"] * (1 - d.exp())
        g = -p * slope[:, None]
        g.scatter_add_(1, a, slope[:, None])
        if case["entropy"]:
            g += case["entropy"] * (torch.special.xlogy(p, p) + p * h[:, None])
        grad[rows] = g * (w * GRAD_SCALE / tau)[:, None]
        terms[rows] = torch.stack([w * (pg + case["kl"] * kl - case["entropy"] * h), w * pg, w * kl, w * h, w * ratio, w * ~inside, w, torch.ones_like(w)], 1)
    return logp, H, grad, terms


def _exact_loss(s, case):
    logp, _, grad, terms = _exact_rows(s, case, True)
    stats = torch.zeros((s["cap"] + 1, 8), dtype=torch.float64, device=DEV)
    off, slot = s["off"].tolist(), s["slot"].tolist()
    for a, b, t in zip(off[:-1], off[1:], slot):
        stats[t if t >= 0 else s["cap"]] += terms[a:b].sum(0)
    return dict(dlogits=grad, logp=logp, stats=stats)


def _exact_value(code, expo, bits):
    """Value of codes with `bits` exponent bits and 3 mantissa bits, the largest exponent being the block's."""
    code, lowest = code.long(), (expo.long() - (2 ** bits - 1)).clamp(min=0)[:, None]
    ex, man = code // 8 + lowest, code % 8
    # exponent field 0 holds the type's subnormals
    v = torch.where(ex > 0, (1 + man / 8.0) * torch.exp2(ex.double() - 127), (man / 8.0) * 2.0 ** -126)
    return torch.where(code > 0, v.double(), torch.zeros_like(v, dtype=torch.float64))


def _exact_round(x, u, bits, keep):
    """Positive x rounded to 3 mantissa bits by the uniform numbers u, on the grid of a block's `bits` exponent bits."""
    x = x.clamp(max=1.875 * 2.0 ** 127)
    top = x.amax(1, keepdim=True)
    man, ex = torch.frexp(top)                       # top = man 2^ex, man in [0.5, 1)
    biggest = torch.where(man > 0.9375, ex + 1, ex) - 1
    lowest = torch.clamp(biggest + 127 - (2 ** bits - 1), min=0) - 127
    ulp = torch.exp2((torch.frexp(x)[1] - 1).clamp(min=-126).double() - 3)
    r = torch.floor(x / ulp + u) * ulp
    least = torch.where(lowest >= -126, 1.125 * torch.exp2(lowest.double()), torch.full_like(top, 2.0 ** -129))
    return torch.where(r < least, torch.where(x > 0, least, torch.zeros_like(r)) if keep else torch.zeros_like(r), r)


def _exact_adamw(s, case):
    h, f, out = ADAM, lambda v: float(np.float32(v)), {}
    b1, b2 = f(h["beta1"]), f(h["beta2"])
    for x in ("A", "B"):
        st = s["state" + x]
        nb = st.shape[0]
        mc = st[:, :BLOCK]
        m = _exact_value(mc & 127, st[:, 2 * BLOCK], 4) * torch.where(mc >= 128, -1.0, 1.0)
        v = _exact_value(st[:, BLOCK:2 * BLOCK], st[:, 2 * BLOCK + 1], 5)
        g = f(h["grad_scale"]) * s["grad" + x].double().view(nb, BLOCK)
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        theta = s["theta" + x].double().view(nb, BLOCK)
        theta = theta - f(h["lr"]) * (m / (1 - b1 ** h["step"]) / (torch.sqrt(v / (1 - b2 ** h["step"])) + f(h["eps"])) + f(h["weight_decay"]) * theta)
        e = s["e" + x].view(nb, BLOCK)
        k = 0xFFFFFFFF
        e = ((e ^ (e >> 16)) * 0x9E3779B9) & k
        e = ((e ^ (e >> 15)) * 0xB504F333) & k
        e = e ^ (e >> 16)
        out["theta" + x] = theta.reshape(-1)
        out["m" + x] = (_exact_round(m.abs(), (e % 65536) / 65536.0, 4, False) * torch.sign(m)).reshape(-1)
        out["v" + x] = _exact_round(v, (e // 65536) / 65536.0, 5, True).reshape(-1)
        store = torch.zeros(s["store" + x].numel(), dtype=torch.float64, device=DEV)
        store[s["at" + x]] = theta.reshape(-1)
        out["store" + x] = store[:-1]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "advantages":
        return _exact_advantages(s, case)
    if case["op"] == "adamw":
        return _exact_adamw(s, case)
    if case["op"] == "loss":
        return _exact_loss(s, case)
    logp, H, _, _ = _exact_rows(s, case, False)
    return dict(logp=logp, entropy=H) if case["entropy"] else dict(logp=logp)
