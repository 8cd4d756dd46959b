"""Measured cases of the training-step operators around the adapted layers: cross entropy from hidden states without kept
logits, dropout in the adapters, and layer norm with parameters of each tenant.

`run` computes a case either in its plain form (elementary torch operations in 32 bits, `own = False`) or through the
library's calls (`own = True`) on the same inputs.  `exact` gives the definition's values in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
INV_TEMPERATURE, GRAD_SCALE = 1.0 / 0.9, 0.5
ALPHA = 16.0
SEED, OFFSET = 0x5DEECE66D1234567, 41       # of the dropout masks
RANKS = (8, 16, 32, 64)
RATES = (0.05, 0.1, 0.0, 0.2)               # tenants' dropout rates, in turn
EPS = 1e-5


def listed():
    return [
        # log-probabilities of the tokens that one decode step of a small model sampled
        dict(name="head logp decode", op="head", T=32, d=1024, V=32768, grad=False, ignored=0.0, tenants=8),
        # reference-policy pass over a training batch, an odd vocabulary
        dict(name="head logp odd", op="head", T=1021, d=2048, V=50001, grad=False, ignored=0.25, tenants=8),
        # loss and gradient of a small batch: launches count
        dict(name="head loss small", op="head", T=64, d=512, V=8000, grad=True, ignored=0.1, tenants=4),
        # a training batch over a large vocabulary, a quarter prompt tokens
        dict(name="head loss large", op="head", T=4096, d=4096, V=131072, grad=True, ignored=0.25, tenants=10),
        # one tenant's few tokens through a small projection
        dict(name="dropout forward small", op="dropout", back=False, T=100, K=512, N=512, tenants=1, rank=8),
        # 32 tenants' training batch through a square projection of a 7B-shaped model
        dict(name="dropout forward large", op="dropout", back=False, T=8192, K=4096, N=4096, tenants=32, rank=16),
        # mixed ranks, sizes that end inside a tile
        dict(name="dropout backward odd", op="dropout", back=True, T=1000, K=1544, N=1032, tenants=5, rank=0),
        dict(name="dropout backward large", op="dropout", back=True, T=8192, K=4096, N=4096, tenants=32, rank=16),
        # the norm of a decode step
        dict(name="norm forward decode", op="norm", back=False, T=64, d=1024, tenants=8, rms=True),
        # every position of a long training batch
        dict(name="norm forward large", op="norm", back=False, T=65536, d=4096, tenants=32, rms=False),
        # an odd batch, RMS norm
        dict(name="norm backward odd", op="norm", back=True, T=1021, d=1000, tenants=5, rms=True),
        dict(name="norm backward large", op="norm", back=True, T=32768, d=5120, tenants=32, rms=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["head", "head", "dropout", "dropout", "norm", "norm"])
    if op == "head":
        return dict(op=op, T=_log_int(rng, 1, 4096), d=8 * _log_int(rng, 16, 512), V=_log_int(rng, 1000, 131072), grad=rng.random() < 0.5,
                    ignored=rng.choice([0.0, 0.1, 0.25, 0.5]), tenants=rng.randint(1, 32))
    if op == "dropout":
        return dict(op=op, back=rng.random() < 0.5, T=_log_int(rng, 1, 8192), K=8 * _log_int(rng, 16, 512), N=8 * _log_int(rng, 16, 512),
                    tenants=_log_int(rng, 1, 32), rank=rng.choice([0, 5, 8, 16, 32]))
    back, d = rng.random() < 0.5, 8 * _log_int(rng, 8, 640)
    return dict(op=op, back=back, T=min(_log_int(rng, 1, 65536), (1 << 27) // d), d=d, tenants=_log_int(rng, 1, 32), rms=rng.random() < 0.5)


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _batch(case, seed):
    """Sequences of about 128 tokens, tenants in any order, some on the base model alone: offsets, slots, a slot per token."""
    r = np.random.RandomState(seed % (1 << 31))
    T, n = case["T"], max(1, case["T"] // 128)
    off = np.unique(np.concatenate([[0], r.randint(0, T + 1, n - 1), [T]]))
    slot = r.randint(0 if len(off) < 4 else -1, case["tenants"], len(off) - 1)
    return _i32(off), _i32(slot), torch.from_numpy(np.repeat(slot, np.diff(off))).to(DEV)


def _own_pool(s, d_in, d_out, rank):
    from paper_2605_08527_b200 import binding
    s["pool"] = binding.AdapterPool(d_in, d_out, rank, s["case"]["tenants"], device=DEV)
    s["seg"] = binding.Segments(s["off"], s["slot"])
    return binding


def _prepare_head(case, seed):
    T, d, V, g = case["T"], case["d"], case["V"], _gen(seed)
    ld = -(-V // 8) * 8                     # rows on 16-byte boundaries
    W = torch.empty((d, ld), dtype=torch.bfloat16, device=DEV).normal_(0.0, 2.0 / math.sqrt(d), generator=g)[:, :V]
    tgt = torch.randint(0, V, (T,), generator=g, device=DEV)
    # hidden states that lean to their targets, some much and some not at all
    x = torch.randn((T, d), generator=g, device=DEV) + 2.5 * torch.rand((T, 1), generator=g, device=DEV) * W[:, tgt].float().T
    ignored = torch.rand(T, generator=g, device=DEV) < case["ignored"]
    # signed weights, as of advantages that normalise a policy update
    w = torch.randn(T, generator=g, device=DEV)
    off, slot, tok = _batch(case, seed)
    s = dict(case=case, x=x.bfloat16(), W=W, targets=torch.where(ignored, -1, tgt).to(torch.int32), w=w, off=off, slot=slot, tok=tok)
    if own:
        _own_pool(s, 64, 64, 8)
        s["dx"] = torch.empty_like(s["x"]) if case["grad"] else None
    return s


def _ranks(case):
    return [case["rank"] or RANKS[t % 4] for t in range(case["tenants"])]


def _prepare_dropout(case, seed):
    T, K, N, n, g = case["T"], case["K"], case["N"], case["tenants"], _gen(seed)
    ranks = _ranks(case)
    RP = -(-max(ranks) // 16) * 16
    live = torch.arange(RP, device=DEV) < torch.tensor(ranks, device=DEV)[:, None]             # [n][RP]
    x = torch.randn((T, K), generator=g, device=DEV).bfloat16()
    W = (torch.randn((K, N), generator=g, device=DEV) / math.sqrt(K)).bfloat16()
    A = (torch.randn((n, K, RP), generator=g, device=DEV) / math.sqrt(K) * live[:, None, :]).bfloat16()
    B = (0.05 * torch.randn((n, RP, N), generator=g, device=DEV) * live[:, :, None]).bfloat16()
    rates = torch.tensor([RATES[t % 4] for t in range(n)], device=DEV)
    off, slot, tok = _batch(case, seed)
    s = dict(case=case, x=x, W=W, A=A, B=B, RP=RP, rates=rates, off=off, slot=slot, tok=tok,
             scale=torch.tensor([np.float32(ALPHA) / np.float32(r) for r in ranks], device=DEV))
    if case["back"]:
        # the layer's training step has the gradient of its output and the h that its forward pass kept
        s["dy"] = torch.randn((T, N), generator=g, device=DEV).bfloat16()
        s["h"] = _own_columns(s, torch.where(_keep(s), x.float(), 0.0) @ _wide(A.float()))
    if own:
        B_ = _own_pool(s, K, N, max(ranks))
        for t, r in enumerate(ranks):
            B_.marlaas_adapter_pool_register(s["pool"], 1000 + t, 0, r, ALPHA, A[t, :, :r].contiguous(), B[t, :r].contiguous())
        if case["back"]:
            s["dx"] = torch.empty_like(x)
            # the tenants' gradients one after another in a buffer for all
            s["allA"], s["allB"] = torch.empty(K * sum(ranks), device=DEV), torch.empty(N * sum(ranks), device=DEV)
            s["dA"] = [a.view(K, -1) for a in s["allA"].split([K * r for r in ranks])]
            s["dB"] = [b.view(-1, N) for b in s["allB"].split([N * r for r in ranks])]
        else:
            s["y"], s["h"] = torch.empty((T, N), dtype=torch.bfloat16, device=DEV), torch.empty((T, RP), device=DEV)
    return s


def _prepare_norm(case, seed):
    T, d, n, g = case["T"], case["d"], case["tenants"], _gen(seed)
    # a residual stream: tokens of different sizes, channels with offsets, a few channels much larger than the rest
    size = torch.exp(0.5 * torch.randn((T, 1), generator=g, device=DEV))
    channel = torch.where(torch.rand(d, generator=g, device=DEV) < 0.01, 8.0, 1.0)
    shift = 0.3 * torch.randn(d, generator=g, device=DEV)
    x = torch.randn((T, d), generator=g, device=DEV).add_(shift).mul_(size).mul_(channel).bfloat16()
    off, slot, tok = _batch(case, seed)
    s = dict(case=case, x=x, off=off, slot=slot, tok=tok, row=torch.where(tok < 0, n, tok),
             gain=1.0 + 0.1 * torch.randn((n + 1, d), generator=g, device=DEV), bias=0.1 * torch.randn((n + 1, d), generator=g, device=DEV))
    if case["back"]:
        s["dy"] = (torch.randn((T, d), generator=g, device=DEV) * 0.01).bfloat16()
        s["mean"], s["rstd"] = _moments(x.float(), case["rms"])
    if own:
        _own_pool(s, 64, 64, 8)
        if case["back"]:
            s["dx"], s["dgain"], s["dbias"] = torch.empty_like(x), torch.empty_like(s["gain"]), torch.empty_like(s["bias"])
        else:
            s["y"], s["mean"], s["rstd"] = torch.empty_like(x), torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    return s


def prepare(case, seed):
    return {"head": _prepare_head, "dropout": _prepare_dropout, "norm": _prepare_norm}[case["op"]](case, seed)


# ---- plain forms -------------------------------------------------------------------------------------------------------

def _plain_head(s, case):
    T, n = case["T"], case["tenants"]
    active = s["targets"] >= 0
    y = torch.where(active, s["targets"], 0).long()[:, None]
    z = (s["x"].float() @ s["W"].float()).mul_(INV_TEMPERATURE)
    top = z.amax(1, keepdim=True)
    zy = torch.gather(z, 1, y)
    p = z.sub_(top).exp_()
    total = p.sum(1, keepdim=True)
    logp = torch.where(active, (zy - top - torch.log(total))[:, 0], 0.0)
    w = torch.where(active, s["w"], 0.0)
    terms = torch.stack([-w * logp, w, -logp, active.float()], 1).double()
    bucket = torch.where(s["tok"] < 0, n, s["tok"]) == torch.arange(n + 1, device=DEV)[:, None]
    out = dict(logp=logp, stats=(bucket.double() @ terms).float())
    if case["grad"]:
        p.div_(total).scatter_add_(1, y, torch.full_like(zy, -1.0))
        out["dx"] = ((p * (w * (GRAD_SCALE * INV_TEMPERATURE))[:, None]) @ s["W"].float().T).bfloat16()
    return out


def _product(a, b):
    """High and low 32 bits of a product of two 32-bit numbers held in 64."""
    p = a * b
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _keep(s):
    """[T][K]: the elements of x that dropout keeps.  Philox-4x32 of seven rounds (Salmon, Moraes, Dror and Shaw, 2011) with the
    counter (column / 8, token, offset) and the seed as its key gives eight columns 16 bits each; those below a tenant's rate
    times 65536 are dropped."""
    T, K = s["x"].shape
    c0 = torch.arange(-(-K // 8), device=DEV).expand(T, -1)
    c1 = torch.arange(T, device=DEV)[:, None]
    c2, c3 = torch.tensor(OFFSET & 0xFFFFFFFF, device=DEV), torch.tensor(OFFSET >> 32, device=DEV)
    k0, k1 = SEED & 0xFFFFFFFF, SEED >> 32
    for _ in range(7):
        h0, l0 = _product(c0, 0xD2511F53)
        h1, l1 = _product(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([w.expand(T, -1) for w in (c0, c1, c2, c3)], 2)
    bits = torch.stack([words & 0xFFFF, words >> 16], 3).view(T, -1)[:, :K]
    return bits >= _threshold(s)[s["tok"].clamp(min=0)][:, None]


def _threshold(s):
    return torch.round(s["rates"].double() * 65536).long()


def _wide(a):
    """The tenants' A [n][K][RP] side by side, [K][n RP]."""
    return a.permute(1, 0, 2).reshape(a.shape[1], -1)


def _own_columns(s, h):
    """[T][RP]: of the products with all tenants' matrices the token's own; 0 on the base model."""
    h = h.view(h.shape[0], -1, s["RP"])[torch.arange(h.shape[0], device=DEV), s["tok"].clamp(min=0)]
    return torch.where(s["tok"][:, None] >= 0, h, 0.0)


def _spread(s, h, f):
    """[T][n RP]: a token's values times its tenant's factor in the columns of its tenant, zeros elsewhere."""
    mine = s["tok"][:, None] == torch.arange(s["case"]["tenants"], device=DEV)
    return (h[:, None, :] * (mine * f)[:, :, None]).view(h.shape[0], -1)


def _plain_dropout(s, case):
    keep, x, W, n = _keep(s), s["x"].float(), s["W"].float(), case["tenants"]
    f = s["scale"] * (65536.0 / (65536.0 - _threshold(s).float()))       # alpha / r / (1 - rate)
    A, B = _wide(s["A"].float()), s["B"].float().view(-1, case["N"])
    xd = torch.where(keep, x, 0.0)
    if not case["back"]:
        h = _own_columns(s, xd @ A)
        return dict(y=(x @ W + _spread(s, h, f) @ B).bfloat16(), h=h)
    dy = s["dy"].float()
    g = _spread(s, _own_columns(s, dy @ B.T), f)
    dA = (xd.T @ g).view(case["K"], n, s["RP"])
    dB = (_spread(s, s["h"], f).T @ dy).view(n, s["RP"], case["N"])
    return dict(dx=(dy @ W.T + torch.where(keep, g @ A.T, 0.0)).bfloat16(),
                dA=torch.cat([dA[:, t, :r].reshape(-1) for t, r in enumerate(_ranks(case))]), dB=torch.cat([dB[t, :r].reshape(-1) for t, r in enumerate(_ranks(case))]))


def _moments(x, rms):
    mean = torch.zeros_like(x[:, 0]) if rms else x.mean(1)
    return mean, torch.rsqrt((x - mean[:, None]).square().mean(1) + EPS)


def _plain_norm(s, case):
    x, n, rms = s["x"].float(), case["tenants"], case["rms"]
    if not case["back"]:
        mean, rstd = _moments(x, rms)
        y = (x - mean[:, None]) * rstd[:, None] * s["gain"][s["row"]]
        return dict(y=(y if rms else y + s["bias"][s["row"]]).bfloat16(), mean=mean, rstd=rstd)
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * rstd
    a = dy * s["gain"][s["row"]]
    dx = a - xh * (a * xh).mean(1, keepdim=True)
    if not rms:
        dx -= a.mean(1, keepdim=True)
    mine = (s["row"] == torch.arange(n + 1, device=DEV)[:, None]).double()      # long sums
    out = dict(dx=(rstd * dx).bfloat16(), dgain=(mine @ (dy * xh).double()).float())
    return out if rms else out | dict(dbias=(mine @ dy.double()).float())


# ---- one pass ----------------------------------------------------------------------------------------------------------

def _own_head(s, case):
    from paper_2605_08527_b200 import binding as B
    logp, stats = B.marlaas_head_cross_entropy(s["pool"], s["x"], s["W"], s["targets"], s["seg"], weight=s["w"], dx=s["dx"],
                                               inv_temperature=INV_TEMPERATURE, grad_scale=GRAD_SCALE)
    return dict(logp=logp, stats=stats, dx=s["dx"]) if case["grad"] else dict(logp=logp, stats=stats)


def _own_dropout(s, case):
    from paper_2605_08527_b200 import binding as B
    drop = dict(rates=s["rates"], seed=SEED, offset=OFFSET)
    if not case["back"]:
        B.marlaas_lora_forward_dropout(s["pool"], s["x"], s["W"], s["seg"], y=s["y"], h_save=s["h"], **drop)
        return dict(y=s["y"], h=s["h"])
    B.marlaas_lora_backward_dropout(s["pool"], s["x"], s["W"], s["dy"], s["seg"], dx=s["dx"], dA=s["dA"], dB=s["dB"], h_saved=s["h"], **drop)
    return dict(dx=s["dx"], dA=s["allA"], dB=s["allB"])


def _own_norm(s, case):
    from paper_2605_08527_b200 import binding as B
    rms = case["rms"]
    flags = B.MARLAAS_FLAG_RMS_NORM if rms else 0
    if not case["back"]:
        B.marlaas_layer_norm(s["pool"], s["x"], s["seg"], s["gain"], None if rms else s["bias"], eps=EPS, y=s["y"], mean=s["mean"],
                             rstd=s["rstd"], flags=flags)
        return dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
    B.marlaas_layer_norm_backward(s["pool"], s["x"], s["dy"], s["seg"], s["gain"], s["mean"], s["rstd"], dx=s["dx"], dgain=s["dgain"],
                                  dbias=None if rms else s["dbias"], flags=flags)
    out = dict(dx=s["dx"], dgain=s["dgain"])
    return out if rms else out | dict(dbias=s["dbias"])


def run(state):
    case = state["case"]
    if own:
        return {"head": _own_head, "dropout": _own_dropout, "norm": _own_norm}[case["op"]](state, case)
    return {"head": _plain_head, "dropout": _plain_dropout, "norm": _plain_norm}[case["op"]](state, case)


def work(case):
    T, n = case["T"], case["tenants"]
    if case["op"] == "head":
        d, V, live = case["d"], case["V"], T * (1 - case["ignored"])
        passes = 2 if case["grad"] else 1
        return {"bytes": 2 * (live * d + d * V) + 12 * T + 16 * (n + 1) + (2 * T * d if case["grad"] else 0), "flops": passes * 2 * live * d * V}
    if case["op"] == "norm":
        d = case["d"]
        tables = 4 * (n + 1) * d * (1 if case["rms"] else 2)
        return {"bytes": (6 if case["back"] else 4) * T * d + 8 * T + tables * (2 if case["back"] else 1), "flops": (16 if case["back"] else 8) * T * d}
    K, N, r = case["K"], case["N"], sum(_ranks(case)) / n
    adapters = 2 * sum(_ranks(case)) * (K + N)
    if not case["back"]:
        return {"bytes": 2 * (T * K + K * N + T * N) + adapters + 4 * T * r, "flops": 2 * T * (K * N + r * (K + N))}
    return {"bytes": 2 * (2 * T * K + K * N + T * N) + 3 * adapters + 4 * T * r, "flops": 2 * T * (K * N + 2 * r * (K + N))}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------

def _exact_head(s, case):
    logp = torch.zeros(case["T"], dtype=torch.float64, device=DEV)
    dx = torch.zeros(s["x"].shape, dtype=torch.float64, device=DEV)
    W, it = s["W"].double(), float(np.float32(INV_TEMPERATURE))
    for rows in torch.nonzero(s["targets"] >= 0)[:, 0].split(512):
        z = (s["x"][rows].double() @ W) * it
        y = s["targets"][rows].long()
        ls = torch.log_softmax(z, 1)
        logp[rows] = ls[torch.arange(len(rows), device=DEV), y]
        if case["grad"]:
            q = torch.softmax(z, 1)
            q[torch.arange(len(rows), device=DEV), y] -= 1
            dx[rows] = (GRAD_SCALE * it * s["w"][rows].double())[:, None] * (q @ W.T)
    stats = torch.zeros((case["tenants"] + 1, 4), dtype=torch.float64, device=DEV)
    on, w = (s["targets"] >= 0).double(), s["w"].double()
    to = torch.where(s["tok"] < 0, case["tenants"], s["tok"])
    stats.index_add_(0, to, torch.stack([-w * logp, w * on, -logp, on], 1))
    return dict(logp=logp, stats=stats, dx=dx) if case["grad"] else dict(logp=logp, stats=stats)


def _exact_keep(case, s):
    """The same masks from the generator's definition on unsigned numbers, on the host."""
    T, K = s["x"].shape
    m32, lo = np.uint64(0xFFFFFFFF), np.uint64(32)
    ctr = [np.tile(np.arange(-(-K // 8), dtype=np.uint64), (T, 1)), np.repeat(np.arange(T, dtype=np.uint64)[:, None], -(-K // 8), 1),
           np.uint64(OFFSET) & m32, np.uint64(OFFSET) >> lo]
    for i in range(7):
        key = [np.uint64((SEED + i * 0x9E3779B9) % 2 ** 32), np.uint64((SEED // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32)]
        a, b = np.uint64(0xD2511F53) * ctr[0], np.uint64(0xCD9E8D57) * ctr[2]
        ctr = [(b >> lo) ^ ctr[1] ^ key[0], b & m32, (a >> lo) ^ ctr[3] ^ key[1], a & m32]
    words = np.stack([np.broadcast_to(c, ctr[0].shape) for c in ctr], -1).astype("<u4")
    bits = np.ascontiguousarray(words).view("<u2").reshape(T, -1)[:, :K]
    limit = np.rint(s["rates"].cpu().numpy().astype(np.float64) * 65536)
    tok = s["tok"].cpu().numpy()
    return torch.from_numpy((bits >= limit[np.maximum(tok, 0)][:, None])).to(DEV)


def _exact_dropout(s, case):
    keep, ranks, K, N = _exact_keep(case, s), _ranks(case), case["K"], case["N"]
    x, W = s["x"].double(), s["W"].double()
    h = torch.zeros((case["T"], s["RP"]), dtype=torch.float64, device=DEV)
    base = s["dy"].double() @ W.T if case["back"] else x @ W
    dA, dB = [], []
    for t, r in enumerate(ranks):
        i = torch.nonzero(s["tok"] == t)[:, 0]
        A, B = s["A"][t, :, :r].double(), s["B"][t, :r].double()
        limit = float(np.rint(float(s["rates"][t]) * 65536))
        f = float(s["scale"][t]) * 65536 / (65536 - limit)
        xd = x[i] * keep[i]
        if not case["back"]:
            h[i, :r] = xd @ A
            base[i] += f * (xd @ A) @ B
            continue
        dy = s["dy"][i].double()
        g = f * (dy @ B.T)
        base[i] += keep[i] * (g @ A.T)
        dA.append((xd.T @ g).reshape(-1))
        dB.append((f * s["h"][i, :r].double().T @ dy).reshape(-1))
    return dict(dx=base, dA=torch.cat(dA), dB=torch.cat(dB)) if case["back"] else dict(y=base, h=h)


def _exact_norm(s, case):
    T, d, rms = case["T"], case["d"], case["rms"]
    rows, n = s["row"], case["tenants"]
    if not case["back"]:
        x = s["x"].double()
        mean = torch.zeros(T, dtype=torch.float64, device=DEV) if rms else x.sum(1) / d
        x -= mean[:, None]
        rstd = 1 / torch.sqrt((x * x).sum(1) / d + EPS)
        y = x.mul_(rstd[:, None]).mul_(s["gain"][rows])
        return dict(y=y if rms else y.add_(s["bias"][rows]), mean=mean, rstd=rstd)
    dx = torch.empty((T, d), dtype=torch.float64, device=DEV)
    dgain, dbias = (torch.zeros((n + 1, d), dtype=torch.float64, device=DEV) for _ in range(2))
    for i in torch.arange(T, device=DEV).split(8192):
        dy, r = s["dy"][i].double(), s["rstd"][i, None].double()
        xh = (s["x"][i].double() - s["mean"][i, None].double()) * r
        dgain.index_add_(0, rows[i], dy * xh)
        dbias.index_add_(0, rows[i], dy)
        a = dy * s["gain"][rows[i]].double()
        dx[i] = r * (a - xh * ((a * xh).sum(1, keepdim=True) / d) - (0 if rms else a.sum(1, keepdim=True) / d))
    out = dict(dx=dx, dgain=dgain)
    return out if rms else out | dict(dbias=dbias)


def exact(case, seed):
    return {"head": _exact_head, "dropout": _exact_dropout, "norm": _exact_norm}[case["op"]](prepare(case, seed), case)
