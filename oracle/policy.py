"""Plain float64 definitions of the policy update's operators (numpy, row by row; shares no code with the GPU path):
group-relative advantages and token weights, token log-probabilities, the clipped policy loss with its gradient, and AdamW
with 8-bit moments."""
import math

import numpy as np


def group_advantages(seg_offsets, seg_slot, rewards, group_offsets, targets, eps, token_mean=False, no_std=False):
    S, T = len(seg_slot), len(targets)
    r = np.asarray(rewards, dtype=np.float64)
    seq_adv, adv, weight = np.zeros(S), np.zeros(T), np.zeros(T)
    for a, b in zip(group_offsets[:-1], group_offsets[1:]):
        if b <= a:
            continue
        d = r[a:b] - r[a]
        d = d - d.mean()
        sd = math.sqrt(float((d * d).mean()))
        for i in range(a, b):
            seq_adv[i] = d[i - a] if no_std else (0.0 if d[i - a] == 0 else d[i - a] / (sd + eps))
    active = np.asarray(targets) >= 0
    n = [int(active[seg_offsets[s]:seg_offsets[s + 1]].sum()) for s in range(S)]
    for s in range(S):
        if not n[s]:
            continue
        mine = [q for q in range(S) if seg_slot[q] == seg_slot[s] and n[q]]
        w = 1.0 / sum(n[q] for q in mine) if token_mean else 1.0 / (len(mine) * n[s])
        for i in range(seg_offsets[s], seg_offsets[s + 1]):
            if active[i]:
                adv[i], weight[i] = seq_adv[s], w
    return seq_adv, adv, weight


def _distribution(z, inv_temperature):
    """log-probabilities of one row of logits, or None if no logit is finite."""
    z = np.asarray(z, dtype=np.float64)
    m = z.max()
    if m == -math.inf:
        return None
    y = (z - m) * inv_temperature
    return y - math.log(np.exp(y).sum())


def token_logprobs(logits, targets, inv_temperature):
    T = len(targets)
    logp, entropy = np.zeros(T), np.zeros(T)
    for i in range(T):
        y = _distribution(logits[i], inv_temperature) if targets[i] >= 0 else None
        if y is None:
            continue
        p = np.exp(y)
        logp[i] = y[targets[i]]
        entropy[i] = -sum(p[p > 0] * y[p > 0])
    return logp, entropy


def policy_loss(logits, targets, tok_slot, n_slots, old_logp, ref_logp, adv, weight, clip_low, clip_high, kl_coef=0.0,
                entropy_coef=0.0, inv_temperature=1.0, grad_scale=1.0):
    """(stats [n_slots + 1][8], dlogits [T][V], logp [T])."""
    T, V = np.shape(logits)
    stats, grad, logp = np.zeros((n_slots + 1, 8)), np.zeros((T, V)), np.zeros(T)
    for i in range(T):
        y = _distribution(logits[i], inv_temperature) if targets[i] >= 0 else None
        if y is None:
            continue
        logp[i] = y[targets[i]]
        w, A = float(weight[i]), float(adv[i])
        if w == 0:
            continue
        p = np.exp(y)
        on = p > 0
        H = -float((p[on] * y[on]).sum())
        ratio = math.exp(logp[i] - float(old_logp[i]))
        unclipped, clipped = ratio * A, min(max(ratio, 1 - clip_low), 1 + clip_high) * A
        is_clipped = clipped < unclipped
        pg = -min(unclipped, clipped)
        slope, kl = (0.0 if is_clipped else -unclipped), 0.0
        if kl_coef:
            d = float(ref_logp[i]) - logp[i]
            kl = math.exp(d) - d - 1
            slope += kl_coef * (1 - math.exp(d))
        dy = np.zeros(V)                    # by log-softmax's outputs, then through it
        g = -p * slope
        g[targets[i]] += slope
        dy[on] = entropy_coef * p[on] * (y[on] + H)
        grad[i] = grad_scale * w * inv_temperature * (g + dy)
        b = tok_slot[i] if tok_slot[i] >= 0 else n_slots
        stats[b] += [w * (pg + kl_coef * kl - entropy_coef * H), w * pg, w * kl, w * H, w * ratio, w * is_clipped, w, 1.0]
    return stats, grad, logp


# ---- AdamW with 8-bit moments: the format of marlaas.h in floating-point terms ----

BLOCK, STATE_BLOCK = 256, 528


def _mix(x):
    x &= 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xB504F333) & 0xFFFFFFFF
    return x ^ (x >> 16)


def random_bits(n, seed, step, tenant, part, matrix):
    """The 32 random bits of each of a matrix's n elements: low half for m, high half for v."""
    k = 0
    for word in (seed & 0xFFFFFFFF, seed >> 32, step & 0xFFFFFFFF, step >> 32, tenant & 0xFFFFFFFF, tenant >> 32, 2 * part + matrix):
        k = _mix((k + 0x9E3779B9) ^ word)
    x = (np.arange(n, dtype=np.uint64) + np.uint64(k)) & np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x9E3779B9)) & np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xB504F333)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def _lowest(top, orders):
    """The fp32 exponent field where a block's codes begin, from the field of its largest value."""
    return max(top - orders, 0)


def decode_state(state, n):
    """(m, v) in float64 of a state of n elements."""
    blocks = np.asarray(state, dtype=np.uint8).reshape(-1, STATE_BLOCK)
    m, v = np.zeros(len(blocks) * BLOCK), np.zeros(len(blocks) * BLOCK)
    for b, blk in enumerate(blocks):
        for out, codes, orders, top in ((m, blk[:BLOCK], 15, int(blk[512])), (v, blk[BLOCK:2 * BLOCK], 31, int(blk[513]))):
            c = codes.astype(np.int64)
            mag = c & 127 if orders == 15 else c
            field = _lowest(top, orders) + mag // 8
            x = np.where(field > 0, (1 + (mag % 8) / 8.0) * 2.0 ** (field - 127.0), (mag % 8) / 8.0 * 2.0 ** -126)
            x = np.where(mag > 0, x, 0.0)
            out[b * BLOCK:(b + 1) * BLOCK] = np.where((c >= 128) & (orders == 15), -x, x)
    return m[:n], v[:n]


def held_moments(state, n):
    """(m, v) that a step starts from.  A v of 0 in a block with an m of 1 or more stands for a square that has left fp32's
    range (a positive v never becomes 0): both start anew from 0."""
    m, v = decode_state(state, n)
    large = np.repeat(np.asarray(state, dtype=np.uint8).reshape(-1, STATE_BLOCK)[:, 512] >= 127, BLOCK)[:n]
    return np.where((v == 0) & large, 0.0, m), v


def encode_state(m, v, bits):
    """The state that stands for the moments rounded with the given random bits."""
    n = len(m)
    nb = -(-n // BLOCK)
    state = np.zeros((nb, STATE_BLOCK), dtype=np.uint8)
    for b in range(nb):
        lo, hi = b * BLOCK, min(n, (b + 1) * BLOCK)
        r = np.asarray(bits[lo:hi], dtype=np.uint64).astype(np.int64)
        for k, (x, orders, rnd) in enumerate(((m, 15, r & 0xFFFF), (v, 31, r >> 16))):
            x = np.asarray(x[lo:hi], dtype=np.float64)
            mag = np.where(np.isfinite(x), np.minimum(np.abs(x), 1.875 * 2.0 ** 127), 0.0)
            # units of 1/8 of a binary order: code number of the fp32 grid with 3 mantissa bits, rounded up or down
            ex = np.frexp(np.where(mag > 0, mag, 1.0))[1] - 1
            ex = np.maximum(ex, -126)
            code = np.floor(mag / 2.0 ** (ex - 3.0) + rnd / 65536.0).astype(np.int64) + (ex + 127) * 8 - 8
            small = np.where(ex == -126, mag, 0.0)
            code = np.where(ex == -126, np.floor(small / 2.0 ** -129 + rnd / 65536.0).astype(np.int64), code)
            code = np.where(mag > 0, code, 0)
            largest = float(mag.max()) if len(mag) else 0.0
            le = max(int(np.frexp(largest)[1]) - 1, -126) if largest > 0 else -127
            top = 0 if largest == 0 else int(np.ceil(largest / 2.0 ** (le - 3.0))) + (le + 127) * 8 - 8
            if 0 < largest < 2.0 ** -126:
                top = int(np.ceil(largest / 2.0 ** -129))
            E = top // 8
            code = code - 8 * _lowest(E, orders)
            code = np.where(mag > 0, np.maximum(code, 0 if k == 0 else 1), 0)
            if k == 0:
                code = code + np.where(x < 0, 128, 0)
            state[b, k * BLOCK:k * BLOCK + hi - lo] = code
            state[b, 512 + k] = E
    return state.reshape(-1)


def adamw_compact_step(theta, grad, state, bits, lr, beta1, beta2, eps, weight_decay, grad_scale, step):
    """(theta, m, v, state) after a step; m, v are the new moments before they are rounded into the state."""
    n = len(theta)
    f = lambda x: float(np.float32(x))      # noqa: E731 - the call's fp32 hyper-parameters
    m, v = held_moments(state, n)
    g = f(grad_scale) * np.asarray(grad, dtype=np.float64)
    m = f(beta1) * m + (1 - f(beta1)) * g
    v = f(beta2) * v + (1 - f(beta2)) * g * g
    mh, vh = m / (1 - f(beta1) ** step), v / (1 - f(beta2) ** step)
    theta = np.asarray(theta, dtype=np.float64)
    theta = theta - f(lr) * (mh / (np.sqrt(vh) + f(eps)) + f(weight_decay) * theta)
    return theta, m, v, encode_state(m, v, bits)
