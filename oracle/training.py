"""Plain float64 definitions of the operators around a training step's layers (numpy; shares no code with the GPU path): layer
norm with parameters per tenant, dropout in the adapters, cross entropy of a vocabulary head."""
import numpy as np


# ---- layer norm ----

def layer_norm(x, rows, gain, bias, eps, rms=False):
    """(y, mean, rstd); rows[i] is the row of gain and bias that token i uses."""
    x = np.asarray(x, dtype=np.float64)
    mean = np.zeros(len(x)) if rms else x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / np.sqrt((c * c).mean(1) + eps)
    y = c * rstd[:, None] * np.asarray(gain, dtype=np.float64)[rows]
    if bias is not None:
        y = y + np.asarray(bias, dtype=np.float64)[rows]
    return y, mean, rstd


def layer_norm_backward(x, dy, rows, gain, mean, rstd, rms=False):
    """(dx, dgain, dbias)."""
    x, dy, gain = (np.asarray(v, dtype=np.float64) for v in (x, dy, gain))
    rstd = np.asarray(rstd, dtype=np.float64)[:, None]
    xh = x * rstd if rms else (x - np.asarray(mean, dtype=np.float64)[:, None]) * rstd
    a = dy * gain[rows]
    dx = a - xh * (a * xh).mean(1, keepdims=True)
    if not rms:
        dx = dx - a.mean(1, keepdims=True)
    dgain, dbias = np.zeros(gain.shape), np.zeros(gain.shape)
    np.add.at(dgain, rows, dy * xh)
    np.add.at(dbias, rows, dy)
    return rstd * dx, dgain, dbias


# ---- dropout ----

def philox(counter, key, rounds=7):
    """Philox-4x32 (Salmon, Moraes, Dror and Shaw, 2011): four 32-bit words for a counter of four words and a key of two."""
    c, k = [int(v) for v in counter], [int(v) for v in key]
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def threshold(rate):
    """Of 65536: how many of the 16-bit numbers drop an element; a rate that is not positive (or NaN) drops none."""
    rate = np.float64(np.float32(rate))
    return int(np.rint(min(rate, 1.0) * 65536)) if rate > 0 else 0


def dropout_keep(tok_slot, width, rates, seed, offset):
    """[T][width] of truth values; tokens of slot -1 keep everything."""
    T = len(tok_slot)
    keep = np.ones((T, width), dtype=bool)
    for i in range(T):
        limit = threshold(rates[tok_slot[i]]) if tok_slot[i] >= 0 else 0
        if limit == 0:
            continue
        bits = []
        for c in range(-(-width // 8)):
            for w in philox((c, i, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32)):
                bits += [w & 0xFFFF, w >> 16]
        keep[i] = np.array(bits[:width]) >= limit
    return keep


def dropout_factor(scale, rate):
    """s / (1 - rate), of the rate as it is rounded; 0 where everything is dropped."""
    limit = threshold(rate)
    return scale * 65536.0 / (65536 - limit) if limit < 65536 else 0.0


def dropout_forward(x, W, tok_slot, A, B, scale, rates, keep):
    """(y, h per token as a list)."""
    x, W = np.asarray(x, dtype=np.float64), np.asarray(W, dtype=np.float64)
    y, h = x @ W, []
    for i, t in enumerate(tok_slot):
        if t < 0 or A[t] is None:
            h.append(None)
            continue
        h.append((x[i] * keep[i]) @ A[t])
        y[i] += dropout_factor(scale[t], rates[t]) * (h[-1] @ B[t])
    return y, h


def dropout_backward(x, W, dy, tok_slot, A, B, scale, rates, keep):
    """(dx, dA, dB)."""
    x, W, dy = (np.asarray(v, dtype=np.float64) for v in (x, W, dy))
    dx = dy @ W.T
    dA, dB = [None if a is None else np.zeros(a.shape) for a in A], [None if b is None else np.zeros(b.shape) for b in B]
    for i, t in enumerate(tok_slot):
        if t < 0 or A[t] is None:
            continue
        f, xd = dropout_factor(scale[t], rates[t]), x[i] * keep[i]
        g = f * (B[t] @ dy[i])
        dx[i] += keep[i] * (A[t] @ g)
        dA[t] += np.outer(xd, g)
        dB[t] += f * np.outer(xd @ A[t], dy[i])
    return dx, dA, dB


# ---- cross entropy of a vocabulary head ----

def head_cross_entropy(x, W, targets, weight, tok_slot, n_slots, inv_temperature=1.0, grad_scale=1.0):
    """(logp [T], stats [n_slots + 1][4], dx [T][d]); a token with a negative target or a weight of 0 is ignored."""
    x, W = np.asarray(x, dtype=np.float64), np.asarray(W, dtype=np.float64)
    T = len(targets)
    logp, stats, dx = np.zeros(T), np.zeros((n_slots + 1, 4)), np.zeros(x.shape)
    for i in range(T):
        w = 1.0 if weight is None else float(weight[i])
        if targets[i] < 0 or w == 0:
            continue
        z = (x[i] @ W) * inv_temperature
        if np.all(z == -np.inf):
            p, logp[i] = np.zeros(len(z)), 0.0
        else:
            z = z - z.max()
            p = np.exp(z) / np.exp(z).sum()
            logp[i] = z[targets[i]] - np.log(np.exp(z).sum())
            e = p.copy()
            e[targets[i]] -= 1
            dx[i] = grad_scale * inv_temperature * w * (W @ e)
        stats[tok_slot[i] if tok_slot[i] >= 0 else n_slots] += (-w * logp[i], w, -logp[i], 1.0)
    return logp, stats, dx
