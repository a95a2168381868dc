"""Plain 64-bit CPU implementations of the router, the balance loss, the gate gradient and AdamW, written from their formulas.

Test infrastructure only: loops and numpy, one token, sequence or element at a time where that is the clearest.  Scores, gates and
moments come in as float64 arrays that hold what the 32- or 16-bit inputs hold.
"""
from __future__ import annotations

import numpy as np

SOFTMAX_SELECTED, SOFTMAX_ALL, SIGMOID, SIGMOID_NORMALISED = range(4)


def top_k(scores, k):
    """ids [T,k]: largest first, the lower index first among equal scores; NaN ranks with -inf."""
    out = np.empty((scores.shape[0], k), dtype=np.int64)
    for t, row in enumerate(scores):
        key = [-np.inf if np.isnan(s) else s for s in row]
        out[t] = sorted(range(len(key)), key=lambda e: (-key[e], e))[:k]
    return out


def _softmax(x):
    top = np.max(x)
    if top == -np.inf:
        return np.zeros_like(x)
    e = np.exp(x - top)
    return e / e.sum()


def _sigmoid(x):
    return np.where(x >= 0, 1.0 / (1.0 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1.0 + np.exp(-np.abs(x))))


def _log_sigmoid(x):
    return np.minimum(x, 0.0) - np.log1p(np.exp(-np.abs(x)))


def probabilities(row, gating):
    """Over all experts: softmax, or sigmoids over their sum (taken through logarithms, so no score is too small)."""
    return _softmax(_log_sigmoid(row) if gating >= SIGMOID else row)


def gates(scores, ids, gating, mask=None):
    out = np.zeros(ids.shape)
    with np.errstate(invalid="ignore", over="ignore"):
        for t in range(ids.shape[0]):
            if mask is not None and not mask[t]:
                continue
            chosen = scores[t, ids[t]]
            if gating == SOFTMAX_SELECTED:
                out[t] = _softmax(chosen)
            elif gating == SOFTMAX_ALL:
                out[t] = _softmax(scores[t])[ids[t]]
            elif gating == SIGMOID:
                out[t] = _sigmoid(chosen)
            else:
                out[t] = _softmax(_log_sigmoid(chosen))
    return out


def balance(scores, ids, gating, alpha, offsets=None, mask=None):
    """counts, mean probabilities, coefficients [S,E] and the loss."""
    T, E = scores.shape
    k = ids.shape[1]
    offsets = [0, T] if offsets is None else list(offsets)
    S = len(offsets) - 1
    counts, prob, coef, loss = np.zeros((S, E), dtype=np.int64), np.zeros((S, E)), np.zeros((S, E)), 0.0
    for s in range(S):
        tokens = [t for t in range(offsets[s], offsets[s + 1]) if mask is None or mask[t]]
        n = len(tokens)
        if n == 0:
            continue
        for t in tokens:
            prob[s] += probabilities(scores[t], gating) / n
            for e in ids[t]:
                if 0 <= e < E:
                    counts[s, e] += 1
        f = counts[s] / (k * n)
        loss += alpha * E * float(f @ prob[s])
        coef[s] = alpha * E * f / n
    return counts, prob, coef, loss


def route_bwd(scores, gating, ids=None, dlog=None, coef=None, offsets=None, mask=None):
    """Gradient by the scores: of the balance loss whose coefficients are given, and of gates whose gradients by their logs are."""
    T, E = scores.shape
    ds = np.zeros((T, E))
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        row = scores[t]
        if coef is not None:
            where = 0 if offsets is None else next((s for s in range(len(offsets) - 1) if offsets[s] <= t < offsets[s + 1]), None)
            if where is not None:
                p, c = probabilities(row, gating), coef[where]
                ds[t] += p * (c - c @ p) * (_sigmoid(-row) if gating >= SIGMOID else 1.0)
        if dlog is not None:
            slots = [(int(e), q) for e, q in zip(ids[t], dlog[t]) if 0 <= e < E]
            if not slots:
                continue
            at, q = np.array([e for e, _ in slots]), np.array([v for _, v in slots])
            if gating == SOFTMAX_ALL:
                ds[t] -= _softmax(row) * q.sum()
                u = q
            elif gating == SIGMOID:
                u = q * _sigmoid(-row[at])
            else:
                g = _softmax(row[at]) if gating == SOFTMAX_SELECTED else _softmax(_log_sigmoid(row[at]))
                u = q - g * q.sum()
                if gating == SIGMOID_NORMALISED:
                    u = u * _sigmoid(-row[at])
            for e, v in zip(at, u):
                ds[t, e] += v
    return ds


def gate_bwd(dY, rows, src_to_row, k):
    """dlog [T,k] = <dY[t], rows[src_to_row[t k + j]]>."""
    T = dY.shape[0]
    return np.array([[float(dY[t] @ rows[src_to_row[t * k + j]]) for j in range(k)] for t in range(T)]).reshape(T, k)


# ---- AdamW -------------------------------------------------------------------------------------------------------


def adamw(w, g, m, v, lr, beta1, beta2, eps, weight_decay, step, grad_scale=1.0):
    g = g * grad_scale
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    w = w - lr * weight_decay * w - lr / (1.0 - beta1 ** step) * m / (np.sqrt(v / (1.0 - beta2 ** step)) + eps)
    return w, m, v


def noise(places, seed):
    """32 bits per place of the list (uint64 array), a function of the place and the seed."""
    word = np.uint64(0xffffffff)
    p = np.asarray(places, dtype=np.uint64)
    h = ((p & word) + (p >> np.uint64(32)) * np.uint64(0x632BE5AB) + np.uint64((seed * 0x9E3779B1) & 0xffffffff)) & word
    h ^= h >> np.uint64(16)
    h = (h * np.uint64(0xA3D95FA9)) & word
    h ^= h >> np.uint64(15)
    h = (h * np.uint64(0x7B1D4E65)) & word
    return h ^ (h >> np.uint64(16))


def root_bits(words, beta2):
    """The 20 random bits that round sqrt(v): a word's lower 12 and a half, or 8 bits more where 1 - beta2 < 2^-10."""
    h = np.asarray(words, dtype=np.uint64)
    more = (h * np.uint64(0x85EBCA6D) & np.uint64(0xffffffff)) >> np.uint64(24) if np.float32(1.0 - beta2) < 2.0 ** -10 else np.uint64(128)
    return ((h & np.uint64(0xfff)) << np.uint64(8) | more).astype(np.int64)


def places_of(sizes):
    """The places of every tensor's elements: tensors one after the other, each rounded up to a multiple of 32."""
    at, out = 0, []
    for n in sizes:
        out.append(np.arange(at, at + n, dtype=np.uint64))
        at += -(-n // 32) * 32
    return out


def e4m3_value(code):
    """The number a code of sign, 4 exponent bits (bias 7) and 3 mantissa bits stands for; 0x7f is NaN."""
    sign = -1.0 if code & 0x80 else 1.0
    e, f = (code >> 3) & 15, code & 7
    if e == 15 and f == 7:
        return np.nan
    return sign * (f / 8.0 * 2.0 ** -6 if e == 0 else (1 + f / 8.0) * 2.0 ** (e - 7))


E4M3 = np.array([e4m3_value(c) for c in range(256)])


def decode(codes, exps):
    """Values of 8-bit codes under their blocks' exponents."""
    scale = np.where(np.asarray(exps) == 255, np.nan, 2.0 ** (np.asarray(exps, dtype=np.float64) - 127))
    return E4M3[codes] * np.repeat(scale, 32)[:len(codes)]


def shared_exponents(x):
    """Per 32 neighbours of x >= 0: the least biased exponent under which the largest is at most 448; 255 for a NaN or infinity."""
    out = []
    for a in range(0, len(x), 32):
        top = x[a:a + 32].max() if not np.isnan(x[a:a + 32]).any() else np.nan
        if not np.isfinite(top):
            out.append(255)
        else:
            e = -127
            if top > 0:
                e = int(np.floor(np.log2(top / 448.0)))
                while top > 448.0 * 2.0 ** e:
                    e += 1
                while e > -127 and top <= 448.0 * 2.0 ** (e - 1):
                    e -= 1
            out.append(max(e, -127) + 127)
    return np.array(out, dtype=np.int64)


def neighbours(x, exps):
    """The e4m3 numbers around x >= 0 under the blocks' exponents, as values: the largest not above, the smallest not below."""
    grid = E4M3[:127]
    scale = np.repeat(2.0 ** (exps.astype(np.float64) - 127), 32)[:len(x)]
    y = np.minimum(x / scale, 448.0)
    low = grid[np.searchsorted(grid, y, side="right") - 1]
    high = grid[np.minimum(np.searchsorted(grid, y, side="left"), 126)]
    return low * scale, high * scale
