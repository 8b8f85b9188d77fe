"""Plain numpy forms, in 64 bits, of the weight dropout and of the experts' balance (ws.h states both): what the CUDA
entry points are compared with, and what stands behind their names on CPU ranks."""
import numpy as np

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
LOW = np.uint64(0xFFFFFFFF)


def philox(key, counter, rounds):
    """Philox4x32: key (2 words), counter (4 arrays of words) -> 4 arrays of words."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(x) for x in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(M0), c[2] * np.uint64(M1)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & LOW, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & LOW]
        k = [(k[0] + W0) & 0xFFFFFFFF, (k[1] + W1) & 0xFFFFFFFF]
    return c


def threshold(p):
    return min(int(np.floor(p * 65536 + 0.5)), 65535)


def scale(p):
    return 65536.0 / (65536.0 - threshold(p))


def keep(p, seed, step, replica, t, n, start=0):
    """Which of elements start ... start + n - 1 (start a multiple of 8) of tensor t replica `replica` keeps."""
    assert start % 8 == 0
    j = np.arange(start // 8, (start + n + 7) // 8, dtype=np.uint64)
    one = np.ones_like(j)
    w = philox((seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF),
               (j & LOW, one * np.uint64(step & 0xFFFFFFFF), one * np.uint64(t), one * np.uint64(replica) + ((j >> np.uint64(32)) << np.uint64(16))), 7)
    halves = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], axis=-1).ravel()[:n]
    return halves >= threshold(p)


def hand_out(w, p, seed, step, replica, t):
    """Replica's copy of tensor t from its full-precision values."""
    return np.where(keep(p, seed, step, replica, t, w.size), w.astype(np.float64).ravel() * scale(p), 0.0)


def masked_sum(grads, p, seed, step, replica, t):
    """(sum, sum of magnitudes) of the replicas' gradients of tensor t, masked and scaled."""
    total, size = 0.0, 0.0
    with np.errstate(invalid="ignore"):
        for k, g in enumerate(grads):
            v = np.where(keep(p, seed, step, replica + k, t, g.size), g.astype(np.float64).ravel(), 0.0) * scale(p)
            total, size = total + v, size + np.abs(v)
    return total, size


# ------------------------------------------------------------------ routers
def counts(picks, valid, experts):
    """[layers][experts + 1] from picks[layer][replica] and valid (None, or one array or None per replica)."""
    out = np.zeros((len(picks), experts + 1), dtype=np.int64)
    for l, layer in enumerate(picks):
        for k, p in enumerate(layer):
            live = np.ones(len(p), dtype=bool) if valid is None or valid[k] is None else valid[k].astype(bool)
            q = p[live].ravel()
            q = q[(q >= 0) & (q < experts)]
            np.add.at(out[l], q, 1)
            out[l, experts] += live.sum()
    return out


def scores(x, score):
    """(p, lse, dp factor, top) of rows x in 64 bits; rows without an expert to pick are 0."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        top = np.max(x, axis=1, keepdims=True)
        top = np.where(np.isfinite(top), top, 0.0)
        if score == "softmax":
            s, q = np.exp(x - top), np.ones_like(x)
        else:                   # p from log s: the ratios last where the scores vanish
            logs = np.where(x == -np.inf, -np.inf, np.minimum(x, 0.0) - np.log1p(np.exp(-np.abs(x))))
            best = np.max(logs, axis=1, keepdims=True)
            s, q = np.exp(logs - np.where(np.isfinite(best), best, 0.0)), 1.0 / (1.0 + np.exp(x))
        total = s.sum(1, keepdims=True)
        empty = total == 0
        p = np.where(empty, 0.0, s / total)
        lse = np.where(empty, 0.0, top + np.log(total)) if score == "softmax" else np.zeros_like(top)
    return p, lse, q, np.abs(top)


def balance(logits, valid, cnt, topk, score, coef, z, upstream=1.0):
    """(loss [layers][2], dlogits[layer][replica], their error scale) from the counts; a token whose byte is 0 has gradient 0.
    The scale is what a relative error of the fp32 scores is multiplied with in a gradient."""
    experts = cnt.shape[1] - 1
    loss = np.zeros((len(logits), 2))
    grads, sizes = [], []
    for l, layer in enumerate(logits):
        n = float(cnt[l, experts])
        inv = 1.0 / n if n else 0.0
        f = cnt[l, :experts] * inv / topk
        grads.append([])
        sizes.append([])
        for k, x in enumerate(layer):
            live = np.ones(len(x), dtype=bool) if valid is None or valid[k] is None else valid[k].astype(bool)
            x = np.where(live[:, None], x.astype(np.float64), 0.0)
            p, lse, q, top = scores(x, score)
            s = (p * f).sum(1, keepdims=True)
            loss[l, 0] += coef * experts * inv * s[live].sum()
            loss[l, 1] += z * inv * np.square(lse[live]).sum()
            a, b = upstream * coef * experts * inv, 2 * upstream * z * inv
            d = p * q * a * (f - s) + (b * lse * p if z else 0.0)
            grads[-1].append(np.where(live[:, None], d, 0.0))
            sizes[-1].append(np.where(live[:, None], p * q * abs(a) * (f + s) + abs(b) * p * (np.abs(lse) + top + 1), 0.0))
    return loss, grads, sizes
