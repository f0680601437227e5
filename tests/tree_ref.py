"""Plain 64-bit forms of the operators around a drafted tree, for the GPU tests: quantised rows, tree attention, the
walk of the verification, each from its definition, one prompt at a time."""
import math

import numpy as np
import torch

TINY = 2.0 ** -126


def quantised(x, fmt):
    """What rows x [..., hd] (numpy, any float type) read back as, in fp32."""
    x = np.asarray(x, np.float64)
    a = np.abs(x).max(-1, keepdims=True)
    with np.errstate(all="ignore"):
        if fmt == "int8":
            s = np.maximum((a / 127).astype(np.float32).astype(np.float64), TINY)
            code = np.rint(x / s)
        else:
            e = np.where(a > 0, np.ceil(np.log2(np.where(a > 0, a, 1) / 448)), -1000)
            s = np.maximum(2.0 ** e, TINY)
            r = np.abs(x / s)
            grain = 2.0 ** (np.floor(np.log2(np.maximum(r, 2.0 ** -6))) - 3)
            code = np.sign(x) * np.rint(r / grain) * grain
        y = (code * s).astype(np.float32)
    return np.where(np.isfinite(a), y, np.float32(np.nan))


def sees(n, parents):
    """[n, n]: the nodes a node sees."""
    if parents is None:
        return np.tril(np.ones((n, n), bool))
    up = np.zeros((n, n), bool)
    for i in range(n):
        j = i
        while True:
            up[i, j] = True
            if not 0 <= parents[j] < j:
                break
            j = int(parents[j])
    return up


def attention(q, K, V, L, parents, scale):
    """(o, bound) of q [n, H, hd] over K, V [L + n, heads, hd] (all float64, numpy): the attention and, per output, what
    its rounding may be (see tolerance)."""
    n, H, hd = q.shape
    G = H // K.shape[1]
    mask = np.concatenate([np.ones((n, L), bool), sees(n, parents)], 1)
    o, mag, top = np.empty_like(q), np.empty_like(q), np.empty((n, H, 1))
    for h in range(H):
        k, v = K[:, h // G], V[:, h // G]
        z = np.where(mask, scale * (q[:, h] @ k.T), -np.inf)
        w = np.exp(z - z.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        o[:, h], mag[:, h] = w @ v, w @ np.abs(v)
        top[:, h, 0] = np.where(mask, abs(scale) * (np.abs(q[:, h]) @ np.abs(k).T), 0).max(1)
    return o, mag, top


def tolerance(mag, top, hd, keys, bf16):
    """Bound on |o - exact|.  A score is a sum of 3 hd products (bf16: hd, exact ones) in fp32, scaled twice, so it is off
    by (3 hd + 8) 2^-24 of the sum of its terms' sizes; exp2 and its argument's rounding add 2^-21 of the probability
    (arguments down to -30 that matter).  A probability enters its product off by 2^-16 (bf16: 2^-8).  The sums of
    probabilities and products run over the keys: 2 keys 2^-24.  Each counts in the numerator and in the denominator.
    A bf16 result rounds by 2^-8 of itself, which is at most mag."""
    p = (3 * hd + 8) * 2.0 ** -24 * top + 2.0 ** -21
    t = 2 * p + (2.0 ** -8 if bf16 else 2.0 ** -16) + 4 * (keys + 8) * 2.0 ** -24
    return mag * (t + (2.0 ** -8 if bf16 else 2.0 ** -24)) + 1e-37


def walk(p, q, tokens, parents, u, v, replace):
    """(path, next token) of one prompt (numpy; p, q [n, V] fp32) by the definition, in float64."""
    p, q = p.astype(np.float64), q.astype(np.float64)
    n, V = p.shape
    cur, path = 0, [0]
    P, Q, rest, dead = p[0], q[0].copy(), 1.0, False
    for j in range(1, n):
        x = int(tokens[j])
        if parents[j] != cur or not 0 <= x < V or dead or not rest > 0:
            continue
        qx = Q[x] / rest
        if P[x] > 0 and float(u[j]) * qx <= P[x]:
            cur = j
            path.append(j)
            P, Q, rest = p[j], q[j].copy(), 1.0
            continue
        R = np.maximum(0, P - Q / rest)
        if R.sum() > 0:
            P = R / R.sum()
        else:
            dead = True
        if not replace:
            rest -= Q[x]
            Q[x] = 0
    if dead:
        return path, int(np.argmax(p[cur]))
    c = np.cumsum(P)
    if not c[-1] > 0:
        return path, -1
    hit = np.nonzero(c > float(v) * c[-1])[0]
    return path, int(hit[0]) if len(hit) else int(np.nonzero(P > 0)[0][-1])


def random_tree(rng, n, width, shape="tree"):
    if shape == "chain":
        return np.arange(-1, n - 1).astype(np.int32)
    if shape == "star":
        return np.array([-1] + [0] * (n - 1), np.int32)
    if shape == "forest":      # several roots, and parents that end the way up
        par = rng.integers(-3, np.maximum(1, np.arange(n)))
        return par.astype(np.int32)
    return np.array([-1] + [int(rng.integers(max(0, j - 2 * width), j)) for j in range(1, n)], np.int32)


def paged(rng, layers, B, tokens, heads, hd, fmt, spare=2, fill=None):
    """A QuantCache whose pages hold leftovers, in no order."""
    from paper_2412_10418_amd.binding import QuantCache
    per = -(-tokens // 32)
    pages = B * per + spare
    pool = QuantCache.empty(layers, pages, heads, hd)
    if fill is None:
        pool.copy_(torch.from_numpy(rng.integers(0, 256, pool.shape, dtype=np.uint8)))
    else:
        pool.fill_(fill)
    table = torch.from_numpy(rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32)).cuda()
    return QuantCache(pool, table, hd, fmt)


def close(got, ref, tol, what):
    """Prints the worst case and holds every entry to its bound."""
    err = np.abs(got.astype(np.float64) - ref)
    worst = float((err / tol).max()) if err.size else 0.0
    print(f"{what}: error at most {worst:.3f} of its bound", flush=True)
    assert not math.isnan(worst) and worst <= 1, worst
