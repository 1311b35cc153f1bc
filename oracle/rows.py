"""Plain float64 definitions of the row operators: the counter-based mask, dropout, layer normalisation, sampling (TEST INFRASTRUCTURE).

NumPy, one operation after the other, no regard for speed.  What the library defines bit by bit -- the mask, the sum of a residual
stream -- is computed with the same roundings."""
import numpy as np

M0, M1, W0, W1, LOW = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85, 0xFFFFFFFF


def philox4x32(counter, key, rounds):
    """Four words from a counter of four and a key of two, in Python's whole numbers."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        p0, p1 = M0 * c[0], M1 * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & LOW, (p0 >> 32) ^ c[3] ^ k[1], p0 & LOW]
        k = [(k[0] + W0) & LOW, (k[1] + W1) & LOW]
    return c


def mask(rows, cols, ratio, seed, offset, site):
    """keep[row, col] as chn_dropout defines it."""
    nb = (cols + 3) // 4
    c = [np.broadcast_to(np.arange(nb, dtype=np.uint64), (rows, nb)), np.broadcast_to(np.arange(rows, dtype=np.uint64)[:, None], (rows, nb)),
         np.full((rows, nb), offset & LOW, np.uint64), np.full((rows, nb), site, np.uint64)]
    k = [seed & LOW, (seed >> 32) & LOW]
    s32, low = np.uint64(32), np.uint64(LOW)
    for _ in range(7):
        p0, p1 = np.uint64(M0) * c[0], np.uint64(M1) * c[2]
        c = [(p1 >> s32) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> s32) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + W0) & LOW, (k[1] + W1) & LOW]
    words = np.stack(c, -1).reshape(rows, nb * 4)[:, :cols]
    return words >= np.uint64(min(int(ratio * 2.0 ** 32 + 0.5), LOW))


def dropout(x, ratio, seed=0, offset=0, site=0, residual=None):
    """In fp32, operation by operation: the result before it is stored."""
    x = np.asarray(x, np.float32)
    if x.size == 0:
        return x
    rows = x.reshape(-1, x.shape[-1]) if x.ndim else x.reshape(1, 1)
    with np.errstate(over="ignore", invalid="ignore"):
        if ratio > 0:
            keep = mask(rows.shape[0], rows.shape[1], ratio, seed, offset, site)
            y = np.where(keep, rows * np.float32(1.0 / (1.0 - ratio)), np.float32(0)).reshape(x.shape)
        else:
            y = x
        return y if residual is None else np.asarray(residual, np.float32) + y


def layer_norm(x, gamma=None, beta=None, eps=1e-5):
    x = np.asarray(x, np.float64)
    mean = x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    y = (x - mean) * rstd
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    if beta is not None:
        y = y + np.asarray(beta, np.float64)
    return y, mean[:, 0], rstd[:, 0]


def layer_norm_bwd(dy, x, mean, rstd, gamma=None):
    dy, x, mean, rstd = (np.asarray(a, np.float64) for a in (dy, x, mean, rstd))
    h = (x - mean[:, None]) * rstd[:, None]
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """Tokens by row; parameters: one value for each row, or None."""
    logits = np.asarray(logits, np.float64)
    out = []
    for n, z in enumerate(logits):
        ids = np.nonzero(z > -np.inf)[0]
        if len(ids) == 0:
            out.append(-1)
            continue
        best = z[ids].max()
        t = 1.0 if temperature is None else float(temperature[n])
        if not t > 0:
            out.append(ids[z[ids] == best][0])
            continue
        with np.errstate(all="ignore"):
            w = np.where(z == best, 1.0, np.exp((z - best) / t))
        order = ids[np.lexsort((ids, -z[ids]))]                  # descending logits, equals by index
        if top_k is not None and top_k[n] > 0:
            order = order[:int(top_k[n])]
        if top_p is not None and float(top_p[n]) < 1:
            before = np.concatenate([[0.0], np.cumsum(w[order])])
            keep = before[:-1] < float(top_p[n]) * before[-1]
            keep[0] = True
            order = order[keep]
        if min_p is not None and float(min_p[n]) > 0:
            order = order[w[order] >= min(float(min_p[n]), 1.0)]
        kept = np.sort(order[w[order] > 0])
        run, un = np.cumsum(w[kept]), float(u[n])
        hit = np.nonzero(run > un * run[-1])[0] if un > 0 else np.array([0])
        out.append(kept[hit[0]] if len(hit) else kept[-1])
    return np.array(out, np.int64)
