"""Plain float64 definitions of the gated linear recurrence, scaled embeddings and adjusted logits, with bounds for fp32 results (TEST INFRASTRUCTURE).

NumPy, one step after the other.  U is half a step of fp32."""
import numpy as np

U = 2.0 ** -24


def _parts(kind, gate, x):
    """(a, what is multiplied with x) of every step."""
    if kind == "decay":
        return gate, np.ones_like(gate)
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-gate)), 1.0 / (1.0 + np.exp(gate))


def gated_scan(gate, x, h0, kind, lengths=None):
    """y (T,B,D), the state before every step and behind the last one (T+1,B,D), and bounds for what fp32 makes of the states.

    A gate's two parts are off by up to 9 U of themselves each (exp 4, the sum and the reciprocal 4, their product 1), a product and a sum add 2; so a
    step adds 12 U of the magnitudes that meet in it, however the steps are grouped: a decay's error counts once for every step that its magnitude goes through."""
    gate, x = np.asarray(gate, np.float64), np.asarray(x, np.float64)
    T, Bn, D = gate.shape
    a, rest = _parts(kind, gate, x)
    h = np.zeros((Bn, D)) if h0 is None else np.asarray(h0, np.float64)
    ends = np.full(Bn, T) if lengths is None else np.clip(lengths, 0, T)
    y, states, bound = np.zeros((T, Bn, D)), np.empty((T + 1, Bn, D)), np.zeros((T + 1, Bn, D))
    states[0], m, e = h, np.abs(h), np.zeros((Bn, D))
    for t in range(T):
        on = t < ends
        u = np.where(on[:, None], rest[t] * np.where(on[:, None], x[t], 0.0), 0.0)
        at = np.where(on[:, None], a[t], 1.0)
        h = at * h + u
        m = np.abs(at) * m + np.abs(u)
        e = np.abs(at) * e + np.where(on[:, None], 12 * U * m, 0.0)
        states[t + 1], bound[t + 1] = h, e
        y[t] = np.where(on[:, None], h, 0.0)
    return y, states, bound


def gated_scan_bwd(gate, x, h0, dy, dh_last, kind, lengths=None):
    """(dgate, dx, dh0) and their bounds before they are stored."""
    gate, x, dy = (np.asarray(v, np.float64) for v in (gate, x, dy))
    T, Bn, D = gate.shape
    a, rest = _parts(kind, gate, x)
    _, states, bound = gated_scan(gate, x, h0, kind, lengths)
    ends = np.full(Bn, T) if lengths is None else np.clip(lengths, 0, T)
    G = np.zeros((Bn, D)) if dh_last is None else np.asarray(dh_last, np.float64)
    m, e = np.abs(G), np.zeros((Bn, D))
    dg, dx, bg, bx = (np.zeros((T, Bn, D)) for _ in range(4))
    for t in range(T - 1, -1, -1):
        on = (t < ends)[:, None]
        at, rt, xt = (np.where(on, v[t], z) for v, z in ((a, 1.0), (rest, 0.0), (x, 0.0)))
        g = G + np.where(on, dy[t], 0.0)
        m = m + np.where(on, np.abs(dy[t]), 0.0)
        e = e + np.where(on, U * m, 0.0)
        if kind == "sigmoid":
            dx[t], bx[t] = rt * g, rt * (e + 12 * U * m)
            d = states[t] - xt
            dg[t] = d * at * rt * g
            bg[t] = at * rt * (m * (bound[t] + 2 * U * (np.abs(states[t]) + np.abs(xt))) + np.abs(d) * (e + 24 * U * m))
        else:
            dx[t], bx[t] = np.where(on, g, 0.0), np.where(on, e, 0.0)
            dg[t], bg[t] = np.where(on, states[t] * g, 0.0), np.where(on, m * (bound[t] + 2 * U * np.abs(states[t])) + np.abs(states[t]) * e, 0.0)
        G, m, e = at * g, np.abs(at) * m, np.abs(at) * (e + np.where(on, 12 * U * m, 0.0))
    return (dg, dx, G), (bg, bx, e)


def embed_scaled(table, ids, scale):
    table, ids = np.asarray(table, np.float64), np.asarray(ids)
    ok = (ids >= 0) & (ids < len(table))
    out = np.zeros((len(ids), table.shape[1]))
    out[ok] = table[ids[ok]] * scale
    return out


def embed_scaled_bwd(ids, dout, rows, scale):
    """The table's gradient and its bound: up to 256 ids a token's rows one after the other; above, rows one after the other in pieces of 64 at most, then the pieces (in 8
    shares, each of which is no longer than all of them); then the scale.  A sum is off by a rounding of the sum of magnitudes for each addition on a row's way."""
    ids, dout = np.asarray(ids), np.asarray(dout, np.float64)
    ok = (ids >= 0) & (ids < rows)
    g, s, n = np.zeros((rows, dout.shape[1])), np.zeros((rows, dout.shape[1])), np.zeros(rows)
    np.add.at(g, ids[ok], dout[ok])
    np.add.at(s, ids[ok], np.abs(dout[ok]))
    np.add.at(n, ids[ok], 1)
    depth = (n if len(ids) <= 256 else np.minimum(n, 64) + np.ceil(n / 64)) + 20
    return g * scale, s * abs(scale) * (depth * U)[:, None]


def adjust(z, tokens=None, lengths=None, prompt=None, repetition=None, frequency=None, presence=None, bias_ids=None, bias=None, allowed=None):
    """Adjusted logits and the bound for fp32: every operation rounds once, what it rounds is no larger than the magnitudes that it joins."""
    z = np.array(z, np.float64)
    m = np.abs(z)
    V = z.shape[1]
    for n in range(len(z)):
        if tokens is not None:
            L = tokens.shape[1]
            end = L if lengths is None else min(max(int(lengths[n]), 0), L)
            mine = 0 if prompt is None else min(max(int(prompt[n]), 0), L)
            row = [int(t) for t in tokens[n, :end]]
            count = {}
            for i, t in enumerate(row):
                if 0 <= t < V:
                    count[t] = count.get(t, 0) + (i >= mine)
            for t, c in count.items():
                if repetition is not None:
                    z[n, t] = z[n, t] / repetition[n] if z[n, t] > 0 else z[n, t] * repetition[n]
                    m[n, t] = max(m[n, t], abs(z[n, t]))
                if frequency is not None:
                    z[n, t] -= frequency[n] * c
                    m[n, t] += abs(frequency[n] * c)
                if presence is not None and c > 0:
                    z[n, t] -= presence[n]
                    m[n, t] += abs(presence[n])
        if bias is not None:
            total = {}
            for i, b in zip(bias_ids[n], bias[n]):
                if 0 <= i < V:
                    total[int(i)] = total.get(int(i), 0.0) + float(b)
                    m[n, int(i)] += 4 * abs(float(b))
            for i, b in total.items():
                z[n, i] += b
        if allowed is not None:
            bits = np.unpackbits(np.ascontiguousarray(allowed[n]).view(np.uint8), bitorder="little")[:V]
            z[n, bits == 0] = -np.inf
    return z, 6 * U * m
