"""Plain reference of the operators on 4-bit pages, in 64 bits on the CPU, one value at a time where that is the plainest."""
import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
H24, H8 = 2.0 ** -24, 2.0 ** -8        # half a step of fp32 and bf16 relative to a value


def scale_exponent(amax):
    """The smallest e in -125 .. 125 with amax <= 7 * 2^e (125 if none is large enough)."""
    if amax == 0.0:
        return -125
    e = math.frexp(amax)[1] - 4
    while amax > 7.0 * 2.0 ** e:
        e += 1
    return min(max(e, -125), 125)


def nearest_code(a):
    """Code of a magnitude in units of the scale: nearest, ties to the even code, 7 (6.0) above."""
    d = np.abs(GRID - a)
    best = np.flatnonzero(d == d.min())
    return int(best[0]) if len(best) == 1 or best[0] % 2 == 0 else int(best[1])


def quantise(x):
    """x [hd] -> (values held [hd], exponents [hd / 32])."""
    out, es = np.empty(len(x)), []
    for c in range(len(x) // 32):
        b = x[32 * c: 32 * c + 32].astype(np.float64)
        e = scale_exponent(float(np.abs(b).max()))
        es.append(e)
        out[32 * c: 32 * c + 32] = [math.copysign(GRID[nearest_code(abs(v) / 2.0 ** e)] * 2.0 ** e, v) for v in b]
    return out, es


def half_step(a):
    """What rounding to a code may be off by, for a magnitude a in units of the scale."""
    return np.where(a <= 2.0, 0.25, np.where(a <= 4.0, 0.5, 1.0))


def frequencies(r):
    n, theta = r["rot_dim"], r.get("theta", 10000.0)
    theta = float(np.float32(theta))
    kind, factor, low, high, ctx = r.get("scaling", "none"), float(np.float32(r.get("factor", 1.0))), r.get("low", 1.0), r.get("high", 4.0), r.get("orig_ctx", 4096)
    out = []
    for i in range(n // 2):
        f = theta ** (-2.0 * i / n)
        if kind == "linear":
            f /= factor
        elif kind == "wave":
            s = min(1.0, max(0.0, (ctx * f / (2 * math.pi) - low) / (high - low)))
            f *= s + (1 - s) / factor
        elif kind == "index":
            at = lambda t: n * math.log(ctx / (2 * math.pi * t)) / (2 * math.log(theta))  # noqa: E731
            a, b = max(0, math.floor(at(high))), min(n - 1, math.ceil(at(low)))
            s = min(1.0, max(0.0, (i - a) / max(b - a, 0.001)))
            f *= (1 - s) + s / factor
        out.append(f)
    return np.array(out)


def rotate(x, pos, r):
    """x [rows, heads, hd] in 64 bits; returns (rotated, bound on what 32-bit arithmetic may be off by).

    cos and sin are rounded (half a step each), so are the two products and their sum: 2 (|x c| + |y s|) + |result| half steps, at most
    3 gain (|x| + |y|); a frequency or angle in 64 bits adds position * 2^-52, nothing beside that."""
    x = x.astype(np.float64)
    y, err = x.copy(), np.zeros_like(x)
    n = r["rot_dim"]
    if n == 0:
        return y, err
    gain = float(np.float32(r.get("gain", 1.0)))
    ang = np.asarray(pos, np.float64)[:, None] * frequencies(r)[None]
    c, s = np.cos(ang)[:, None] * gain, np.sin(ang)[:, None] * gain
    i = np.arange(n // 2)
    a, b = (i, i + n // 2) if r.get("style", "half") == "half" else (2 * i, 2 * i + 1)
    x1, x2 = x[..., a], x[..., b]
    y[..., a], y[..., b] = x1 * c - x2 * s, x2 * c + x1 * s
    slack = abs(gain) * (np.abs(x1) + np.abs(x2)) * (3 * H24 * 1.01 + 2.0 ** -51 * np.abs(np.asarray(pos, np.float64))[:, None, None] * 4)
    err[..., a], err[..., b] = slack, slack
    return y, err


def page_plan(table, held, ring, state, lens, n_new, page, rows):
    """One request after the other; lists and arrays are changed in place.  Returns slots, pos, start, served."""
    B, width = table.shape
    n_pages = len(ring)
    head, count = int(state[0]), int(state[1])
    slots, pos, start, served = np.full(rows, -1, np.int64), np.full(rows, -1, np.int64), np.zeros(B + 1, np.int64), np.zeros(B, np.int64)
    L, N = np.maximum(lens, 0).astype(np.int64), np.maximum(n_new, 0).astype(np.int64)
    start[1:] = np.cumsum(N)
    need = -(-(L + N) // page)
    back = [int(table[b, j]) for b in range(B) for j in range(need[b], held[b])]
    wanted, taken = 0, 0
    for b in range(B):
        if need[b] > width or start[b + 1] > rows:
            held[b] = min(held[b], need[b])
            continue
        take = max(0, int(need[b] - held[b]))
        wanted += take
        if take and wanted > count:
            continue
        for j in range(take):
            table[b, held[b] + j] = ring[(head + taken) % n_pages]
            taken += 1
        held[b] = need[b]
        served[b] = 1
    for b in range(B):
        for i in range(int(start[b]), int(min(start[b + 1], rows))):
            p = int(L[b]) + i - int(start[b])
            pos[i] = p
            if served[b]:
                slots[i] = int(table[b, p // page]) * page + p % page
    for i, x in enumerate(back):
        ring[(head + count + i) % n_pages] = x
    state[0], state[1] = (head + taken) % n_pages, count - taken + len(back)
    return slots, pos, start, served


def attention(q, K, V, lens, n_new, scale, bf16):
    """q [rows, H, hd], K, V lists of [L, KH, hd] per request (held values).  Returns (out, bound).

    Bound.  A score is off by A = scale sum |q| |k| times: fp32, the three-term q (2^-24); its sum in 32 bits (hd + 4 terms of 2^-24, each
    product exact).  The exponent's argument and exp2 add (|score| + 4) 2^-23.  An error d of all scores moves every weight by at most a
    factor e^(2 d), 2.1 d while d is small.  Weights: bf16, half a step 2^-8 (fp32, three terms: 2^-24)
    each, and bf16 ones are divided by the sum of the rounded weights: with w_i (1 + e_i), |e_i| <= 2^-8, the output is off by
    sum w_i e_i (v_i - out) to first order, at most 2^-8 (sum w_i |v_i| + |out|); their sum and the products' L 2^-24; the merges
    and the division 64 2^-24.  Output in bf16: half a step of it."""
    rows, H, hd = q.shape
    out, bound = np.zeros((rows, H, hd)), np.zeros((rows, H, hd))
    at = 0
    for b, n in enumerate(n_new):
        L, G = int(lens[b]), H // K[b].shape[1] if len(K[b]) else 1
        for i in range(n):
            see = min(L, L - n + i + 1)
            if see > 0:
                for h in range(H):
                    k, v, x = K[b][:see, h // G], V[b][:see, h // G], q[at + i, h]
                    s = scale * (k @ x)
                    if np.isnan(s).any():
                        out[at + i, h] = np.nan
                        continue
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    out[at + i, h] = w @ v
                    d = float((scale * (np.abs(k) @ np.abs(x))).max()) * ((0 if bf16 else H24) + (hd + 4) * H24) + (np.abs(s).max() * 1.5 + 4) * 2 * H24
                    rel = 2.1 * d + (H8 if bf16 else H24) + (see + 64) * H24
                    bound[at + i, h] = (w @ np.abs(v)) * rel * 1.01 + (2 * H8 * np.abs(out[at + i, h]) * 1.01 if bf16 else 0) + 1e-37
        at += n
    return out, bound


def accept(P, Q, d, n, u, w):
    """Alg. 3 on probabilities, row by row; P [rows, gamma + 1, V] fp32 and so on, as numpy arrays."""
    R, G1, V = P.shape
    acc, tokens = np.zeros(R, np.int64), np.full((R, G1), -1, np.int64)
    for b in range(R):
        nd = G1 - 1 if n is None else min(max(int(n[b]), 0), G1 - 1)
        k = 0
        while k < nd:
            t = int(d[b, k])
            if not 0 <= t < V:
                break
            q = float(Q[b, k, t]) if Q is not None else 1.0
            if not float(u[b, k]) * q < float(P[b, k, t]):
                break
            k += 1
        p = P[b, k].astype(np.float64)
        law = np.where(p > 0, p, 0.0)
        if k < nd:
            if Q is not None:
                with np.errstate(invalid="ignore"):
                    r = p - Q[b, k].astype(np.float64)
                r = np.where(r > 0, r, 0.0)
            else:
                r = law.copy()
                if 0 <= d[b, k] < V:
                    r[int(d[b, k])] = 0.0
            if r.sum() > 0:
                law = r
        c = np.cumsum(law)
        above = np.flatnonzero(c > float(w[b]) * c[-1])
        token = int(above[0]) if len(above) else -1
        acc[b] = k
        tokens[b, :k] = d[b, :k]
        tokens[b, k] = token
    return acc, tokens
