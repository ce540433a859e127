"""Plain fp64 references of rotary positions, the paged cache and the attention
of drafted tokens, written from their definitions (include/hstu.h): loops over
tokens, the 8-bit codes by search among all values a code can stand for."""
import numpy as np


def rotate(x, positions, inv_freq, interleaved, amplitude=1.0, back=False):
    """x [T, h, d] turned; also |a| + |b| of each output's pair (0 for copies)."""
    x = np.asarray(x, np.float64)
    out, size = x.copy(), np.zeros_like(x)
    n = len(inv_freq)
    for m in range(n):
        ia, ib = (2 * m, 2 * m + 1) if interleaved else (m, m + n)
        theta = np.asarray(positions, np.float64) * inv_freq[m] * (-1.0 if back else 1.0)
        c, s = amplitude * np.cos(theta)[:, None], amplitude * np.sin(theta)[:, None]
        a, b = x[:, :, ia], x[:, :, ib]
        out[:, :, ia], out[:, :, ib] = a * c - b * s, a * s + b * c
        size[:, :, ia] = size[:, :, ib] = abs(amplitude) * (np.abs(a) + np.abs(b))
    return out, size


def e4m3_values():
    """The magnitudes of codes 0 .. 126: 4 exponent bits (bias 7), 3 of mantissa."""
    out = []
    for code in range(127):
        e, m = code >> 3, code & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(out)


def quantise(x, kind):
    """(codes as the numbers they stand for, scale) of rows x [..., d]."""
    x = np.asarray(x, np.float64)
    codes, scale = np.zeros_like(x), np.ones(x.shape[:-1])
    table = e4m3_values()
    for at in np.ndindex(x.shape[:-1]):
        row = x[at]
        if not np.isfinite(row).all():
            scale[at] = np.nan
            continue
        top = np.abs(row).max()
        if top < 2.0 ** -100:
            continue
        if kind == "int8":
            s = float(np.float32(top * float(np.float32(1.0 / 127.0))))
            codes[at] = np.rint(row / s)
        else:
            e = -200
            while e < 119 and top > 448.0 * 2.0 ** e:
                e += 1
            s = 2.0 ** e
            y = np.minimum(np.abs(row) / s, 448.0)
            hi = np.clip(np.searchsorted(table, y), 1, 126)
            lo = hi - 1
            up = (table[hi] - y < y - table[lo]) | ((table[hi] - y == y - table[lo]) & (hi % 2 == 0))
            codes[at] = np.copysign(np.where(up, table[hi], table[lo]), row)
        scale[at] = s
    return codes, scale


def held(x, kind):
    """What a cache of this kind gives back of rows x (fp64, not rounded)."""
    if kind == "bf16":
        import oracle
        return oracle.round_store(np.asarray(x, np.float64), "bf16")
    codes, scale = quantise(x, kind)
    return codes * scale[..., None]


def depths(parents):
    """Depth and way to the root (itself first) of each node of one forest."""
    ways = []
    for i, p in enumerate(parents):
        ways.append([i] + (ways[p] if 0 <= p < i else []))
    return np.array([len(w) - 1 for w in ways], dtype=np.int64), ways


def bucket(dt, nb):
    return min(nb - 1, max(abs(int(dt)), 1).bit_length() - 1)


def tree(q, k, v, t, kc, vc, tc, parents, rab_pos, rab_time, N):
    """One sequence: drafted q, k, v [L, h, d], t [L] over cached kc, vc [n, h, d],
    tc [n].  Returns (out [L, h, d_v], slack [L, h, d_v]): slack bounds what
    rounding the attention weights to bf16 and summing scores in fp32 can change."""
    L, h, d = q.shape
    n = len(tc)
    nb = len(rab_time)
    dep, ways = depths(parents)
    out, slack = np.zeros((L, h, v.shape[2])), np.zeros((L, h, v.shape[2]))
    for i in range(L):
        pi = n + dep[i]
        idx = ways[i]
        keys = np.concatenate([kc, k[idx]]) if n else k[idx]
        vals = np.concatenate([vc, v[idx]]) if n else v[idx]
        pos = np.concatenate([np.arange(n), n + dep[idx]])
        tim = np.concatenate([tc, t[idx]])
        bias = (rab_pos[np.maximum(0, N - 1 + pos - pi)]
                + rab_time[[bucket(t[i] - x, nb) for x in tim]])
        for a in range(h):
            s = keys[:, a] @ q[i, a] + bias
            p = s / (1.0 + np.exp(-s))
            out[i, a] = p @ vals[:, a] / N
            size = np.abs(keys[:, a]) @ np.abs(q[i, a]) + np.abs(bias)
            off = np.abs(p) * (2.0 ** -8 + 2.0 ** -18) + 1.1 * size * (d + 8) * 2.0 ** -24
            slack[i, a] = off @ np.abs(vals[:, a]) / N
    return out, slack
