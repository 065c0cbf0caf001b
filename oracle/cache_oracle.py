"""Plain fp64 definitions of the operators on a key/value cache in pages: rotary positions, append, attention with the
mass per slot, eviction.  Loops and elementary numpy, one request at a time; no code shared with the library."""
import math

import numpy as np

TWO_PI = np.longdouble("6.28318530717958647692528676655900576839")


def rope_angles(positions, section, theta, per_axis):
    """[rows, pairs] angles in radians within one turn: the product is taken in 64-bit-mantissa floats and whole turns
    are dropped before it is rounded to fp64."""
    n = sum(section)
    out = np.zeros((len(positions), n))
    i = 0
    for axis, size in enumerate(section):
        for j in range(size):
            e = np.longdouble(j) / size if per_axis else np.longdouble(i) / n
            turns = np.asarray(positions)[:, axis].astype(np.longdouble) * (np.longdouble(theta) ** -e / TWO_PI)
            out[:, i] = ((turns - np.floor(turns)) * TWO_PI).astype(np.float64)
            i += 1
    return out


def rope(x, angles, neighbours=False, inverse=False):
    """x [rows, heads, dh]; pair (x[i], x[n + i]) or (x[2i], x[2i + 1]) turned by angles[:, i]."""
    y = np.array(x, dtype=np.float64)
    n = angles.shape[1]
    for i in range(n):
        lo, hi = (2 * i, 2 * i + 1) if neighbours else (i, n + i)
        c, s = np.cos(angles[:, i])[:, None], np.sin(angles[:, i])[:, None]
        if inverse:
            s = -s
        a, b = x[:, :, lo].astype(np.float64), x[:, :, hi].astype(np.float64)
        y[:, :, lo], y[:, :, hi] = a * c - b * s, a * s + b * c
    return y


def places(table_row, n, page_size):
    """Flat slot numbers in the pool of a request's first n slots."""
    return np.array([int(table_row[j // page_size]) * page_size + j % page_size for j in range(n)], dtype=np.int64)


def attend(q, k, v, scale):
    """q [rows, H, dh], k and v [n, Hkv, dh] of one request.  Returns out [rows, H, dh], p [rows, H, n], and for error
    bounds sum_j p |v| [rows, H, dh] and the largest sum |q||k| scale."""
    rows, H, dh = q.shape
    n, kv, _ = k.shape
    out, mag, p = np.zeros((rows, H, dh)), np.zeros((rows, H, dh)), np.zeros((rows, H, n))
    reach = 0.0
    for h in range(H if n else 0):
        g = h // (H // kv)
        s = q[:, h] @ k[:, g].T * scale
        reach = max(reach, float((np.abs(q[:, h]) @ np.abs(k[:, g]).T).max()) * scale) if rows else reach
        e = np.exp(s - s.max(axis=1, keepdims=True))
        p[:, h] = e / e.sum(axis=1, keepdims=True)
        out[:, h] = p[:, h] @ v[:, g]
        mag[:, h] = p[:, h] @ np.abs(v[:, g])
    return out, p, mag, reach


def evict(weight, token, budget, protect_from=None):
    """Slots of one request.  Returns (new length, [(source slot, destination slot), ..])."""
    n = len(weight)
    keep = min(max(int(budget), 0), n)

    def rank(j):
        w = float(weight[j])
        first = math.isnan(w) or (protect_from is not None and token[j] >= protect_from)
        return (0 if first else 1, 0.0 if first else -w, j)

    kept = set(sorted(range(n), key=rank)[:keep])
    gaps = [j for j in range(keep) if j not in kept]
    movers = [j for j in range(keep, n) if j in kept]
    assert len(gaps) == len(movers)
    return keep, list(zip(movers, gaps))
