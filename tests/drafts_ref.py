"""Plain models of the operators for drafted tokens, for their tests: NumPy, in 64 bits where numbers are added up, in
32 bits with one rounding per operation where the library defines them so, and Python integers."""
import numpy as np

f32 = np.float32


# ------------------------------------------------------------------ e4m3
def e4m3_values():
    """The 256 codes' values: sign, four bits of exponent (bias 7), three of mantissa; 0x7f and 0xff are NaN."""
    out = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
        out[c] = np.nan if (c & 127) == 127 else -v if c & 128 else v
    return out


E4M3 = e4m3_values()
_POSITIVE = E4M3[:127]  # rising


def e4m3(v):
    """Values of v rounded to the nearest code, ties to even codes, limited to +-448."""
    v = np.asarray(v, np.float64)
    a = np.minimum(np.abs(v), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    x, y = _POSITIVE[lo], _POSITIVE[hi]
    up = (a - x > y - a) | ((a - x == y - a) & (hi % 2 == 0))
    r = np.where(up, y, x)
    return np.where(np.isnan(v), np.nan, np.copysign(r, v))


def quantize(x, rows):
    """(values of the codes, scales) of x [n, k] in fp32 by blocks of `rows` x 128."""
    n, k = x.shape
    nb, kb = -(-n // rows), -(-k // 128)
    q, s = np.zeros((n, k)), np.zeros((nb, kb), f32)
    with np.errstate(all="ignore"):
        for i in range(nb):
            for j in range(kb):
                at = np.s_[i * rows:(i + 1) * rows, 128 * j:128 * (j + 1)]
                a = np.abs(x[at]).max()
                s[i, j] = np.nan if np.isnan(a) else max(f32(a) * f32(1 / 448), f32(2.0 ** -100))
                q[at] = e4m3((x[at] * (f32(1) / s[i, j])).astype(f32))
    return q, s


# ------------------------------------------------------------------ probabilities
def probs(x, temperature, min_p):
    """x [T, V] fp32 values -> [T, V] float64."""
    out = np.zeros(x.shape)
    least = f32(np.log(min_p)) if min_p else f32(-np.inf)
    with np.errstate(all="ignore"):
        for r in range(x.shape[0]):
            t, best = f32(temperature[r]), x[r].max()
            if np.isnan(t) or np.isnan(best):
                out[r] = np.nan
            elif best == -np.inf:  # nothing is open
                out[r] = np.nan
            elif not t > 0:
                out[r, np.argmax(x[r])] = 1
            else:
                z = (x[r] - best) * (f32(1) / max(t, f32(2.0 ** -120)))
                keep = z >= least
                y = (x[r].astype(np.float64) - best) / max(float(t), 2.0 ** -120)
                e = np.where(keep, np.exp(y), 0.0)
                out[r] = e / e.sum() if keep.any() else np.nan
    return out


# ------------------------------------------------------------------ verification
def weights(w):
    """floor(2^40 w) of w limited to [0, 1], NaN as 0, as Python integers."""
    w = np.nan_to_num(np.asarray(w, f32), nan=0.0, posinf=1.0, neginf=0.0)
    return [int(v) for v in np.floor(np.clip(w, 0, 1).astype(np.float64) * 2.0 ** 40)]


def draw(w, u):
    u24 = int(np.floor(min(max(float(u), 0.0), 1 - 2.0 ** -24) * 2 ** 24)) if u == u else 0
    total = sum(w)
    if total == 0:
        return -1
    t = (total * u24) >> 24
    up = 0
    for v, x in enumerate(w):
        up += x
        if up > t:
            return v


def verify(p, q, ids, cu, drafts, accept, sample):
    """(accepted, rejected, next) as lists; p, q fp32 values [T, V], q may be None."""
    out = ([], [], [])
    v = p.shape[1]
    with np.errstate(all="ignore"):
        for b, n in enumerate(drafts):
            r0, r1 = cu[b], cu[b + 1]
            if r0 == r1 or not (0 <= r0 <= r1 <= p.shape[0] and 0 <= n < r1 - r0):
                for o, x in zip(out, (0, 0, -1)):
                    o.append(x)
                continue
            first, a = r1 - 1 - n, 0
            while a < n:
                d, row = ids[first + a + 1], first + a
                if not 0 <= d < v:
                    break
                asked = f32(1) if q is None else q[row, d]
                if not f32(accept[row]) * asked < p[row, d]:
                    break
                a += 1
            row, rest = first + a, p[first + a]
            if a < n:
                other = np.zeros(v, f32)
                if q is not None:
                    other = q[row]
                elif 0 <= ids[row + 1] < v:
                    other[ids[row + 1]] = 1
                rest = (p[row] - other).astype(f32)
                if not any(weights(rest)):
                    rest = p[row]
            for o, x in zip(out, (a, n - a, draw(weights(rest), sample[b]))):
                o.append(x)
    return out


# ------------------------------------------------------------------ tokens taken back
def retract(cached, drop, table, free, page):
    """(lens, free) after it, or None where the library refuses; `free` is the stack up to its height."""
    if any(c < 0 or d < 0 or d > c for c, d in zip(cached, drop)):
        return None
    free = list(free)
    lens = [c - d for c, d in zip(cached, drop)]
    for b, (c, n) in enumerate(zip(cached, lens)):
        free += list(table[b][-(-n // page):-(-c // page)])
    return lens, free
