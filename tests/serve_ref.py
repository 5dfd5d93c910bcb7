"""Plain models of the serving operators for their tests: NumPy in 64 bits (attention, log
probabilities), NumPy in 32 bits with one rounding per operation (norms, rotation, 4-bit rows, which
the library defines bit for bit), and Python integers (tables)."""
import numpy as np

from paper_2405_03594_gb300 import synth

f32 = np.float32


# ------------------------------------------------------------------ tables
class Tables:
    """The tables of include/sp_serve.h on the host."""

    def __init__(self, cached, table, free, page, max_tokens):
        self.cached, self.table, self.free = list(cached), [list(r) for r in table], list(free)
        self.page, self.max_tokens = page, max_tokens

    def step(self, new, allocate=True):
        """(lens, cu_q, slots, positions, table, free, status); `free` is the stack up to its height."""
        page, pages_of = self.page, lambda n: -(-n // self.page)
        width = len(self.table[0]) if self.table else 0
        lens = [0 if a < 0 else c + a for c, a in zip(self.cached, new)]
        need = [0 if a < 0 else pages_of(n) - pages_of(c) for c, a, n in zip(self.cached, new, lens)]
        back = [pages_of(c) if a < 0 else 0 for c, a in zip(self.cached, new)]
        total = sum(a for a in new if a > 0)
        status = 0
        if allocate and sum(need) > len(self.free) + sum(back):
            status |= 1
        if any(n > width * page for n in lens):
            status |= 2
        if total > self.max_tokens:
            status |= 4
        slots, pos = [-1] * self.max_tokens, [0] * self.max_tokens
        table, free = [list(r) for r in self.table], list(self.free)
        if status:
            return self.cached, [0] * (len(new) + 1), slots, pos, table, free, status
        if allocate:
            for b, n in enumerate(back):
                free += table[b][:n]
            for b, n in enumerate(need):
                for j in range(n):
                    table[b][pages_of(self.cached[b]) + j] = free.pop()
        cu = [0]
        for b, a in enumerate(new):
            for i in range(max(a, 0)):
                p = self.cached[b] + i
                slots[cu[-1] + i] = table[b][p // page] * page + p % page
                pos[cu[-1] + i] = p
            cu.append(cu[-1] + max(a, 0))
        return lens, cu, slots, pos, table, free, 0


# ------------------------------------------------------------------ norms, rotation, 4-bit rows
def norm(x, w, eps):
    y = x * x
    while y.shape[-1] > 1:
        y = y[..., 0::2] + y[..., 1::2]
    r = f32(1) / np.sqrt(y * f32(1 / x.shape[-1]) + f32(eps))
    return x * r * w


def rotate(x, cos, sin, pairs):
    """x [T, H, D]; cos, sin [T, rot / 2]."""
    half = cos.shape[-1]
    out = x.copy()
    c, s = cos[:, None, :], sin[:, None, :]
    lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., lo], x[..., hi]
    out[..., lo] = a * c - b * s
    out[..., hi] = b * c + a * s
    return out


def quantize(x):
    """(codes uint8, scale fp16, minimum fp16) of fp32 rows."""
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
        bad = ~np.isfinite(x).all(-1, keepdims=True)
        lo, hi = np.clip(lo, f32(-32768), f32(32768)), np.clip(hi, f32(-32768), f32(32768))
        m = np.where(bad, f32(np.nan), lo).astype(np.float16)
        s = np.where(bad, f32(0), (hi - lo) * f32(1 / 15)).astype(np.float16)
        sf, mf = s.astype(f32), m.astype(f32)
        n = np.clip(np.rint((x - mf) * (f32(1) / sf)), f32(0), f32(15))
        n = np.where(sf > 0, n, f32(0))
    return n.astype(np.uint8), s[..., 0], m[..., 0]


def values(n, s, m):
    return s[..., None].astype(np.float64) * n + m[..., None].astype(np.float64)


def pack(kn, ks, km, vn, vs, vm):
    """The cache's bytes from codes [pages, heads, P, D] and parameters [pages, heads, P]."""
    pages, heads = kn.shape[:2]
    rows = [(n[..., 0::2] | (n[..., 1::2] << 4)).reshape(pages, heads, -1) for n in (kn, vn)]
    pars = [np.ascontiguousarray(np.stack([s, m], -1)).view(np.uint8).reshape(pages, heads, -1) for s, m in ((ks, km), (vs, vm))]
    return np.concatenate(rows + pars, -1).reshape(-1)


def unpack(data, pages, heads, page, dim):
    """The inverse of pack."""
    b = data.reshape(pages, heads, page * (dim + 8))
    out, at = [], 0
    for _ in range(2):
        c = b[..., at:at + page * dim // 2].reshape(pages, heads, page, dim // 2)
        n = np.empty((pages, heads, page, dim), np.uint8)
        n[..., 0::2], n[..., 1::2] = c & 15, c >> 4
        out.append(n)
        at += page * dim // 2
    for i in range(2):
        p = np.ascontiguousarray(b[..., at:at + 4 * page]).view(np.float16).reshape(pages, heads, page, 2)
        out += [p[..., 0], p[..., 1]]
        at += 4 * page
    kn, vn, ks, km, vs, vm = out
    return kn, ks, km, vn, vs, vm


# ------------------------------------------------------------------ attention
def attend(q, k, v, scale):
    """q [a, H, D] float64, the last a tokens of k, v [L, Hkv, D]; causal."""
    a, heads, _ = q.shape
    n, kv, _ = k.shape
    out = np.zeros(q.shape)
    seen = n - a + np.arange(a) + 1
    for h in range(heads):
        x = scale * (q[:, h] @ k[:, h * kv // heads].T)
        x = np.where(np.arange(n)[None, :] < seen[:, None], x, -np.inf)
        for i in range(a):
            if seen[i] <= 0:
                continue
            y = x[i, :seen[i]]
            if np.isnan(y).any():
                out[i, h] = np.nan
                continue
            e = np.exp(y - y.max())
            out[i, h] = (e / e.sum()) @ v[:seen[i], h * kv // heads]
    return out


# ------------------------------------------------------------------ log probabilities
def logprobs(x, ids, top):
    """x [T, V] float64 -> (logp, entropy, top logp, top ids)."""
    t, v = x.shape
    logp, ent = np.zeros(t), np.zeros(t)
    tl, ti = np.zeros((t, top)), np.zeros((t, top), np.int64)
    for r in range(t):
        y = x[r]
        if np.isnan(y).any() or (y == np.inf).any():
            lp = np.full(v, np.nan)
            ent[r] = np.nan
        elif (y == -np.inf).all():
            lp = np.full(v, -np.inf)
        else:
            m = y.max()
            lp = y - m - np.log(np.exp(y - m).sum())
            p = np.exp(lp)
            ent[r] = -(p[p > 0] * lp[p > 0]).sum()
        logp[r] = 0 if ids[r] < 0 else lp[ids[r]] if ids[r] < v else np.nan
        key = np.where(np.isnan(y), np.inf, y)
        order = np.lexsort((np.arange(v), -key, ~np.isnan(y)))[:top]
        tl[r], ti[r] = lp[order], order
    return logp, ent, tl, ti


def bf16(x):
    """float32 values and bits of x rounded to bf16."""
    u = synth.bf16_from_f32(np.asarray(x, f32))
    return synth.bf16_to_f32(u), u
