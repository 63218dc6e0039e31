"""The 8-bit key/value cache and rotary positions by their definitions, in numpy and 64 bits
on the CPU: shares no code with the library."""
from fractions import Fraction

import numpy as np
import torch

PAGE, BLOCK = 64, 16
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# half a step of rounding to nearest, relative to the value
HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def _table():
    v = np.zeros(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        x = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[b] = np.nan if b & 127 == 127 else (-x if b >> 7 else x)
    return v


E4M3 = _table()
_UP = E4M3[:127]                                   # ascending, 0 .. 448


def encode(x):
    """The nearest code to each of x (at most 448), ties to the even one, signs kept."""
    a = np.abs(np.asarray(x, np.float64))
    hi = np.searchsorted(_UP, a).clip(0, 126)
    lo = (hi - 1).clip(0)
    dl, dh = a - _UP[lo], _UP[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def scale_exponent(top):
    """The smallest e >= -126 with top <= 448 * 2^e."""
    e = -126
    while top > np.ldexp(448.0, e):
        e += 1
    return e


class Cache:
    """pages x heads of records, as lce.h lays them out."""

    def __init__(self, pages, heads, dim, fill=0xFF):
        self.pages, self.heads, self.dim = pages, heads, dim
        self.data = np.full((pages, heads, 128 * dim + 128), fill, np.uint8)

    def at(self, t, part):
        """Byte offsets of token t's codes, and of its scale."""
        c, d = np.arange(self.dim), self.dim
        return (64 * d + (t // 4 * d + c) * 4 + t % 4 if part else t * d + c,
                128 * d + 4 * part + t // BLOCK)

    def append(self, table, length, k, v):
        """k, v [n, heads, dim] become the last tokens of a sequence."""
        n = len(k)
        new = {length - n + i: i for i in range(n) if length - n + i >= 0}
        for b0 in sorted({p // BLOCK * BLOCK for p in new}):
            page = table[b0 // PAGE]
            if not 0 <= page < self.pages:
                continue
            held = [p for p in range(b0, b0 + BLOCK) if p < max(length - n, 0)]
            mine = [p for p in range(b0, b0 + BLOCK) if p in new]
            for h in range(self.heads):
                odd = {p for p in mine
                       if not (np.isfinite(k[new[p], h]).all() and np.isfinite(v[new[p], h]).all())}
                for part, x in enumerate((k, v)):
                    rows = {p: np.asarray(x[new[p], h], np.float64) for p in mine}
                    if part:
                        rows = {p: np.where(np.isfinite(r), r, 0.0) for p, r in rows.items()}
                    else:
                        rows = {p: r for p, r in rows.items() if p not in odd}
                    e = scale_exponent(max([np.abs(r).max() for r in rows.values()] + [0.0]))
                    rec, was = self.data[page, h], None
                    _, sc = self.at(b0 % PAGE, part)
                    if held:
                        was = int(np.clip(rec[sc], 1, 247)) - 127
                        e = max(e, was)
                        if e > was:
                            for p in held:
                                at, _ = self.at(p % PAGE, part)
                                val = E4M3[rec[at]]
                                again = encode(np.where(np.isnan(val), 0, val) * 2.0 ** (was - e))
                                rec[at] = np.where(np.isnan(val), rec[at], again)
                    rec[sc] = e + 127
                    for p in mine:
                        at, _ = self.at(p % PAGE, part)
                        rec[at] = 0x7F if p in odd and not part else encode(np.ldexp(rows[p], -e))
                    if part:                       # words of four tokens are written whole
                        last = max(mine) % PAGE
                        for t in range(last + 1, last // 4 * 4 + 4):
                            rec[self.at(t, part)[0]] = 0

    def read(self, slot):
        """Keys and values [heads, dim] of a slot."""
        page, t = divmod(int(slot), PAGE)
        out = []
        for part in range(2):
            at, sc = self.at(t, part)
            out.append(np.ldexp(E4M3[self.data[page][:, at]],
                                self.data[page][:, sc].astype(np.int64)[:, None] - 127))
        return out


class Batch:
    """Sequences of given lengths on shuffled pages; table entries past a length are junk, and
    so is what the cache holds behind the last tokens."""

    def __init__(self, seed, lengths, queries, q_heads, kv_heads, dim, dtype, width=None, loud=None,
                 odd=(), spread=0.0):
        rng = np.random.default_rng(seed)
        self.rng, self.lengths, self.queries = rng, list(lengths), list(queries)
        self.q_heads, self.kv_heads, self.dim, self.dtype = q_heads, kv_heads, dim, dtype
        used = [-(-n // PAGE) for n in lengths]
        self.cache = Cache(sum(used) + 3, kv_heads, dim)
        order = rng.permutation(self.cache.pages)
        width = max(1, max(used)) if width is None else width
        self.table = rng.integers(-2 ** 31, 2 ** 31 - 1, (len(lengths), width)).astype(np.int32)
        at, self.k, self.v = 0, [], []
        for b, n in enumerate(lengths):
            self.table[b, :used[b]] = order[at:at + used[b]]
            at += used[b]
            k, v = (rng.standard_normal((n, kv_heads, dim)) for _ in range(2))
            if spread:
                # blocks of very different sizes
                size = np.repeat(rng.uniform(-spread, spread, (n // BLOCK + 1, kv_heads, 1)), BLOCK, 0)
                v *= np.exp2(np.round(size[:n]))
                k *= np.exp2(np.round(size[:n] / 8))
            for (ob, oj, oh, oc, which, what) in odd:
                if ob == b:
                    (k if which == "k" else v)[oj, oh, oc] = what
            if n:
                self.cache.append(self.table[b], n, k, v)
            both = [self.cache.read(self.table[b, j // PAGE] * PAGE + j % PAGE) for j in range(n)]
            shape = (n, kv_heads, dim)
            self.k.append(np.array([x[0] for x in both]).reshape(shape))
            self.v.append(np.array([x[1] for x in both]).reshape(shape))
        self.start = np.concatenate(([0], np.cumsum(queries))).astype(np.int32)
        self.tokens = int(self.start[-1])
        q = rng.standard_normal((self.tokens, q_heads, dim)) * (loud or 1.0)
        self.q = torch.from_numpy(q).to(DTYPES[dtype])

    def sees(self, b, i, causal, window, prefix):
        n = self.lengths[b]
        j = np.arange(n)
        p = n - self.queries[b] + i
        m = (j <= p) | (j < (prefix[b] if prefix is not None else 0)) if causal else np.ones(n, bool)
        return m & (j > p - window) if window else m

    def attention(self, scale, causal=True, window=0, cap=0.0, slopes=None, prefix=None,
                  weights=None):
        """out, lse and what they may be off by.

        A score's products are exact (float16: of keys held to 2^-33 of their page's largest
        scale) and summed in float32, at most dim + 3 additions of terms whose absolute
        values add up to `reach`; with the subtraction of the maximum and the exponential's
        last place off by 2 * (dim + 8) * 2^-24 * (reach + 1).  A cap adds its exponential
        and reciprocal (a last place each of 1 - 2/(e + 1), in all 2^-21 of the cap), a
        slope its own rounding and the product's, 2^-22 of the bias.  Each weight is off by
        its score's error and by half a unit of its type where it is rounded (or by `weights`), the
        result by
        half a unit of its type, sums of n float32 terms by n * 2^-24 of the sum of their
        absolute values.  float16 weights have a last place of 2^-31 of the largest,
        values one of 2^-32 of the largest scale, results one of 2^-24."""
        g, u = self.q_heads // self.kv_heads, HALF_ULP[self.dtype]
        half = self.dtype == "f16"
        out = np.zeros((self.tokens, self.q_heads, self.dim))
        lse = np.full((self.tokens, self.q_heads), -np.inf)
        bound, lse_bound = np.zeros_like(out), np.zeros_like(lse)
        q = self.q.double().numpy()
        for b in range(len(self.lengths)):
            n = self.lengths[b]
            for i in range(self.queries[b]):
                t, p = self.start[b] + i, n - self.queries[b] + i
                for h in range(self.q_heads):
                    m = self.sees(b, i, causal, window, prefix)
                    if not m.any():
                        continue
                    k, v, j = self.k[b][m, h // g], self.v[b][m, h // g], np.nonzero(m)[0]
                    with np.errstate(invalid="ignore"):
                        s = scale * (k @ q[t, h])
                        reach = scale * (np.abs(k) @ np.abs(q[t, h]))
                        err = 2 * (self.dim + 8) * 2.0 ** -24 * (reach + 1)
                        if half:
                            far = scale * np.abs(q[t, h]).sum() * np.abs(k).max() / 224
                            err = err + 2.0 ** -33 * far
                        if cap:
                            s = cap * np.tanh(s / cap)
                            err = err + 2.0 ** -21 * cap
                        if slopes is not None:
                            bias = float(slopes[h]) * np.abs(p - j)
                            s = s - bias
                            err = err + 2.0 ** -22 * np.abs(bias)
                        top = s.max()
                        e = np.exp(s - top)
                        lse[t, h] = top + np.log(e.sum())
                        w = e / e.sum()
                        out[t, h] = w @ v
                        # (a mean's error is at most twice that of its weights times the values)
                        rel = (np.expm1(err) + (u if weights is None else weights)
                               + (len(w) + 64) * 2.0 ** -24)
                        mean = np.abs(w @ v)
                        bound[t, h] = (w * rel) @ np.abs(v) + (w @ rel) * mean + u * 1.01 * mean
                        if half:
                            low = 2.0 ** -32 * w.max()
                            bound[t, h] += (low * np.abs(v).sum(0) + low * len(w) * mean
                                            + 2.0 ** -33 * np.abs(v).max() / 224 + 2.0 ** -25)
                        lse_bound[t, h] = (w @ np.expm1(err) + (len(w) + 64) * 2.0 ** -24
                                           + 2.0 ** -22 * (1 + abs(lse[t, h])))
        return out, lse, bound, lse_bound

    def device(self, lce):
        """(cache, q, table, q_start, lengths) on the GPU."""
        c = lce.KV8Cache(self.kv_heads, self.dim, data=torch.from_numpy(self.cache.data).cuda())
        return (c, self.q.cuda(), torch.from_numpy(self.table).cuda(),
                torch.from_numpy(self.start).cuda(),
                torch.tensor(self.lengths, dtype=torch.int32).cuda())


PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def far_angles(positions, freqs):
    """Radians [n, pairs] of any positions: frequencies in turns to the nearest 2^-64, whole
    turns left out, in whole numbers."""
    turns = [round(Fraction(float(f)) / (2 * PI) * 2 ** 64) for f in freqs]
    a = [[(int(p) * t) % 2 ** 64 for t in turns] for p in positions]
    return np.array([[2 * np.pi * (x / 2 ** 64) for x in row] for row in a])


def rotary(x, positions, freqs, scale, interleaved, backward=False):
    """float64 [n, heads, dim] turned, by complex numbers; positions [n], or angles [n, pairs]."""
    r = 2 * len(freqs)
    angles = np.asarray(positions, np.float64)
    if angles.ndim == 1:
        angles = angles[:, None] * np.asarray(freqs)[None]
    turn = scale * np.exp((-1j if backward else 1j) * angles)[:, None]
    y = np.array(x, np.float64)
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    z = (y[..., a] + 1j * y[..., b]) * turn
    y[..., a], y[..., b] = z.real, z.imag
    return y
