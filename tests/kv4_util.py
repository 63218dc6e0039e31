"""The 4-bit key/value cache by its definition, in numpy and 64 bits on the CPU: shares no
code with the library."""
import numpy as np
import torch

PAGE = 64
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# the largest relative error of rounding to nearest with p significant bits: 2^-p
HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def quantise(x):
    """float64 [..., D] -> codes uint8 [..., D], scale bytes uint8 [..., D/32], finite [..., D/32]."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(x.shape[:-1] + (-1, 32))
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[..., None], g, 0.0)
    top = np.abs(g).max(-1)
    e = np.frexp(top)[1] - 1 - 2                       # frexp's mantissa is in [0.5, 1)
    e = np.where(top == 0, -127, np.maximum(e, -127))
    y = np.abs(g) / np.exp2(e.astype(np.float64))[..., None]
    dist = np.abs(y[..., None] - E2M1)
    # nearest, and of two equally near the even code
    best = np.argmin(dist + np.where(np.arange(8) % 2 == 1, 1e-300, 0.0), -1)
    tie = (dist == dist.min(-1, keepdims=True))
    even = tie & (np.arange(8) % 2 == 0)
    best = np.where(even.any(-1), np.argmax(even, -1), best)
    codes = best + 8 * np.signbit(g)
    byte = np.where(fine, e + 127, 255)
    codes = np.where(fine[..., None], codes, 0)
    return codes.reshape(x.shape).astype(np.uint8), byte.astype(np.uint8), fine


def values(codes, byte):
    """What codes and scale bytes stand for, float64."""
    c = codes.reshape(codes.shape[:-1] + (-1, 32))
    v = np.where(c >= 8, -1.0, 1.0) * E2M1[c & 7]
    s = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    return (v * s[..., None]).reshape(codes.shape)


def quantise_pair(k, v):
    """Key and value parts with the rule for tokens that hold no number."""
    kc, ks, kf = quantise(k)
    vc, vs, vf = quantise(v)
    fine = (kf.all(-1) & vf.all(-1))[..., None]
    return np.where(fine, kc, 0), np.where(fine, ks, 255).astype(np.uint8), vc, vs


class Cache:
    """pages x heads of records, as lce.h lays them out; written token by token."""

    def __init__(self, pages, heads, dim, fill=0xFF):
        self.pages, self.heads, self.dim = pages, heads, dim
        self.data = np.full((pages, heads, 76 * dim), fill, dtype=np.uint8)

    def places(self, t):
        """Byte offsets of token t's key codes, value codes, key scales, value scales, signs."""
        d = self.dim
        c = np.arange(0, d, 2)
        k = t * d // 2 + c // 2
        r, w = c // (d // 16), c % (d // 16)
        v = 32 * d + ((t // 4 * 16 + r) * 4 + t % 4) * (d // 32) + w // 2
        g = np.arange(d // 32)
        ks = 64 * d + (t % 16 * (d // 32) + g) * 4 + t // 16
        vs = 66 * d + g * 64 + t % 16 // 4 * 16 + t // 16 * 4 + t % 4
        s = 68 * d + t * d // 8 + np.arange(d // 8)
        return k, v, ks, vs, s

    def write(self, slot, k, v):
        """k, v [heads, dim] into one slot."""
        page, t = divmod(int(slot), PAGE)
        kc, ks, vc, vs = quantise_pair(k, v)
        at = self.places(t)
        rec = self.data[page]
        rec[:, at[0]] = kc[:, 0::2] | kc[:, 1::2] << 4
        rec[:, at[1]] = vc[:, 0::2] | vc[:, 1::2] << 4
        rec[:, at[2]] = ks
        rec[:, at[3]] = vs
        rec[:, at[4]] = np.packbits(np.asarray(k) < 0, axis=-1, bitorder="little")

    def read(self, slot):
        page, t = divmod(int(slot), PAGE)
        at = self.places(t)
        rec = self.data[page]
        out = []
        for codes, scales in ((at[0], at[2]), (at[1], at[3])):
            b = rec[:, codes]
            c = np.stack((b & 15, b >> 4), -1).reshape(self.heads, self.dim)
            out.append(values(c, rec[:, scales]))
        return out

    def signs(self, slot):
        page, t = divmod(int(slot), PAGE)
        bits = np.unpackbits(self.data[page][:, self.places(t)[4]], axis=-1, bitorder="little")
        return 1 - 2 * bits.astype(np.int64)


class Batch:
    """Sequences of given lengths on shuffled pages; table entries past a length are junk."""

    def __init__(self, seed, lengths, queries, q_heads, kv_heads, dim, dtype, width=None,
                 spare=3, odd=()):
        rng = np.random.default_rng(seed)
        self.rng, self.lengths, self.queries = rng, list(lengths), list(queries)
        self.q_heads, self.kv_heads, self.dim, self.dtype = q_heads, kv_heads, dim, dtype
        used = [-(-n // PAGE) for n in lengths]
        self.cache = Cache(sum(used) + spare, kv_heads, dim)
        order = rng.permutation(self.cache.pages)
        width = max(1, max(used)) if width is None else width
        self.table = rng.integers(-2 ** 31, 2 ** 31 - 1, (len(lengths), width)).astype(np.int32)
        at = 0
        self.k, self.v, self.sign = [], [], []
        for b, n in enumerate(lengths):
            pages = order[at:at + used[b]]
            self.table[b, :used[b]] = pages
            at += used[b]
            k = rng.standard_normal((n, kv_heads, dim)) * np.where(np.arange(dim) % 29 == 3, 3, 1)
            v = rng.standard_normal((n, kv_heads, dim))
            for (ob, oj, oh, oc, which, what) in odd:
                if ob == b:
                    (k if which == "k" else v)[oj, oh, oc] = what
            ks, vs, ss = [], [], []
            for j in range(n):
                slot = pages[j // PAGE] * PAGE + j % PAGE
                self.cache.write(slot, k[j], v[j])
                a, c = self.cache.read(slot)
                ks.append(a)
                vs.append(c)
                ss.append(self.cache.signs(slot))
            shape = (n, kv_heads, dim)
            self.k.append(np.array(ks).reshape(shape))
            self.v.append(np.array(vs).reshape(shape))
            self.sign.append(np.array(ss, dtype=np.int64).reshape(shape))
        self.start = np.concatenate(([0], np.cumsum(queries))).astype(np.int32)
        self.tokens = int(self.start[-1])
        self.q = torch.from_numpy(rng.standard_normal((self.tokens, q_heads, dim))).to(DTYPES[dtype])

    def sees(self, b, i, causal, window):
        n = self.lengths[b]
        j = np.arange(n)
        p = n - self.queries[b] + i
        m = j <= p if causal else np.ones(n, bool)
        return m & (j > p - window) if window else m

    def attention(self, scale, causal=True, window=0, pages=None):
        """out, lse and the error bounds that go with them (see error_bounds)."""
        g = self.q_heads // self.kv_heads
        out = np.zeros((self.tokens, self.q_heads, self.dim))
        lse = np.full((self.tokens, self.q_heads), -np.inf)
        bound, lse_bound = np.zeros_like(out), np.zeros_like(lse)
        q = self.q.double().numpy()
        for b in range(len(self.lengths)):
            for i in range(self.queries[b]):
                t = self.start[b] + i
                for h in range(self.q_heads):
                    hk = h // g
                    m = self.sees(b, i, causal, window)
                    if pages is not None:
                        m = m & np.isin(np.arange(len(m)) // PAGE, pages[t, hk][pages[t, hk] >= 0])
                    if not m.any():
                        continue
                    k, v = self.k[b][m, hk], self.v[b][m, hk]
                    s = scale * (k @ q[t, h])
                    top = s.max()
                    p = np.exp(s - top)
                    lse[t, h] = top + np.log(p.sum())
                    w = p / p.sum()
                    out[t, h] = w @ v
                    self._bounds(bound[t, h], w, v, out[t, h],
                                 scale * (np.abs(k) @ np.abs(q[t, h])).max(), lse[t, h])
                    lse_bound[t, h] = self._lse_bound
        return out, lse, bound, lse_bound

    def _bounds(self, bound, w, v, out, reach, lse):
        """Errors allowed.  A score's products are exact and summed in float32, at most
        dim + 3 additions of terms whose absolute values add up to `reach`: off by
        dim * 2^-24 * reach, twice that with the subtraction of the maximum and the
        exponential's own last place.  Each weight is off by that and by half a unit of its
        type where it is rounded, the result by half a unit of its type, and sums of n
        float32 terms by n * 2^-24 of the sum of their absolute values."""
        u = HALF_ULP[self.dtype]
        n = len(w)
        score = 2 * (self.dim + 8) * 2.0 ** -24 * (reach + 1) + 4 * 2.0 ** -24
        mass = w @ np.abs(v)
        bound += (u + 2 * score + 2 * (n + 64) * 2.0 ** -24) * mass + u * 1.01 * np.abs(out)
        if self.dtype == "f16":         # weights and results below 2^-14 have a fixed last place
            bound += 2.0 ** -25 * (np.abs(v).sum(0) + 1)
        self._lse_bound = score + (n + 64) * 2.0 ** -24 + 2.0 ** -22 * (1 + abs(lse))

    def select(self, count, keep_first=1, keep_last=1, causal=True, window=0):
        g = self.q_heads // self.kv_heads
        qs = np.where(self.q.double().numpy() < 0, -1, 1).astype(np.int64)
        res = np.full((self.tokens, self.kv_heads, count), -1, np.int32)
        for b in range(len(self.lengths)):
            for i in range(self.queries[b]):
                t = self.start[b] + i
                m = self.sees(b, i, causal, window)
                up = np.nonzero(self.sees(b, i, causal, 0))[0]
                pages = 0 if not len(up) else up[-1] // PAGE + 1
                for h in range(self.kv_heads):
                    s = (self.sign[b][:, h] @ qs[t, h * g:(h + 1) * g].T).sum(-1) if len(m) else []
                    rank = []
                    for pg in range(pages):
                        mine = np.nonzero(m[pg * PAGE:(pg + 1) * PAGE])[0] + pg * PAGE
                        if not len(mine):
                            continue
                        kept = pg < keep_first or pg >= pages - keep_last
                        rank.append((not kept, 0 if kept else -max(s[mine]), pg))
                    best = sorted(pg for _, _, pg in sorted(rank)[:count])
                    res[t, h, :len(best)] = best
        return res

    def device(self, lce):
        """(cache, q, table, q_start, lengths) on the GPU."""
        c = lce.KV4Cache(self.kv_heads, self.dim, data=torch.from_numpy(self.cache.data).cuda())
        return (c, self.q.cuda(), torch.from_numpy(self.table).cuda(),
                torch.from_numpy(self.start).cuda(),
                torch.tensor(self.lengths, dtype=torch.int32).cuda())
