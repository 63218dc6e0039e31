"""Attention over the 8-bit cache whose scores float32 holds exactly and whose results are small
beside the values that make them, so that what weights are rounded to shows."""
import numpy as np
import torch

from tests import kv8_util as ref

SCALE = 0.25


def snap(x):
    """To four significant bits, and to what one scale holds of them all: 0, or 2^-7 .. 24."""
    m, e = np.frexp(np.clip(x, -24, 24))
    x = np.ldexp(np.round(m * 16) / 16, e)
    return np.where(np.abs(x) < 2.0 ** -7, 0, x)


def batch(seed, lengths, queries, q_heads, kv_heads, dim, dtype):
    """A Batch with one channel of keys that counts, scores of 0 to -4 in steps of 2^-5, and
    values that sum to about 2^-8 of their absolute values' sum: the last two tokens of each
    channel take back what is left."""
    b = ref.Batch(seed, lengths, queries, q_heads, kv_heads, dim, dtype)
    rng = np.random.default_rng(seed)
    for i, n in enumerate(lengths):
        k = np.zeros((n, kv_heads, dim))
        k[:, :, 3] = -snap(rng.integers(0, 128, (n, kv_heads)) / 8.0)
        w = np.exp(SCALE * k[:, :, 3:4])
        v = snap(rng.uniform(0.5, 2, k.shape) * rng.choice((-1, 1), k.shape))
        # in the order of their weights: the largest ones first, the corrections by middle ones
        for h in range(kv_heads):
            order = np.argsort(-w[:, h, 0], kind="stable")
            order = np.concatenate((np.delete(order, [n // 3, n // 2]), order[[n // 3, n // 2]]))
            left = np.zeros(dim)
            for j in order[:-2]:
                left += w[j, h] * v[j, h]
            for j in order[-2:]:
                v[j, h] = snap(-left / w[j, h])
                left += w[j, h] * v[j, h]
        b.cache.append(b.table[i], n, k, v)
        both = [b.cache.read(b.table[i, j // ref.PAGE] * ref.PAGE + j % ref.PAGE) for j in range(n)]
        b.k[i], b.v[i] = (np.array([x[part] for x in both]) for part in range(2))
        assert np.array_equal(b.k[i], k) and np.array_equal(b.v[i], v)
    q = torch.zeros(b.q.shape, dtype=torch.float64)
    q[..., 3] = 1
    b.q = q.to(b.q.dtype)
    return b


def expected(b, weights):
    """out of every row (none is masked), and what it may be off by where weights are off by
    `weights` of themselves.

    Scores are exact.  Of their product with the scale in log2 units (at most 8) three
    roundings are left, 3 * 2^-21, of the exponential one last place of float32, of sums of n
    terms and of their joining (n + 64) * 2^-24 of their absolute values; the result is rounded
    by half a unit of its type, and float16 has steps of 2^-24."""
    g, u = b.q_heads // b.kv_heads, ref.HALF_ULP[b.dtype]
    out = np.zeros((b.tokens, b.q_heads, b.dim))
    bound, parts = np.zeros_like(out), []
    for i, n in enumerate(b.lengths):
        rel = weights + 3 * 2.0 ** -21 + 2.0 ** -23 + (n + 64) * 2.0 ** -24
        for h in range(b.q_heads):
            k, v = b.k[i][:, h // g], b.v[i][:, h // g]
            w = np.exp(SCALE * k[:, 3])
            mean, size = w @ v / w.sum(), w @ np.abs(v) / w.sum()
            rows = slice(b.start[i], b.start[i + 1])
            out[rows, h] = mean
            bound[rows, h] = rel * (size + np.abs(mean)) + u * 1.01 * np.abs(mean) + 2.0 ** -25
            parts.append((i, h, w, v))
    return out, bound, parts
