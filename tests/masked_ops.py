"""Plain 64-bit forms of windows with sinks and of drafted trees, and drafted trees to run them on."""
import numpy as np
import torch

import plain_ops as P


def attention(q, k, v, seen):
    """softmax over the seen tokens: q [n][Hq][D], k and v [tokens][Hkv][D] float64, seen [n][tokens]; rows that see nothing are zeros.  Also
    how far fp32 sums with probabilities of 16 significant bits may be off, element by element, as derived at plain_ops.attention: relative to
    sum_t p_t |v_t|, 2^-16 and 2^-19 of the largest sum |q k| / sqrt(D) of a seen token."""
    n, hq, d = q.shape
    hkv, g = k.shape[1], q.shape[1] // k.shape[1]
    out, tol = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    if not seen.any():
        return out, tol
    # (what no row sees may hold anything)
    some = seen.any(axis=0)
    k, v, seen = k[some], v[some], seen[:, some]
    for j in range(hq):
        h = j // g
        z = np.where(seen, q[:, j] @ k[:, h].T / np.sqrt(d), -np.inf)
        far = np.where(seen, np.abs(q[:, j]) @ np.abs(k[:, h]).T / np.sqrt(d), 0.0).max(axis=1, keepdims=True)
        m = z.max(axis=1, keepdims=True)
        p = np.exp(z - np.where(np.isfinite(m), m, 0.0))
        den = p.sum(axis=1, keepdims=True)
        p = np.divide(p, den, out=np.zeros_like(p), where=den > 0)
        out[:, j] = p @ v[:, h]
        tol[:, j] = (2.0 ** -16 + 2.0 ** -19 * far) * (p @ np.abs(v[:, h]))
    return out, tol


def window_seen(ctx, n, window, sinks):
    """Which of a row's ctx tokens its last n queries see."""
    p, t = np.arange(ctx - n, ctx)[:, None], np.arange(max(ctx, 0))[None]
    return (t <= p) & ((t > p - window) | (t < sinks))


def tree_seen(ctx, masks, window, sinks):
    """The same of drafted tokens with masks (ints), the last of the row's ctx tokens."""
    n = len(masks)
    base, t = ctx - n, np.arange(max(ctx, 0))
    if base < 0:
        return np.zeros((n, max(ctx, 0)), dtype=bool)
    seen = np.zeros((n, ctx), dtype=bool)
    for i, m in enumerate(masks):
        m &= (1 << n) - 1
        p = base + max(bin(m).count("1") - 1, 0)
        seen[i] = (t < base) & ((t > p - window) | (t < sinks) | (window == 0))
        seen[i, base:] = [bool(m >> j & 1) for j in range(n)]
    return seen


def positions(masks):
    return [max(bin(m & (1 << len(masks)) - 1).count("1") - 1, 0) for m in masks]


def random_tree(rng, n, branch):
    """Masks of n drafted tokens: each continues the one before or, with probability `branch`, any earlier one or the context."""
    masks = []
    for i in range(n):
        p = i - 1 if rng.random() >= branch else int(rng.integers(-1, i)) if i else -1
        masks.append(1 << i | (masks[p] if p >= 0 else 0))
    return masks


def path_of(mask):
    return [j for j in range(mask.bit_length()) if mask >> j & 1]


def words_of(masks, words):
    """int64 [tokens][words] on the GPU."""
    rows = np.array([[(m >> 64 * w) & ((1 << 64) - 1) for w in range(words)] for m in masks], dtype=np.uint64).reshape(len(masks), words)
    return torch.from_numpy(rows.view(np.int64)).cuda()


def check(got, q, row_of, n, seen_of):
    """got [sum n][Hq][D] float64 against rows of row_of(s) -> (k, v); n: query tokens of each sequence."""
    at = 0
    for s, m in enumerate(n):
        k, v = row_of(s)
        seen = seen_of(s)
        want, tol = attention(P.f64(q[at:at + m]), k[:seen.shape[1]], v[:seen.shape[1]], seen)
        err = np.abs(got[at:at + m] - want)
        assert np.all(err <= tol + 1e-30), (s, m, float((err / np.maximum(tol, 1e-30)).max()), np.argwhere(~(err <= tol + 1e-30))[:3].tolist())
        at += m


def same(a, b, q, row_of, n, seen_of):
    """Two calls' outputs: either is within the tolerance of 64 bits, so they are within twice that of each other."""
    at, diff = 0, (a - b).abs().cpu().double().numpy()
    for s, m in enumerate(n):
        k, v = row_of(s)
        seen = seen_of(s)
        _, tol = attention(P.f64(q[at:at + m]), k[:seen.shape[1]], v[:seen.shape[1]], seen)
        assert np.all(diff[at:at + m] <= 2.0 * tol), (s, float((diff[at:at + m] / np.maximum(tol, 1e-30)).max()))
        at += m
