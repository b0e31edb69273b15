"""Plain 64-bit forms of the operators between projections and attention, and a small model to run them on."""
import numpy as np
import torch

from workloads import gen

T = 16


def bits(x):
    """float64 numpy -> bf16 bit patterns (through fp32: to nearest even twice differs from once by less than an fp32 step)."""
    return gen.to_bf16_bits(torch.from_numpy(np.ascontiguousarray(x)).float())


def f64(b):
    return gen.bf16_bits_to_f64(b)


def dev(b):
    """bf16 bit patterns on the GPU as int16."""
    return torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).cuda()


def host(t):
    return t.cpu().numpy().view(np.uint16)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def frequencies(rot, base=10000.0):
    return base ** (-2.0 * np.arange(rot // 2) / rot)


def turned(x, pos, weight=None, eps=1e-6, rot=0, pairs=False, freq=None, magnitude=1.0):
    """x [rows][heads][D] float64 at positions pos [rows]: normed and rotated, and the sum of what each element is made of, |a| + |b|
    times the magnitude, which rounding errors are relative to."""
    y = x.copy()
    if weight is not None:
        y = y / np.sqrt((y * y).mean(axis=-1, keepdims=True) + eps) * weight
    size = np.abs(y)
    if rot:
        ang = np.asarray(pos, dtype=np.float64)[:, None] * freq[None]
        c, s = np.cos(ang)[:, None] * magnitude, np.sin(ang)[:, None] * magnitude
        ia, ib = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if pairs else (np.arange(rot // 2), np.arange(rot // 2, rot))
        a, b = y[..., ia].copy(), y[..., ib].copy()
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        size[..., ia] = size[..., ib] = (np.abs(a) + np.abs(b)) * abs(magnitude)
    return y, size


def attention(q, k, v, limits):
    """softmax(q K^T / sqrt(D)) V: q [n][Hq][D], k and v [tokens][Hkv][D] float64; row i sees the first limits[i] tokens, none: zeros.
    Also how far fp32 sums with probabilities of 16 significant bits may be off, element by element: relative to sum_t p_t |v_t|,
    2^-17 for the rounding of p with as much again for exponentials, sums and products, and what a logit is off by, which is some steps
    of 2^-24 of sum |q k| / sqrt(D): 2^-19 of it."""
    n, hq, d = q.shape
    hkv, g = k.shape[1], q.shape[1] // k.shape[1]
    out, tol = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    top = max(limits, default=0)
    if top <= 0:
        return out, tol
    seen = np.arange(top)[None, :] < np.asarray(limits)[:, None]
    for h in range(hkv):
        for j in range(h * g, (h + 1) * g):
            z = np.where(seen, q[:, j] @ k[:top, h].T / np.sqrt(d), -np.inf)
            far = np.where(seen, np.abs(q[:, j]) @ np.abs(k[:top, h]).T / np.sqrt(d), 0.0).max(axis=1, keepdims=True)
            m = z.max(axis=1, keepdims=True)
            p = np.exp(z - np.where(np.isfinite(m), m, 0.0))
            den = p.sum(axis=1, keepdims=True)
            p = np.divide(p, den, out=np.zeros_like(p), where=den > 0)
            out[:, j] = p @ v[:top, h]
            tol[:, j] = (2.0 ** -16 + 2.0 ** -19 * far) * (p @ np.abs(v[:top, h]))
    return out, tol


class Cache:
    """One model on the library whose rows hold `lens` tokens of room; blocks of the rows interleave over scattered frames, and every byte
    of the pool is a NaN until it is written (not of an elastic one)."""

    def __init__(self, be, hq, hkv, d, dtype, lens, seed=3, frames=48, frame_bytes=1 << 20, poison=0xFF, n_layers=1, elastic=False):
        self.be, self.hq, self.hkv, self.d, self.dtype, self.lens = be, hq, hkv, d, dtype, list(lens)
        if elastic:
            frame_bytes = 2 << 20
            self.pool = be.pool_create_elastic(frames * frame_bytes, T, frame_bytes)
        else:
            self.storage = torch.full((frames * frame_bytes,), poison, dtype=torch.uint8, device="cuda")
            self.pool = be.pool_create(frames * frame_bytes, T, frame_bytes, self.storage)
        assert self.pool >= 0 and be.pool_seed_free_order(self.pool, gen.free_order(frames, gen.generator(seed, 1))) == 0
        self.m = be.model_register(self.pool, hq, hkv, d, dtype, len(lens), max(1, max(-(-n // T) for n in lens)), n_layers)
        assert self.m >= 0 and be.balloon_resize(self.m, frames) == frames
        for upto in range(48, max(max(lens), 1) + 48, 48):
            assert be.seq_reserve_batch(self.m, list(range(len(lens))), [min(n, upto) for n in lens]) >= 0

    def fill(self, row, kv, n=None):
        n = kv["k"].shape[0] if n is None else n
        b = -(-n // T)
        if n:
            ks, vs = kv.get("k_scale"), kv.get("v_scale")
            assert self.be.kv_write(self.m, row, 0, kv["k"][:n], kv["v"][:n], None if ks is None else ks[:b], None if vs is None else vs[:b]) == n

    def read(self, row, begin, n):
        """Values float64 [n][Hkv][D] of K and V."""
        rc, k, v, ks, vs = self.be.kv_read(self.m, row, begin, n)
        assert rc == n
        if self.dtype == 0:
            return f64(k), f64(v)
        of = lambda c, s: torch.from_numpy(c).view(torch.float8_e4m3fn).double().numpy() * s.astype(np.float64)[:, :, None]
        return of(k, ks), of(v, vs)

    def close(self):
        torch.cuda.synchronize()
        for s in range(len(self.lens)):
            self.be.seq_release(self.m, s)
        assert self.be.balloon_resize(self.m, 0) == 0 and self.be.model_unregister(self.m) == 0 and self.be.pool_destroy(self.pool) == 0
