"""Plain 64-bit forms of the key/value cache's operators (numpy, loops), and the
random caches that the tests read."""
import numpy as np
import torch

from paper_2608_26581_amd import workloads as wl

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16(x):
    """x rounded to bf16, as float64."""
    return wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(np.asarray(x, np.float32))).astype(np.float64)


def decode(codes, scales):
    """float64 values [.., D] of codes [.., D / 2] and scale bytes [.., D / 32]."""
    c = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
    v = np.where(c & 8, -1.0, 1.0) * E2M1[c & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def rotate(x, positions, cos_sin, axes, interleaved, backward=False, dtype=np.float64):
    """x [T][H][D] rotated in dtype, products and sums rounded to it one by one."""
    x = np.asarray(x, dtype)
    y = x.copy()
    R2 = cos_sin.shape[1]
    for j in range(R2):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + R2)
        p = positions[axes[j]]
        inside = (p >= 0) & (p < cos_sin.shape[0])
        cs = cos_sin[np.where(inside, p, 0), j].astype(dtype)
        cs[~inside] = np.nan
        c, s = cs[:, :1], cs[:, 1:]
        s = -s if backward else s
        u, w = x[:, :, a], x[:, :, b]
        y[:, :, a] = u * c - w * s
        y[:, :, b] = w * c + u * s
    return y


def table(max_pos, rotary, theta=10000.0):
    angle = np.arange(max_pos)[:, None] * theta ** (-np.arange(0, rotary, 2) / rotary)
    return np.stack((np.cos(angle), np.sin(angle)), -1).astype(np.float32)


class Cache:
    """A cache of random codes for requests of the given lengths: shuffled blocks,
    unused places full of NaN scales."""

    def __init__(self, rng, lens, heads, page, D, spare=2, width=None):
        held = [-(-n // page) for n in lens]
        self.blocks = max(1, sum(held) + spare)
        self.page, self.D, self.heads = page, D, heads
        order = rng.permutation(self.blocks)
        width = max([1] + held) if width is None else width
        self.tables = np.full((len(lens), width), -1, np.int32)
        at = 0
        for b, h in enumerate(held):
            self.tables[b, :h] = order[at:at + h]
            at += h
        self.parts = []
        for part in range(2):
            codes = rng.integers(0, 256, (self.blocks, heads, page, D // 2), dtype=np.uint8)
            scales = np.full((self.blocks, heads, page, D // 32), 255, np.uint8)
            for b, n in enumerate(lens):
                for i, block in enumerate(self.tables[b, :held[b]]):
                    k = min(page, n - i * page)
                    scales[block, :, :k] = rng.integers(121, 127, (heads, k, D // 32))
            self.parts += [codes, scales]

    def device(self):
        return tuple(torch.from_numpy(p).cuda() for p in self.parts)

    def values(self, b, h, n):
        """K, V [n][D] of request b's first n tokens (NaN where there is no block)."""
        out = []
        for codes, scales in (self.parts[:2], self.parts[2:]):
            rows = []
            for j in range(-(-n // self.page)):
                block = self.tables[b, j]
                rows.append(decode(codes[block, h], scales[block, h]) if 0 <= block < self.blocks
                            else np.full((self.page, self.D), np.nan))
            out.append(np.concatenate(rows)[:n] if rows else np.zeros((0, self.D)))
        return out


def attention(q, cache, lens, starts, scale, causal, window):
    """(out, lse, bound on |P| |V|, bound on |q k|) in float64; rows of q that belong
    to no request are NaN in out."""
    T, Hq, D = q.shape
    G = Hq // cache.heads
    out = np.full(q.shape, np.nan)
    lse = np.full((T, Hq), np.nan)
    pv = np.zeros(q.shape)
    qk = np.zeros((T, Hq))
    for b, n in enumerate(lens):
        nq = starts[b + 1] - starts[b]
        n = min(n, cache.tables.shape[1] * cache.page)
        here = np.array([0 <= cache.tables[b, j // cache.page] < cache.blocks for j in range(n)],
                        bool)
        for h in range(Hq if nq else 0):
            K, V = cache.values(b, h // G, n)
            for i in range(nq):
                p, r = n - nq + i, starts[b] + i
                j = np.arange(n)
                see = here & ((j <= p) if causal else True) & ((j > p - window) if window else True)
                if not see.any():
                    out[r, h], lse[r, h] = 0.0, -np.inf
                    continue
                s = scale * (K[see] @ q[r, h])
                m = s.max() if not np.isnan(s).any() else np.nan
                w = np.exp(s - m)
                out[r, h] = w @ V[see] / w.sum()
                lse[r, h] = m + np.log(w.sum())
                pv[r, h] = w @ np.abs(V[see]) / w.sum()
                qk[r, h] = abs(scale) * (np.abs(K[see]) @ np.abs(q[r, h])).max()
    return out, lse, pv, qk


def assert_attention_close(got, lse, ref, what=""):
    """Tolerances from the arithmetic.  P is rounded to bf16 (2^-9 of each term of
    sum P |v| / sum P); scores are fp32 sums of at most 258 exact products (2^-16 of
    sum |q k|, far less for signs at random), which moves P by that much of itself;
    exp and the sums add a few 2^-22; a P below 2^-126 vanishes (2^-126 of each |v|, at
    most 3 here, of at most 5003: 2^-112); the output is rounded to bf16 (2^-9):
        |out - ref| <= (2^-8 + 2^-15 qk) pv + 2^-8 |ref| + 2^-112,
        |lse - ref| <= 2^-16 (1 + qk)."""
    out_ref, lse_ref, pv, qk = ref
    got, nan = np.asarray(got, np.float64), np.isnan(out_ref)
    assert np.array_equal(np.isnan(got), nan), what
    tol = (2.0 ** -8 + 2.0 ** -15 * qk[..., None]) * pv + 2.0 ** -8 * np.abs(out_ref) + 2.0 ** -112
    bad = np.abs(got - out_ref) > tol
    assert not bad[~nan].any(), (what, np.argwhere(bad & ~nan)[:3], np.abs(got - out_ref)[bad & ~nan][:3])
    if lse is not None:
        lse = np.asarray(lse, np.float64)
        fin = np.isfinite(lse_ref)
        assert np.array_equal(np.isneginf(lse_ref), np.isneginf(lse)), what
        assert np.all(np.abs(lse[fin] - lse_ref[fin]) <= (2.0 ** -16 * (1 + qk))[fin]), what
