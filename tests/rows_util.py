"""Packed rows for the tests of the rotating append, the 4-bit cache and the attention over it: seeded inputs, and the operators
written out in 64 bits on the CPU, sequence by sequence, without the package's code."""
import math

import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # half a step of a type, relative
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


class Batch:
    """spans: (rows, tokens) of every sequence; page tables in shuffled order, `behind` rows that belong to no sequence."""

    def __init__(self, spans, P, seed=0, behind=2, spare=3, extra_cols=0):
        rng = np.random.default_rng(seed)
        self.spans, self.P = spans, P
        self.starts = [0]
        for n, _ in spans:
            self.starts.append(self.starts[-1] + n)
        self.rows = self.starts[-1]
        self.n_rows = max(1, self.rows + behind)
        pages = [-(-t // P) for _, t in spans]
        self.cols = max(1, max(pages)) + extra_cols
        self.n_phys = sum(pages) + spare
        order = rng.permutation(self.n_phys)
        self.tables = np.full((len(spans), self.cols), -1, np.int32)   # (never looked up past a sequence's pages)
        at = 0
        for b, c in enumerate(pages):
            self.tables[b, :c] = order[at:at + c]
            at += c
        self.max_len = max(1, max(t for _, t in spans))
        self.max_rows = max(1, max(n for n, _ in spans))

    def device(self):
        return dict(page_tables=torch.tensor(self.tables, device="cuda"),
                    seq_lens=torch.tensor([t for _, t in self.spans], dtype=torch.int32, device="cuda"),
                    row_starts=torch.tensor(self.starts, dtype=torch.int32, device="cuda"))

    def each_row(self):
        """(row, sequence, position) of every row that exists."""
        for b, (n, t) in enumerate(self.spans):
            for i in range(n):
                if t - n + i >= 0:
                    yield self.starts[b] + i, b, t - n + i


def tables(n_pos, rot_dim, seed=0):
    """cos and sin of angles all over the circle, float32."""
    a = np.random.default_rng(seed).uniform(-math.pi, math.pi, (n_pos, rot_dim // 2))
    return torch.tensor(np.cos(a), dtype=torch.float32), torch.tensor(np.sin(a), dtype=torch.float32)


def rotate(x, cos, sin, interleaved, back=False):
    """x [heads][D], cos / sin [half] -> (float64 rotation, |x1 c| + |x2 s| of every dim).  The products of two floats are exact."""
    x, c, s = x.double(), cos.double(), sin.double()
    if back:
        s = -s
    half = c.shape[0]
    i = torch.arange(half)
    one, two = (2 * i, 2 * i + 1) if interleaved else (i, half + i)
    y, size = x.clone(), x.abs()
    y[:, one] = x[:, one] * c - x[:, two] * s
    y[:, two] = x[:, two] * c + x[:, one] * s
    size[:, one] = (x[:, one] * c).abs() + (x[:, two] * s).abs()
    size[:, two] = (x[:, two] * c).abs() + (x[:, one] * s).abs()
    return y, size


def quantise(x):
    """x [..., D] float64 -> (codes [..., D] uint8, scale bytes [..., D / 32] uint8): nearest code by search, ties to the even one."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(x.shape[:-1] + (-1, 32))
    top = np.abs(blocks).max(-1)
    fine = np.isfinite(top)
    e = np.full(top.shape, -125)
    with np.errstate(divide="ignore"):
        guess = np.where(fine & (top > 0), np.ceil(np.log2(np.where(top > 0, top, 1.0) / 7.0)), -125)
    for k in (-1, 0, 1):   # the smallest exponent with top <= 7 2^e, whatever the logarithm's rounding
        cand = (guess + k).astype(np.int64)
        ok = np.where(fine, top, 0.0) <= np.ldexp(7.0, cand)
        e = np.where(ok & ((k == -1) | (top > np.ldexp(7.0, cand - 1))), cand, e)
    e = np.clip(e, -125, 125)
    a = np.abs(blocks) / np.ldexp(1.0, e)[..., None]
    with np.errstate(invalid="ignore"):
        d = np.abs(np.minimum(a, 6.0)[..., None] - LEVELS)
    best = d.min(-1, keepdims=True)
    hit = d == best
    even = hit & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), hit.argmax(-1)).astype(np.uint8)
    code = np.where(fine[..., None], code + 8 * np.signbit(blocks), 0).astype(np.uint8)
    byte = np.where(fine, e + 127, 255).astype(np.uint8)
    return code.reshape(x.shape), byte


def values(code, byte):
    """float64 values of codes and scale bytes."""
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(byte == 255, np.nan, np.ldexp(1.0, byte.astype(np.int64) - 127))
    return v * np.repeat(s, 32, -1)


def pack(code, byte):
    """codes [..., P, D], bytes [..., P, D / 32] -> tiles."""
    pairs = code[..., 0::2] | (code[..., 1::2] << 4)
    return np.concatenate([pairs.reshape(pairs.shape[:-2] + (-1,)), np.swapaxes(byte, -1, -2).reshape(byte.shape[:-2] + (-1,))], -1)


def unpack(tiles, P, D):
    cut = P * D // 2
    pairs = tiles[..., :cut].reshape(tiles.shape[:-1] + (P, D // 2))
    code = np.stack([pairs & 15, pairs >> 4], -1).reshape(tiles.shape[:-1] + (P, D))
    return code, np.swapaxes(tiles[..., cut:].reshape(tiles.shape[:-1] + (D // 32, P)), -1, -2)


def random_pool(batch, Hkv, D, seed):
    """A kvq pool as numpy: the tokens of every sequence quantised N(0, 1) values, every other byte 255 (NaN scales)."""
    rng = np.random.default_rng(seed)
    P = batch.P
    pool = np.full((batch.n_phys, Hkv, P * (D // 2 + D // 32)), 255, np.uint8)
    for b, (_, t) in enumerate(batch.spans):
        for l in range(-(-t // P)):
            code, byte = quantise(rng.standard_normal((Hkv, P, D)))
            held = min(P, t - l * P)
            code[:, held:], byte[:, held:] = 255 & 15, 255
            pool[batch.tables[b, l]] = pack(code, byte)
    return pool


def sequence_values(batch, pool, b, g, D):
    """float64 [tokens][D] of a sequence's KV head."""
    t = batch.spans[b][1]
    tiles = pool[batch.tables[b, :-(-t // batch.P)], g]
    return values(*unpack(tiles, batch.P, D)).reshape(-1, D)[:t]


def attend(batch, q, k_pool, v_pool, scale, lists=None, terms=2.0 ** -15):
    """(o, lse, tolerance of o, tolerance of lse) in 64 bits for q [n_rows][Hq][D] (torch, CPU), pools as numpy.

    Tolerances, relative to sum p |v|: `terms` for the rounding of the weights, 2 d for the logits' errors d (a dot product of
    D exact products summed in fp32: D 2^-24 sum |q k|, and three roundings of the scaled logit), 2^-20 for exponentials and factors, tokens
    2^-24 for the sums; then half a step of the type."""
    n_rows, Hq, D = q.shape
    Hkv = k_pool.shape[1]
    G, P, half = Hq // Hkv, batch.P, HALF[q.dtype]
    o, tol = np.zeros((n_rows, Hq, D)), np.zeros((n_rows, Hq, D))
    lse, ltol = np.full((Hq, n_rows), -np.inf), np.zeros((Hq, n_rows))
    x = q.double().numpy()
    for b, (n, t) in enumerate(batch.spans):
        for g in range(Hkv):
            if t == 0 or n == 0:
                continue
            k, v = sequence_values(batch, k_pool, b, g, D), sequence_values(batch, v_pool, b, g, D)
            listed = np.ones(t, bool)
            if lists is not None:
                listed = np.isin(np.arange(t) // P, lists[b][g])
            rows = np.arange(batch.starts[b], batch.starts[b] + n)
            for h in range(g * G, (g + 1) * G):
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (x[rows, h] @ k.T)
                    size = scale * (np.abs(x[rows, h]) @ np.abs(k).T)
                for i, r in enumerate(rows):
                    seen = listed & (np.arange(t) <= t - n + i)
                    if not seen.any():
                        continue
                    z, vs = s[i, seen], v[seen]
                    top = z.max()
                    with np.errstate(invalid="ignore"):
                        p = np.exp(z - top)
                        total = p.sum()
                        o[r, h] = (p / total) @ vs
                        lse[h, r] = top + np.log(total)
                        d = np.max((D + 3) * 2.0 ** -24 * (size[i, seen] + np.abs(z)))
                        rel = 2 * d + 2.0 ** -20 + seen.sum() * 2.0 ** -24
                        tol[r, h] = (p / total) @ np.abs(vs) * (terms + rel) + half * np.abs(o[r, h])
                        ltol[h, r] = rel + 2.0 ** -22 * (1 + abs(lse[h, r]))
    return o, lse, tol, ltol


def check(name, got, want, tol):
    """got within tol of want wherever want is finite, and equal elsewhere (NaN to NaN)."""
    got = np.asarray(got, np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{name}: NaN in other places"
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), f"{name}: infinities differ"
    off = np.abs(got[fine] - want[fine])
    bad = off > np.broadcast_to(tol, want.shape)[fine]
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off by up to {off[bad].max():.3g}"
