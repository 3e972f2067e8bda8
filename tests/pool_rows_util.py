"""Pools of bf16 / fp32 rows for the tests of the attention of packed rows over them: seeded pools, and the operator in 64 bits on the CPU."""
import numpy as np
import torch

import rows_util as ru


def random_pool(batch, Hkv, D, dt, seed, fill=float("nan")):
    """[n_phys][Hkv][P][D] (torch, CPU): N(0, 1) where a sequence has a token, `fill` everywhere else."""
    gen = torch.Generator().manual_seed(seed)
    pool = torch.full((batch.n_phys, Hkv, batch.P, D), fill, dtype=dt)
    for b, (_, t) in enumerate(batch.spans):
        for l in range(-(-t // batch.P)):
            held = min(batch.P, t - l * batch.P)
            pool[int(batch.tables[b, l]), :, :held] = torch.randn((Hkv, held, D), generator=gen).to(dt)
    return pool


def values(batch, pool, b, g):
    """[tokens][D] float64 of a sequence and KV head."""
    t = batch.spans[b][1]
    pages = [int(x) for x in batch.tables[b, :-(-t // batch.P)]]
    return pool[pages, g].double().flatten(0, 1)[:t].numpy()


def attend(batch, q, k_pool, v_pool, scale, lists=None):
    """(o, lse, tolerance of o, tolerance of lse) in 64 bits.

    Tolerances, relative to sum p |v|: 2^-15 for weights in two bf16 terms (fp32: 2^-22 for a product and its part of a sum), 2 d for the logits' errors d (a
    dot product of D products summed in fp32: D 2^-24 sum |q k|, and three roundings of the scaled logit), 2^-20 for exponentials and factors, tokens
    2^-24 for the sums; then half a step of the type."""
    n_rows, Hq, D = q.shape
    Hkv = k_pool.shape[1]
    G, P, half = Hq // Hkv, batch.P, ru.HALF[q.dtype]
    terms = 2.0 ** -22 if q.dtype == torch.float32 else 2.0 ** -15
    o, tol = np.zeros((n_rows, Hq, D)), np.zeros((n_rows, Hq, D))
    lse, ltol = np.full((Hq, n_rows), -np.inf), np.zeros((Hq, n_rows))
    x = q.double().numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        for b, (n, t) in enumerate(batch.spans):
            for g in range(Hkv if t and n else 0):
                k, v = values(batch, k_pool, b, g), values(batch, v_pool, b, g)
                listed = np.ones(t, bool) if lists is None else np.isin(np.arange(t) // P, lists[b][g])
                rows = np.arange(batch.starts[b], batch.starts[b] + n)
                for h in range(g * G, (g + 1) * G):
                    s = scale * (x[rows, h] @ k.T)
                    size = scale * (np.abs(x[rows, h]) @ np.abs(k).T)
                    for i, r in enumerate(rows):
                        seen = listed & (np.arange(t) <= t - n + i)
                        if not seen.any():
                            continue
                        z, vs = s[i, seen], v[seen]
                        top = z.max()
                        p = np.exp(z - top)
                        total = p.sum()
                        o[r, h] = (p / total) @ vs
                        lse[h, r] = top + np.log(total)
                        d = np.max((D + 3) * 2.0 ** -24 * (size[i, seen] + np.abs(z)))
                        rel = 2 * d + 2.0 ** -20 + seen.sum() * 2.0 ** -24
                        tol[r, h] = (p / total) @ np.abs(vs) * (terms + rel) + half * np.abs(o[r, h])
                        ltol[h, r] = rel + 2.0 ** -22 * (1 + abs(lse[h, r]))
    return o, lse, tol, ltol
