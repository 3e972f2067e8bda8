"""Generation's steps between two passes of attention, written out on the CPU: pages forked and compacted entry by entry, beam search's selection in 64 bits."""
import math

import numpy as np

NONE, BEGINS = -1, -2


def fork(tables, lens, parents, grow, refs, P, out_cols):
    """Lists in, lists out: (tables, lens, refs, copies, status)."""
    n_phys, cap, out_cap = len(refs), len(tables[0]) * P, out_cols * P
    ok = lambda x: x if 0 <= x < n_phys else -1
    free = [i for i, r in enumerate(refs) if r == 0]
    count, out, lens_out, copies, taken, missing, seen = list(refs), [], [], [], 0, 0, set()

    def take():
        nonlocal taken, missing
        if taken < len(free):
            taken += 1
            return free[taken - 1]
        missing += 1
        return -1

    lens = [min(max(t, 0), cap) for t in lens]
    for row, t in zip(tables, lens):
        for x in row[:-(-t // P)]:
            if ok(x) >= 0:
                count[x] -= 1
    for b, s in enumerate(parents):
        mine, t, copy = [], 0, [-1, -1, 0]
        if 0 <= s < len(tables):
            t = min(lens[s], out_cap)
            mine = [ok(x) for x in tables[s][:-(-t // P)]]
            if t % P and mine[-1] >= 0 and (s in seen or refs[mine[-1]] > 1):
                page = take()
                copy = [mine[-1], page, t % P] if page >= 0 else copy
                mine[-1] = page
            seen.add(s)
        if 0 <= s < len(tables) or s == BEGINS:
            t = min(t + max(0, grow[b] if grow is not None else 0), out_cap)
        while len(mine) < -(-t // P):
            mine.append(take())
        for x in mine:
            if x >= 0:
                count[x] += 1
        out.append(mine + [-1] * (out_cols - len(mine)))
        lens_out.append(t)
        copies.append(copy)
    return out, lens_out, count, copies, [taken, missing]


def compact(tables, lens, refs, P):
    """(tables, refs, moves, map, status)."""
    n_phys, cols = len(refs), len(tables[0])
    n = sum(r > 0 for r in refs)
    holes, movers = [i for i in range(n) if refs[i] <= 0], [i for i in range(n, n_phys) if refs[i] > 0]
    new = [i if r > 0 else -1 for i, r in enumerate(refs)]
    count = [r if i < n and r > 0 else 0 for i, r in enumerate(refs)]
    for a, b in zip(movers, holes):
        new[a], count[b] = b, refs[a]
    out = [[new[x] if l < -(-min(max(t, 0), cols * P) // P) and 0 <= x < n_phys else -1 for l, x in enumerate(row)] for row, t in zip(tables, lens)]
    return out, count, [[a, b, P] for a, b in zip(movers, holes)], new, [n, len(movers)]


def beam(logits, scores, n_out, done=None, pad=0):
    """logits [groups][beams][vocab], scores [groups][beams] (numpy) -> (parents, tokens, scores float64, logits' log-sums)."""
    x, s = np.asarray(logits, np.float64), np.asarray(scores, np.float64)
    groups, W, V = x.shape
    parents, tokens = np.full((groups, n_out), -1), np.full((groups, n_out), -1)
    best = np.full((groups, n_out), -np.inf)
    for g in range(groups):
        cand = np.full((W, V), -np.inf)
        for w in range(W):
            if not math.isfinite(s[g, w]):
                continue
            if done is not None and done[g, w]:
                cand[w, 0] = s[g, w]      # (its place among the beam's candidates does not matter: there is one)
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                top = x[g, w].max()
                z = top + np.log(np.exp(x[g, w] - top).sum())
            if np.isfinite(z):
                cand[w] = s[g, w] + (x[g, w] - z)
        flat = cand.ravel()
        order = np.argsort(-flat, kind="stable")[:n_out]
        order = order[flat[order] > -np.inf]
        k = len(order)
        parents[g, :k], tokens[g, :k], best[g, :k] = g * W + order // V, order % V, flat[order]
        if done is not None:
            tokens[g, :k] = np.where(done[g][order // V] != 0, pad, tokens[g, :k])
    return parents, tokens, best
