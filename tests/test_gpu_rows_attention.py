"""GPU tests of the attention of packed rows over pools of bf16 / fp32 rows, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2602_02108_amd import api

import pool_rows_util as pu
import rows_util as ru

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _queries(b, Hq, D, dt, seed=1):
    return torch.randn((b.n_rows, Hq, D), generator=torch.Generator().manual_seed(seed)).to(dt)


def _lists(b, lists, Hkv):
    width = max(1, max(len(x) for s in lists for x in s)) + 2
    sel = torch.full((len(b.spans), Hkv, width), 7777777, dtype=torch.int32)
    for i, s in enumerate(lists):
        for h, x in enumerate(s):
            sel[i, h, :len(x)] = torch.tensor(x, dtype=torch.int32)
    return sel.cuda(), torch.tensor([[len(x) for x in s] for s in lists], dtype=torch.int32).cuda()


def _run(b, q, pools, scale, lists=None, max_rows=None, workspace=None, max_len=None):
    at = b.device()
    table = at.pop("page_tables")
    g, gp = q.cuda(), [x.cuda() for x in pools]
    if max_len:   # a table with room for that many tokens
        table = torch.cat([table, torch.full((table.shape[0], max_len // b.P - table.shape[1]), -1, dtype=torch.int32, device="cuda")], 1)
    desc = api.make_rows_desc(g, gp[0], table, max_len or b.max_len, scale, max_rows=max_rows or b.max_rows)
    o = torch.full_like(g, 5.0)
    lse = torch.full((g.shape[1], g.shape[0]), 5.0, device="cuda")
    sel, cnt = (None, None) if lists is None else _lists(b, lists, pools[0].shape[1])
    api.paged_attn_fwd_rows(desc, g, *gp, table, sel, cnt, o, lse, workspace, **at)
    torch.cuda.synchronize()
    return o, lse


def _verify(b, q, pools, scale, o, lse, lists=None):
    wo, wl, to, tl = pu.attend(b, q, *pools, scale, lists)
    live = slice(0, b.rows)
    ru.check("LSE", lse.cpu().double().numpy()[:, live], wl[:, live], tl[:, live])
    ru.check("O", o.cpu().double().numpy()[live], wo[live], to[live])
    assert (o[b.rows:] == 5.0).all() and (lse[:, b.rows:] == 5.0).all(), "rows of no sequence were written"


# (type, (Hq, Hkv), D, P, spans)
CASES = [
    (BF, (28, 4), 128, 128, [(1, 1), (1, 15), (1, 16), (1, 17), (1, 31), (1, 32), (1, 33), (1, 127), (1, 128), (1, 129), (1, 1000), (0, 50), (0, 0)]),
    (BF, (14, 2), 128, 128, [(4, 700), (3, 3), (1, 2), (4, 260)]),
    (BF, (6, 2), 128, 64, [(5, 129), (5, 5), (3, 64)]),
    (BF, (8, 8), 64, 16, [(1, 47), (1, 48), (1, 49), (1, 16), (1, 500)]),
    (BF, (14, 2), 64, 16, [(9, 333), (2, 17), (9, 9)]),
    (BF, (28, 4), 128, 32, [(20, 300), (7, 1100)]),
    (BF, (20, 1), 64, 64, [(33, 333)]),
    (BF, (4, 4), 128, 16, [(40, 500), (17, 17), (1, 90)]),
    (F32, (2, 1), 64, 16, [(1, 1), (3, 33), (8, 100), (2, 16)]),
    (F32, (28, 4), 128, 128, [(1, 400), (1, 1)]),
    (F32, (6, 2), 128, 16, [(9, 200), (4, 31)]),
    (F32, (14, 2), 64, 128, [(40, 170), (0, 3), (3, 500)]),
    (F32, (16, 1), 128, 32, [(2, 65), (1, 1000)]),
]
IDS = [f"{'bf16' if c[0] == BF else 'f32'}-h{c[1][0]}-{c[1][1]}-d{c[2]}-p{c[3]}-{i}" for i, c in enumerate(CASES)]


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_every_page(case):
    """Every page; what no row sees (the rest of last pages, spare pages) is NaN."""
    dt, (Hq, Hkv), D, P, spans = case
    b = ru.Batch(spans, P, 5)
    q = _queries(b, Hq, D, dt)
    pools = [pu.random_pool(b, Hkv, D, dt, s) for s in (11, 12)]
    o, lse = _run(b, q, pools, 1.0 / math.sqrt(D))
    _verify(b, q, pools, 1.0 / math.sqrt(D), o, lse)


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_page_lists(case):
    """Lists of a part of the pages, of other lengths per head, some empty, some without the pages of the rows, and with pages
    past the sequence's end."""
    dt, (Hq, Hkv), D, P, spans = case
    b = ru.Batch(spans, P, 6, extra_cols=2)
    rng = np.random.default_rng(8)
    lists = []
    for _, t in spans:
        pages = -(-t // P)
        lists.append([sorted(int(x) for x in rng.permutation(pages + 2)[:rng.integers(0, pages + 3)]) for _ in range(Hkv)])
    q = _queries(b, Hq, D, dt, 2)
    pools = [pu.random_pool(b, Hkv, D, dt, s) for s in (13, 14)]
    o, lse = _run(b, q, pools, 0.1, lists)
    _verify(b, q, pools, 0.1, o, lse, lists)


@pytest.mark.parametrize("dt,Hq,Hkv,D,P,spans,listed", [
    (BF, 7, 1, 128, 128, [(1, 40000)], False),             # a long cache: tokens split over workgroups
    (F32, 2, 1, 64, 16, [(1, 30011), (1, 200)], False),    # small pages: many windows of page ids
    (BF, 28, 4, 128, 128, [(2, 20000), (1, 3000)], True),
    (BF, 14, 2, 64, 16, [(3, 9000)], True),
    (BF, 28, 4, 128, 128, [(600, 700), (571, 571), (1, 40)], False),   # many rows
    (BF, 8, 2, 64, 32, [(513, 1500), (64, 64)], False),
    (BF, 4, 2, 128, 16, [(200, 300), (129, 3000)], True),
    (F32, 28, 4, 64, 32, [(300, 400), (150, 500)], False),
    (F32, 4, 2, 128, 64, [(200, 900)], True),
    (BF, 8, 1, 64, 16, [(300, 2000)], True),
    (BF, 7, 1, 128, 128, [(5, 12000)] * 3 + [(1, 30)] * 5, False),     # several row blocks over long caches
])
def test_long_and_many(dt, Hq, Hkv, D, P, spans, listed):
    b = ru.Batch(spans, P, 7)
    lists = None
    if listed:
        rng = np.random.default_rng(9)
        lists = [[sorted(int(x) for x in rng.permutation(-(-t // P))[:-(-t // P) * 2 // 3]) for _ in range(Hkv)] for _, t in spans]
    q = _queries(b, Hq, D, dt, 3)
    pools = [pu.random_pool(b, Hkv, D, dt, s) for s in (15, 16)]
    o, lse = _run(b, q, pools, 1.0 / math.sqrt(D), lists)
    _verify(b, q, pools, 1.0 / math.sqrt(D), o, lse, lists)


@pytest.mark.parametrize("dt,Hq,Hkv,D,P,spans", [
    (BF, 28, 4, 128, 128, [(1, 700), (1, 5), (0, 0), (1, 3000)]),
    (BF, 8, 4, 64, 32, [(2, 700), (1, 1)]),
    (BF, 8, 4, 128, 16, [(1, 40), (1, 700)]),
    (F32, 8, 4, 128, 64, [(1, 700), (3, 70)]),
    (F32, 4, 4, 64, 128, [(4, 1300)]),
    (BF, 14, 2, 128, 128, [(40, 900), (3, 50)]),
])
def test_room_for_far_longer_sequences(dt, Hq, Hkv, D, P, spans):
    """A bound of two million tokens a sequence over short ones."""
    b = ru.Batch(spans, P, 12)
    q = _queries(b, Hq, D, dt, 13)
    pools = [pu.random_pool(b, Hkv, D, dt, s) for s in (25, 26)]
    o, lse = _run(b, q, pools, 0.1, max_len=1 << 21)
    _verify(b, q, pools, 0.1, o, lse)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("order", ["rising", "falling", "spikes"])
def test_logits_far_apart(dt, order):
    """Logits over a wide range, so that the reference of the softmax moves often, seldom or in jumps."""
    Hq, Hkv, D, P = 4, 2, 64, 16
    b = ru.Batch([(2, 600), (1, 77), (40, 300)], P, 3)
    q = _queries(b, Hq, D, dt, 4)
    pools = [pu.random_pool(b, Hkv, D, dt, s) for s in (17, 18)]
    direction = np.sign(q[0, 0].double().numpy())
    for s, (_, t) in enumerate(b.spans):
        for pos in range(t):
            size = {"rising": pos / 8.0, "falling": (t - pos) / 8.0, "spikes": 30.0 + pos / 16.0 if pos % 97 == 5 else 0.1}[order]
            pools[0][int(b.tables[s, pos // P]), :, pos % P] = torch.tensor(size * direction).to(dt)
    o, lse = _run(b, q, pools, 0.125)
    _verify(b, q, pools, 0.125, o, lse)


@pytest.mark.parametrize("dt,spans,Hq,Hkv,D", [(BF, [(6, 40), (1, 20)], 4, 2, 128), (F32, [(6, 40), (1, 20)], 4, 2, 64), (BF, [(30, 40), (9, 200)], 14, 2, 64),
                                               (F32, [(6, 40), (1, 20)], 4, 2, 128), (BF, [(150, 170), (1, 20)], 4, 2, 128)])
def test_values_that_are_not_finite(dt, spans, Hq, Hkv, D):
    """NaN and infinities in K and V of tokens that some rows see, infinite and NaN queries: only the rows that see them change, of
    V only that dim."""
    P = 16
    b = ru.Batch(spans, P, 4)
    q = _queries(b, Hq, D, dt, 6)
    pools = [pu.random_pool(b, Hkv, D, dt, s) for s in (19, 20)]
    n, t = spans[0]

    def spoil(pool, s, pos, g, d, value):
        pool[int(b.tables[s, pos // P]), g, pos % P, d] = value

    spoil(pools[1], 0, t - n + 2, 0, D - 1, math.nan)    # seen by the rows from the third on
    spoil(pools[1], 0, t - 1, 1, 0, math.inf)            # by the last row alone
    spoil(pools[1], 0, t - 3, 1, 9, -math.inf)
    spoil(pools[0], 0, t - 2, 0, 5, math.nan)
    spoil(pools[1], 1, 3, 1, 1, math.inf)                # by every row of the second sequence
    q[1, 1, 3] = math.nan
    q[2, Hq - 1, 0] = math.inf
    o, lse = _run(b, q, pools, 0.125)
    wo, wl, to, tl = pu.attend(b, q, *pools, 0.125)
    # an infinite query's logits are infinite of either sign or NaN: its row holds nothing
    wo[2, Hq - 1], wl[Hq - 1, 2] = np.nan, np.nan
    live = slice(0, b.rows)
    got = o.cpu().double().numpy()[live]
    assert np.isfinite(wo[live]).mean() > 0.5 and (~np.isfinite(wo[live])).any()
    assert np.array_equal(np.isfinite(got), np.isfinite(wo[live]))
    ru.check("LSE", lse.cpu().double().numpy()[:, live], wl[:, live], tl[:, live])
    ru.check("O", np.where(np.isfinite(got), got, 0), np.where(np.isfinite(wo[live]), wo[live], 0), to[live])


# Many bf16 rows over caches whose second reading costs something: (Hq, Hkv), D, P, spans, listed
MANY = [
    ((14, 2), 128, 16, [(300, 900), (40, 70), (1, 20)], False),      # whole waves without rows, pages of a tile
    ((14, 2), 128, 128, [(301, 1300), (90, 60), (0, 30)], True),     # rows without a token; pages that end inside a stage
    ((14, 2), 64, 32, [(300, 1500), (33, 1200)], False),
    ((14, 2), 64, 128, [(299, 2100), (5, 5)], True),
    ((6, 1), 128, 64, [(40, 50000)], False),                         # few rows, cut into parts
    ((10, 1), 64, 16, [(23, 60001), (4, 9)], True),
    ((3, 3), 128, 32, [(513, 1100), (513, 513), (129, 2000)], False),
    ((28, 4), 128, 128, [(4, 9000), (1, 40)], False),                # two row tiles
    ((8, 1), 128, 16, [(3, 40011), (4, 300)], True),
]
MANY_IDS = [f"h{c[0][0]}-{c[0][1]}-d{c[1]}-p{c[2]}-{i}" for i, c in enumerate(MANY)]


def _many(case, seed):
    (Hq, Hkv), D, P, spans, listed = case
    b = ru.Batch(spans, P, seed)
    # (what makes a call one of many rows: bytes of the caches that are read again, at 32 rows a block, or at 16)
    rows, held = b.max_rows * (Hq // Hkv), min(len(spans) * b.max_len, b.n_phys * P) * Hkv * 4 * D
    assert (-(-rows // 32) - 1) * held > (48 << 20) if rows > 32 else (-(-rows // 16) - 1) * held > (16 << 20)
    rng = np.random.default_rng(seed)
    lists = None
    if listed:
        lists = [[sorted(int(x) for x in rng.permutation(-(-t // P))[:-(-t // P) * 4 // 5]) for _ in range(Hkv)] for _, t in spans]
    return b, lists, _queries(b, Hq, D, BF, seed + 1), [pu.random_pool(b, Hkv, D, BF, s) for s in (seed + 2, seed + 3)]


@pytest.mark.parametrize("case", MANY, ids=MANY_IDS)
def test_many_rows(case):
    """Against the definition; then with pools of tokens before heads, and a workspace of anything: the same bits."""
    b, lists, q, pools = _many(case, 40)
    o, lse = _run(b, q, pools, 0.1, lists)
    _verify(b, q, pools, 0.1, o, lse, lists)
    strided = [x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3) for x in pools]
    o2, lse2 = _run(b, q, strided, 0.1, lists, workspace=torch.full((1 << 26,), 255, dtype=torch.uint8, device="cuda"))
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("case", MANY, ids=MANY_IDS)
@pytest.mark.parametrize("order", ["rising", "falling", "spikes"])
def test_many_rows_logits_far_apart(case, order):
    b, lists, q, pools = _many(case, 50)
    direction = torch.sign(q[0, 0].float())
    for s, (_, t) in enumerate(b.spans):
        pos = torch.arange(t, dtype=torch.float32)
        size = {"rising": pos * 60 / t, "falling": (t - pos) * 60 / t, "spikes": torch.where(pos % 97 == 5, 30 + 30 * pos / t, 0.1)}[order]
        pages = torch.from_numpy(b.tables[s].astype(np.int64))[torch.arange(t) // b.P]
        pools[0][pages, :, torch.arange(t) % b.P] = (size[:, None, None] * direction).to(BF).expand(t, pools[0].shape[1], -1)
    o, lse = _run(b, q, pools, 0.1, lists)
    _verify(b, q, pools, 0.1, o, lse, lists)


@pytest.mark.parametrize("case", MANY, ids=MANY_IDS)
def test_many_rows_values_that_are_not_finite(case):
    """As test_values_that_are_not_finite."""
    b, lists, q, pools = _many(case, 60)
    Hkv, P = pools[0].shape[1], b.P
    n, t = b.spans[0]

    def spoil(pool, s, pos, g, d, value):
        pool[int(b.tables[s, pos // P]), g, pos % P, d] = value

    last = pools[0].shape[3] - 1
    for at, (pos, d, value) in enumerate([(t - n + 2, last, math.nan), (t - 1, 0, math.inf), (t - 3, 9, -math.inf), (t - 2, 40, math.nan), (t - n // 2, 33, math.inf),
                                          (t - n // 2, 34, math.nan), (t - 17, 8, math.inf), (t - 16, 7, -math.inf)]):
        spoil(pools[1], 0, pos, at % Hkv, d, value)
    spoil(pools[1], 0, 3, Hkv - 1, 1, math.inf)          # seen by every row
    spoil(pools[0], 0, t - 5, 0, 5, math.nan)
    q[1, 0, 3] = math.nan
    o, lse = _run(b, q, pools, 0.1, lists)
    wo, wl, to, tl = pu.attend(b, q, *pools, 0.1, lists)
    live = slice(0, b.rows)
    got = o.cpu().double().numpy()[live]
    assert np.isfinite(wo[live]).mean() > 0.5 and (~np.isfinite(wo[live])).any()
    assert np.array_equal(np.isfinite(got), np.isfinite(wo[live]))
    ru.check("LSE", lse.cpu().double().numpy()[:, live], wl[:, live], tl[:, live])
    ru.check("O", np.where(np.isfinite(got), got, 0), np.where(np.isfinite(wo[live]), wo[live], 0), to[live])


def test_many_rows_pages_that_the_pool_does_not_have():
    b, _, q, pools = _many(MANY[1][:4] + (False,), 70)
    bad = [1, 4, 9]
    keep = b.tables.copy()
    b.tables[0, bad] = [b.n_phys, -3, 1 << 30]
    o, lse = _run(b, q, pools, 0.1)
    b.tables = keep
    lists = [[[l for l in range(-(-t // b.P)) if s or l not in bad] for _ in range(2)] for s, (_, t) in enumerate(b.spans)]
    _verify(b, q, pools, 0.1, o, lse, lists)


@pytest.mark.parametrize("dt,Hq,Hkv,D,P,spans", [
    (F32, 14, 2, 128, 16, [(300, 900), (150, 700)]),     # parts of many rows
    (F32, 16, 1, 64, 64, [(70, 3000), (1, 5000)]),
    (BF, 16, 2, 64, 128, [(17, 3000), (9, 2000)]),
])
def test_parts_of_rows(dt, Hq, Hkv, D, P, spans):
    b = ru.Batch(spans, P, 17)
    q = _queries(b, Hq, D, dt, 13)
    pools = [pu.random_pool(b, Hkv, D, dt, s) for s in (25, 26)]
    o, lse = _run(b, q, pools, 0.1)
    _verify(b, q, pools, 0.1, o, lse)


def _spread(n, rows, tokens, seed):
    """Spans of n sequences: lengths over their logarithm, some empty, some without rows, some of fewer tokens than rows."""
    rng = np.random.default_rng(seed)
    spans = []
    for _ in range(n):
        t = int(np.exp(rng.uniform(0, np.log(tokens + 1)))) if rng.random() < 0.95 else 0
        spans.append((int(rng.integers(1, rows + 1)) if rng.random() < 0.9 else 0, t))
    spans[n // 3], spans[-1] = (rows, tokens), (0, 3)
    return spans


@pytest.mark.parametrize("dt,Hq,Hkv,D,P,n,rows,tokens,listed", [
    (BF, 4, 2, 128, 16, 140, 1, 3000, False),      # cut
    (BF, 4, 2, 128, 16, 270, 1, 3000, False),      # more sequences and heads than a workgroup counts by itself
    (BF, 6, 2, 64, 32, 300, 5, 900, True),
    (F32, 4, 4, 128, 32, 170, 5, 900, True),
    (F32, 4, 4, 64, 16, 70, 9, 1500, False),
    (F32, 2, 2, 128, 64, 129, 40, 400, True),      # not cut
    (BF, 2, 2, 64, 16, 2100, 1, 300, False),       # more than the planner takes at a time
    (BF, 4, 2, 64, 16, 2500, 2, 700, True),
    (BF, 8, 1, 128, 16, 4097, 1, 40, False),
    (BF, 16, 8, 64, 16, 40, 200, 1200, False),     # in tiles
])
def test_many_sequences(dt, Hq, Hkv, D, P, n, rows, tokens, listed):
    spans = _spread(n, rows, tokens, 3)
    b = ru.Batch(spans, P, 18)
    lists = None
    if listed:
        rng = np.random.default_rng(9)
        lists = [[sorted(int(x) for x in rng.permutation(-(-t // P))[:rng.integers(0, -(-t // P) + 1)]) for _ in range(Hkv)] for _, t in spans]
    q = _queries(b, Hq, D, dt, 14)
    pools = [pu.random_pool(b, Hkv, D, dt, s) for s in (25, 26)]
    o, lse = _run(b, q, pools, 0.1, lists)
    _verify(b, q, pools, 0.1, o, lse, lists)
    ws = torch.full((1 << 28,), 127, dtype=torch.uint8, device="cuda")
    o2, lse2 = _run(b, q, pools, 0.1, lists, workspace=ws)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def _path(b, Hq, Hkv, D, dt):
    """How a call over every page goes, by its sizes: what runs it, who counts it, how it is cut; and the workspace that follows, which the library is asked for."""
    es, rows, heads = dt.itemsize, b.max_rows * (Hq // Hkv), len(b.spans) * Hkv
    cache = min(heads * b.max_len, b.n_phys * Hkv * b.P) * 2 * D * es
    tiles = dt == BF and rows > 32 and (-(-rows // 32) - 1) * cache > (48 << 20)
    rt = 2 if rows > 16 and (D == 64 or (dt == BF and (-(-rows // 16) - 1) * cache > (16 << 20))) else 1
    block, step, least = (128, 64, 8) if tiles else (16 * rt, 32, 4)
    blocks = min((b.n_rows * (Hq // Hkv) // block + len(b.spans)) * Hkv, -(-rows // block) * heads)
    steps, planned = -(-b.max_len // step), heads > 512
    split = steps > 16 and blocks <= (8192 if planned and not tiles else 1024)
    full = not tiles and blocks > 512
    target = 512 if tiles else blocks + 256 if full else 512 - blocks // 2 if blocks < 512 else blocks
    wgs = min(blocks * -(-steps // least), target + blocks + 2)
    loads = [(-(-n * (Hq // Hkv) // block) * Hkv, max(1, -(-t // step))) for n, t in b.spans]
    total, most = sum(x * y for x, y in loads), max(y for x, y in loads if x)
    per = max(least, -(-most // max(1, int(target * most / total))) if tiles else total // target + 1)
    cut = split and most > (2 * per if full else per)
    return ("tiles" if tiles else f"rows{rt}", "planned" if planned else "full" if full else "counted", "cut" if cut else "split" if split else "whole"), \
        (wgs * block * (D + 2) * 4 if split else 0) + ((heads + 1) * 8 if split or planned else 0)


@pytest.mark.parametrize("dt,Hq,Hkv,D,P,spans,path", [
    (BF, 16, 8, 64, 16, _spread(80, 60, 1500, 5), ("tiles", "planned", "cut")),
    (BF, 16, 8, 128, 32, _spread(80, 55, 1300, 6), ("tiles", "planned", "cut")),
    (BF, 16, 8, 64, 16, _spread(90, 200, 1200, 7), ("tiles", "planned", "whole")),
    (BF, 16, 8, 128, 16, [(40, 250)] * 70, ("tiles", "planned", "whole")),
    (BF, 14, 1, 128, 64, [(10, 300)] * 520, ("tiles", "planned", "whole")),
    (F32, 8, 4, 64, 16, _spread(40, 100, 1500, 8), ("rows2", "full", "cut")),
    (F32, 8, 4, 64, 32, [(60, 700)] * 35, ("rows2", "full", "split")),          # about equal: its parts are whole blocks
    (F32, 4, 2, 128, 16, _spread(60, 70, 1500, 9), ("rows1", "full", "cut")),
    (BF, 4, 2, 64, 16, _spread(100, 70, 700, 10), ("rows2", "full", "cut")),
], ids=lambda x: "-".join(x) if isinstance(x, tuple) else None)
def test_many_sequences_by_every_path(dt, Hq, Hkv, D, P, spans, path):
    b = ru.Batch(spans, P, 19)
    got, need = _path(b, Hq, Hkv, D, dt)
    assert got == path
    q = _queries(b, Hq, D, dt, 15)
    pools = [pu.random_pool(b, Hkv, D, dt, s) for s in (27, 28)]
    table = torch.empty((len(spans), b.cols), dtype=torch.int32)
    assert api.rows_workspace_bytes(api.make_rows_desc(q, pools[0], table, b.max_len, 0.1, max_rows=b.max_rows)) == need
    o, lse = _run(b, q, pools, 0.1)
    _verify(b, q, pools, 0.1, o, lse)
    o2, lse2 = _run(b, q, pools, 0.1, workspace=torch.full((need,), 127, dtype=torch.uint8, device="cuda") if need else None)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("B", [200, 300])
def test_many_sequences_of_equal_rows_and_lengths(B):
    """Without starts and lengths."""
    Hq, Hkv, D, P, t = 4, 2, 64, 16, 40
    b = ru.Batch([(2, t)] * B, P, 18, behind=0)
    q = _queries(b, Hq, D, BF, 14)
    pools = [pu.random_pool(b, Hkv, D, BF, s) for s in (25, 26)]
    table = torch.tensor(b.tables, device="cuda")
    desc = api.make_rows_desc(q.cuda(), pools[0].cuda(), table, t, 0.1, max_rows=2)
    o, lse = api.paged_attn_fwd_rows(desc, q.cuda(), *(x.cuda() for x in pools), table)
    torch.cuda.synchronize()
    _verify(b, q, pools, 0.1, o, lse)


def test_many_sequences_in_a_captured_step():
    """Lengths, rows and tables that change between the replays: each of them the bits of an eager call, with the program's own work in between."""
    P, Hq, Hkv, D, n, dt = 16, 4, 2, 64, 300, BF
    spans = [_spread(n, 3, 900, s) for s in (1, 2, 3)]
    batches = [ru.Batch(x, P, 5) for x in spans]
    rows, cols, n_phys = max(b.n_rows for b in batches), 60, max(b.n_phys for b in batches)
    gen = torch.Generator().manual_seed(3)
    pools = [torch.randn((n_phys, Hkv, P, D), generator=gen).to(dt).cuda() for _ in range(2)]
    q = torch.randn((rows, Hq, D), generator=gen).to(dt).cuda()
    table, lens = torch.zeros((n, cols), dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    starts = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    desc = api.make_rows_desc(q, pools[0], table, cols * P, 0.1, max_rows=3)
    ws = torch.empty(api.rows_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    o, lse = torch.zeros((rows, Hq, D), dtype=dt, device="cuda"), torch.zeros((Hq, rows), device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            api.paged_attn_fwd_rows(desc, q, *pools, table, o=o, lse=lse, workspace=ws, seq_lens=lens, row_starts=starts)
    for i in (0, 1, 2, 1, 0):
        b = batches[i]
        table[:, :b.cols] = torch.tensor(b.tables, device="cuda")
        lens.copy_(torch.tensor([t for _, t in b.spans], dtype=torch.int32))
        starts.copy_(torch.tensor(b.starts, dtype=torch.int32))
        o.fill_(5.0)
        lse.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        o2, lse2 = torch.full_like(o, 5.0), torch.full_like(lse, 5.0)
        api.paged_attn_fwd_rows(desc, q, *pools, table, o=o2, lse=lse2, seq_lens=lens, row_starts=starts)
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        q_here = q.cpu()
        wo, wl, to, tl = pu.attend(b, q_here[:b.n_rows], *(x.cpu() for x in pools), 0.1)
        live = slice(0, b.rows)
        ru.check("O", o.cpu().double().numpy()[live], wo[live], to[live])
        ru.check("LSE", lse.cpu().double().numpy()[:, live], wl[:, live], tl[:, live])
        assert (o[b.rows:] == 5.0).all()


def test_logits_of_minus_infinity_have_no_weight():
    P, D = 16, 64
    for dt in (BF, F32):
        b = ru.Batch([(2, 50), (1, 33)], P, 4)
        q = torch.ones((b.n_rows, 2, D), dtype=dt)
        pools = [pu.random_pool(b, 1, D, dt, s) for s in (19, 20)]
        big = -3.0e38
        for s, pos in [(0, x) for x in range(0, 50, 3)] + [(1, x) for x in range(33)]:
            pools[0][int(b.tables[s, pos // P]), 0, pos % P] = big
        o, lse = _run(b, q, pools, 1.0)
        keep = [x for x in range(50) if x % 3]
        k, v = (pu.values(b, x, 0, 0) for x in pools)
        for i in range(2):
            seen = [x for x in keep if x <= 48 + i]
            z = k[seen].sum(-1)
            p = np.exp(z - z.max())
            want = (p / p.sum()) @ v[seen]
            # two terms of the weights or fp32, sums of 50, half a step of the output
            tol = (2.0 ** -14 if dt == BF else 2.0 ** -18) * np.abs(v[seen]).max() + ru.HALF[dt] * np.abs(want)
            assert (np.abs(o[i, 0].cpu().double().numpy() - want) <= tol).all()
        assert (o[2] == 0).all() and (lse[:, 2] == -math.inf).all()


def test_pages_and_lengths_out_of_range_are_not_seen():
    Hq, Hkv, D, P = 4, 2, 64, 16
    b = ru.Batch([(2, 100), (3, 2), (1, 400), (4, 64)], P, 4)
    q = _queries(b, Hq, D, F32, 7)
    pools = [pu.random_pool(b, Hkv, D, F32, s) for s in (21, 22)]
    at = b.device()
    table = at.pop("page_tables")
    gp = [x.cuda() for x in pools]
    table[0, 3] = b.n_phys          # pages that the pool does not have
    table[0, 0] = -5
    desc = api.make_rows_desc(q.cuda(), gp[0], table, 120, 0.125, max_rows=3)    # lengths are cut to 120, rows to 3
    b.spans = [(2, 100), (3, 2), (1, 120), (4, 64)]
    keep = [r for r in range(b.rows) if r != b.rows - 1]    # the fourth row of the last sequence is beyond max_rows
    sel = torch.tensor([[list(range(7)) + [9000, -3]] * Hkv] * 4, dtype=torch.int32, device="cuda")
    cnt = torch.full((4, Hkv), 9, dtype=torch.int32, device="cuda")
    cnt[3, 1] = 1000                # more than the list's row holds
    for listed in (False, True):
        o, lse = torch.full(q.shape, 5.0, device="cuda"), torch.full((Hq, b.n_rows), 5.0, device="cuda")
        api.paged_attn_fwd_rows(desc, q.cuda(), *gp, table, sel if listed else None, cnt if listed else None, o, lse, **at)
        torch.cuda.synchronize()
        lists = [[[l for l in range(7 if listed else 8) if s or l not in (0, 3)] for _ in range(Hkv)] for s in range(4)]
        wo, wl, to, tl = pu.attend(b, q, *pools, 0.125, lists)
        ru.check("O", o.cpu().double().numpy()[keep], wo[keep], to[keep])
        ru.check("LSE", lse.cpu().double().numpy()[:, keep], wl[:, keep], tl[:, keep])
        assert (o[b.rows - 1:] == 5.0).all() and (o[2] == 0).all() and (lse[:, 2] == -math.inf).all()


def test_lists_without_room_list_nothing():
    b = ru.Batch([(1, 40), (2, 9)], 16, 4)
    q = _queries(b, 4, 64, BF).cuda()
    gp = [pu.random_pool(b, 2, 64, BF, s).cuda() for s in (21, 22)]
    at = b.device()
    table = at.pop("page_tables")
    desc = api.make_rows_desc(q, gp[0], table, 40, 0.125, max_rows=2)
    o, lse = api.paged_attn_fwd_rows(desc, q, *gp, table, torch.zeros((2, 2, 0), dtype=torch.int32, device="cuda"),
                                     torch.ones((2, 2), dtype=torch.int32, device="cuda"), **at)
    torch.cuda.synchronize()
    assert (o == 0).all() and (lse[:, :b.rows] == -math.inf).all()


@pytest.mark.parametrize("dt,D,rows", [(BF, 128, 1), (BF, 64, 40), (F32, 64, 3), (BF, 128, 150)])
def test_strides(dt, D, rows):
    """Pools with tokens before heads, rows that are views of a packed projection, outputs with room between the rows."""
    Hq, Hkv, P = 6, 2, 32
    b = ru.Batch([(rows, 300), (1, 45)], P, 4)
    pools = [pu.random_pool(b, Hkv, D, dt, s) for s in (31, 32)]
    packed = torch.randn((b.n_rows, (Hq + 2 * Hkv) * D), generator=torch.Generator().manual_seed(3)).to(dt).cuda()
    q = packed[:, :Hq * D].unflatten(1, (Hq, D))
    gp = [x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3) for x in pools]
    at = b.device()
    table = at.pop("page_tables")
    room = torch.full((b.n_rows, Hq + 1, D + 16), 5.0, dtype=dt, device="cuda")
    o = room[:, 1:, :D]
    desc = api.make_rows_desc(q, gp[0], table, b.max_len, 0.1, max_rows=rows)
    _, lse = api.paged_attn_fwd_rows(desc, q, *gp, table, o=o, **at)
    torch.cuda.synchronize()
    wo, wl, to, tl = pu.attend(b, q.cpu(), *pools, 0.1)
    live = slice(0, b.rows)
    ru.check("O", o.cpu().double().numpy()[live], wo[live], to[live])
    ru.check("LSE", lse.cpu().double().numpy()[:, live], wl[:, live], tl[:, live])
    assert (room[:, 0] == 5.0).all() and (room[:, :, D:] == 5.0).all() and (room[b.rows:] == 5.0).all()


def test_pool_beyond_4_gib():
    """Offsets past 32 bits."""
    Hq, Hkv, D, P, n_phys = 4, 4, 128, 128, 40000
    pools = [torch.empty((n_phys, Hkv, P, D), dtype=BF, device="cuda") for _ in range(2)]
    assert pools[0].numel() * 2 > 1 << 32
    n = 200
    table = torch.tensor([n_phys - 1, n_phys - 7], dtype=torch.int32, device="cuda")
    b = ru.Batch([(n, n)], P, behind=0)
    small = [pu.random_pool(b, Hkv, D, BF, s) for s in (1, 2)]
    for pool, x in zip(pools, small):
        pool[table.long()] = x[[int(i) for i in b.tables[0, :2]]].cuda()
    q = _queries(b, Hq, D, BF, 8)
    desc = api.make_rows_desc(q.cuda(), pools[0], table, n, 0.1)
    o, lse = api.paged_attn_fwd_rows(desc, q.cuda(), *pools, table)
    torch.cuda.synchronize()
    wo, wl, to, tl = pu.attend(b, q, *small, 0.1)
    ru.check("O", o.cpu().double().numpy(), wo, to)
    ru.check("LSE", lse.cpu().double().numpy(), wl, tl)


@pytest.mark.parametrize("rows", [1, 4])
@pytest.mark.parametrize("dt,D,P", [(BF, 128, 16), (BF, 64, 16), (BF, 128, 128), (BF, 64, 32), (F32, 128, 16), (F32, 64, 64)])
def test_pools_larger_than_the_caches(dt, D, P, rows):
    """Pools and bounds of more than 256 MB, a few pages of which hold something."""
    Hq, Hkv = 28, 4
    b = ru.Batch([(rows, 700), (1, 33), (0, 20), (rows, 2000)], P, 9)
    es = 2 if dt == BF else 4
    n_phys = (300 << 20) // (Hkv * P * D * 2 * es)
    small = [pu.random_pool(b, Hkv, D, dt, s) for s in (1, 2)]
    where = torch.randperm(n_phys, generator=torch.Generator().manual_seed(5))[:b.n_phys]
    pools = [torch.full((n_phys, Hkv, P, D), math.nan, dtype=dt, device="cuda") for _ in range(2)]
    for pool, x in zip(pools, small):
        pool[where.cuda()] = x.cuda()
    q = _queries(b, Hq, D, dt, 8)
    at = b.device()
    max_len = 1 << 19
    table = torch.full((len(b.spans), max_len // P), -1, dtype=torch.int32)
    held = torch.tensor(b.tables)
    table[:, :b.cols] = torch.where(held >= 0, where[held.clamp(min=0).long()].to(torch.int32), -1)
    at["page_tables"] = table.cuda()
    desc = api.make_rows_desc(q.cuda(), pools[0], at["page_tables"], max_len, 0.1, max_rows=rows)
    o, lse = torch.full(q.shape, 5.0, dtype=dt, device="cuda"), torch.full((Hq, b.n_rows), 5.0, device="cuda")
    api.paged_attn_fwd_rows(desc, q.cuda(), *pools, at.pop("page_tables"), o=o, lse=lse, **at)
    torch.cuda.synchronize()
    _verify(b, q, small, 0.1, o, lse)


def test_workspaces_hold_anything_and_results_do_not_depend_on_the_stream():
    b = ru.Batch([(1, 5000), (0, 9), (1, 1), (1, 900)], 128, 14)
    q = _queries(b, 28, 128, BF, 15)
    pools = [pu.random_pool(b, 4, 128, BF, s) for s in (27, 28)]
    got = []
    for fill in (0, 255, 127):
        ws = torch.full((1 << 25,), fill, dtype=torch.uint8, device="cuda")
        got.append(_run(b, q, pools, 0.1, workspace=ws))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got.append(_run(b, q, pools, 0.1))
    for o, lse in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(lse, got[0][1])
    _verify(b, q, pools, 0.1, *got[0])


def test_prompt_in_pieces_then_tokens_and_replays():
    """A prompt appended and attended in pieces that begin and end inside pages, then single tokens in a captured step; all of it against the
    definition over what the cache then holds."""
    Hq, Hkv, D, P, B = 14, 2, 128, 32, 2
    gen = torch.Generator().manual_seed(11)
    cols, lens = 8, [0, 0]
    table = torch.randperm(B * cols, generator=gen).to(torch.int32).view(B, cols).cuda()
    rope = api.rope_tables(cols * P, D)
    pools = [torch.full((B * cols, Hkv, P, D), math.nan, dtype=BF, device="cuda") for _ in range(2)]

    def verify(spans, q_rot, o, lse):
        b = ru.Batch(spans, P, behind=0)
        b.tables, b.n_phys = table.cpu().numpy(), B * cols
        wo, wl, to, tl = pu.attend(b, q_rot.cpu(), *(x.cpu() for x in pools), 0.09)
        ru.check("O", o.cpu().double().numpy(), wo, to)
        ru.check("LSE", lse.cpu().double().numpy(), wl, tl)

    def split(x):
        q, k, v = x.split([Hq * D, Hkv * D, Hkv * D], 1)
        return q.unflatten(1, (Hq, D)), k.unflatten(1, (Hkv, D)), v.unflatten(1, (Hkv, D))

    for piece in ([37, 5], [60, 90], [1, 0], [20, 3]):
        lens = [a + n for a, n in zip(lens, piece)]
        x = torch.randn((sum(piece), (Hq + 2 * Hkv) * D), generator=gen).to(BF).cuda()
        q, k, v = split(x)
        at = dict(seq_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                  row_starts=torch.tensor([0, piece[0], sum(piece)], dtype=torch.int32, device="cuda"))
        desc = api.make_rows_desc(q, pools[0], table, cols * P, 0.09)
        y = api.kv_append_rope(desc, k, v, table, *pools, q=q, rope=rope, **at)
        o, lse = api.paged_attn_fwd_rows(desc, y, *pools, table, **at)
        torch.cuda.synchronize()
        verify(list(zip(piece, lens)), y, o, lse)

    x = torch.zeros((B, (Hq + 2 * Hkv) * D), dtype=BF, device="cuda")
    at = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse, y = torch.zeros((B, Hq, D), dtype=BF, device="cuda"), torch.zeros((Hq, B), device="cuda"), torch.zeros((B, Hq, D), dtype=BF, device="cuda")
    q, k, v = split(x)
    desc = api.make_rows_desc(q, pools[0], table, cols * P, 0.09, max_rows=1)
    ws = torch.empty(max(256, api.rows_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")

    def step():
        at.add_(1)
        api.kv_append_rope(desc, k, v, table, *pools, q=q, q_out=y, rope=rope, seq_lens=at)
        api.paged_attn_fwd_rows(desc, y, *pools, table, o=o, lse=lse, workspace=ws, seq_lens=at)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for i in range(40):
        x.copy_(torch.randn(x.shape, generator=gen).to(BF))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        lens = [t + 1 for t in lens]
        if i % 13 == 0:
            verify([(1, t) for t in lens], y, o, lse)
