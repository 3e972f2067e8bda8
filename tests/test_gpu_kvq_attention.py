"""GPU tests of the attention over a cache held in 4 bits, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2602_02108_amd import api

import rows_util as ru

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _run(b, q, pools, scale, lists=None, max_rows=None, workspace=None, max_len=None):
    at = b.device()
    table = at.pop("page_tables")
    g = q.cuda()
    gp = [torch.tensor(x, device="cuda") for x in pools]
    if max_len:   # a table with room for that many tokens
        table = torch.cat([table, torch.full((table.shape[0], max_len // b.P - table.shape[1]), -1, dtype=torch.int32, device="cuda")], 1)
    desc = api.make_rows_desc(g, gp[0], table, max_len or b.max_len, scale, max_rows=max_rows or b.max_rows)
    o = torch.full_like(g, 5.0)
    lse = torch.full((g.shape[1], g.shape[0]), 5.0, device="cuda")
    sel = cnt = None
    if lists is not None:
        width = max(1, max(len(x) for s in lists for x in s)) + 2
        sel = torch.full((len(b.spans), pools[0].shape[1], width), 7777777, dtype=torch.int32)
        cnt = torch.tensor([[len(x) for x in s] for s in lists], dtype=torch.int32)
        for i, s in enumerate(lists):
            for h, x in enumerate(s):
                sel[i, h, :len(x)] = torch.tensor(x, dtype=torch.int32)
        sel, cnt = sel.cuda(), cnt.cuda()
    api.paged_attn_fwd_kvq(desc, g, *gp, table, sel, cnt, o, lse, workspace, **at)
    torch.cuda.synchronize()
    return o, lse


def _verify(b, q, pools, scale, o, lse, lists=None, terms=None):
    # weights of rows that share a wave with many others are rounded to one bf16 (2^-8 at most), of few rows to two (2^-16)
    G = q.shape[1] // pools[0].shape[1]
    if terms is None:
        terms = 2.0 ** -22 if q.dtype == F32 else 2.0 ** -8 if b.max_rows * G > 32 else 2.0 ** -15
    wo, wl, to, tl = ru.attend(b, q, *pools, scale, lists, terms)
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
    (F32, (2, 1), 64, 16, [(1, 1), (3, 33), (8, 100), (2, 16)]),
    (F32, (28, 4), 128, 128, [(1, 400), (1, 1)]),
    (F32, (6, 2), 128, 16, [(9, 200), (4, 31)]),
    (F32, (14, 2), 64, 128, [(40, 170), (0, 3), (3, 500)]),
]
IDS = [f"{'bf16' if c[0] == BF else 'f32'}-h{c[1][0]}-{c[1][1]}-d{c[2]}-p{c[3]}-{i}" for i, c in enumerate(CASES)]


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_every_page(case):
    dt, (Hq, Hkv), D, P, spans = case
    b = ru.Batch(spans, P, 5)
    q = torch.randn((b.n_rows, Hq, D), generator=torch.Generator().manual_seed(1)).to(dt)
    pools = [ru.random_pool(b, Hkv, D, s) for s in (11, 12)]
    scale = 1.0 / math.sqrt(D)
    o, lse = _run(b, q, pools, scale)
    _verify(b, q, pools, scale, o, lse)


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
    q = torch.randn((b.n_rows, Hq, D), generator=torch.Generator().manual_seed(2)).to(dt)
    pools = [ru.random_pool(b, Hkv, D, s) for s in (13, 14)]
    scale = 1.0 / math.sqrt(D)
    o, lse = _run(b, q, pools, scale, lists)
    _verify(b, q, pools, scale, o, lse, lists)


@pytest.mark.parametrize("dt,Hq,Hkv,D,P,spans,listed", [
    (BF, 7, 1, 128, 128, [(1, 40000)], False),             # a long cache: tokens split over workgroups
    (F32, 2, 1, 64, 16, [(1, 30011), (1, 200)], False),    # small pages: many windows of page ids
    (BF, 28, 4, 128, 128, [(2, 20000), (1, 3000)], True),
    (BF, 14, 2, 64, 16, [(3, 9000)], True),
    (BF, 28, 4, 128, 128, [(1200, 1300), (1171, 1171)], False),   # many rows: row blocks of one wave
    (F32, 28, 4, 64, 32, [(600, 700), (300, 1000)], False),
    (BF, 8, 1, 64, 16, [(300, 2000)], True),
])
def test_long_and_many(dt, Hq, Hkv, D, P, spans, listed):
    b = ru.Batch(spans, P, 7)
    lists = None
    if listed:
        rng = np.random.default_rng(9)
        lists = [[sorted(int(x) for x in rng.permutation(-(-t // P))[:-(-t // P) * 2 // 3]) for _ in range(Hkv)] for _, t in spans]
    q = torch.randn((b.n_rows, Hq, D), generator=torch.Generator().manual_seed(3)).to(dt)
    pools = [ru.random_pool(b, Hkv, D, s) for s in (15, 16)]
    scale = 1.0 / math.sqrt(D)
    o, lse = _run(b, q, pools, scale, lists)
    _verify(b, q, pools, scale, o, lse, lists)


@pytest.mark.parametrize("dt,Hq,Hkv,D,P,spans", [
    (BF, 28, 4, 128, 128, [(1, 700), (1, 5), (0, 0), (1, 3000)]),
    (BF, 8, 4, 64, 32, [(2, 700), (1, 1)]),
    (BF, 8, 4, 128, 16, [(1, 40), (1, 700)]),
    (F32, 8, 4, 128, 64, [(1, 700), (3, 70)]),
    (F32, 4, 4, 64, 128, [(4, 1300)]),
    (BF, 14, 2, 128, 128, [(40, 900), (3, 50)]),
])
def test_room_for_far_longer_sequences(dt, Hq, Hkv, D, P, spans):
    """A bound of two million tokens a sequence (more cache than stays in the caches, thousands of parts at most) over short ones."""
    b = ru.Batch(spans, P, 12)
    q = torch.randn((b.n_rows, Hq, D), generator=torch.Generator().manual_seed(13)).to(dt)
    pools = [ru.random_pool(b, Hkv, D, s) for s in (25, 26)]
    o, lse = _run(b, q, pools, 0.1, max_len=1 << 21)
    _verify(b, q, pools, 0.1, o, lse)


@pytest.mark.parametrize("dt,Hq,Hkv,D,P,spans", [
    (BF, 14, 2, 128, 128, [(40, 900), (1, 300)]), (BF, 4, 2, 64, 16, [(40, 500), (3, 30)]), (BF, 4, 2, 128, 64, [(2, 9000)]),
    (BF, 7, 1, 128, 128, [(64, 20000)]), (F32, 4, 2, 64, 32, [(20, 300)]),
])
def test_constant_values_come_out_as_they_are(dt, Hq, Hkv, D, P, spans):
    """V is 1.5 throughout: O is 1.5 whatever the weights are rounded to (they are divided by the sum of what the product took), in
    every route; keys give the first tokens larger logits, so that the others' weights are alike and no powers of two."""
    b = ru.Batch(spans, P, 18)
    q = torch.ones((b.n_rows, Hq, D), dtype=dt)
    pools = [ru.random_pool(b, Hkv, D, s) for s in (29, 30)]
    for s, (_, t) in enumerate(b.spans):
        for l in range(-(-t // P)):
            pos = l * P + np.arange(P)
            k = np.where(pos < 5, 0.5, 0.0)[None, :, None] * np.ones((Hkv, 1, D))
            for pool, x in ((pools[0], k), (pools[1], np.full((Hkv, P, D), 1.5))):
                code, byte = ru.quantise(x)
                byte[:, min(P, t - l * P):] = 255
                pool[b.tables[s, l]] = ru.pack(code, byte)
    o, lse = _run(b, q, pools, 0.37 / D)
    # one rounding of the output, of a value that is off by the sums' 2^-20 at most
    assert (o[:b.rows].double() - 1.5).abs().max() <= 1.5 * (2.0 ** -19 if dt == F32 else 0.0)
    _verify(b, q, pools, 0.37 / D, o, lse)


def test_workspaces_hold_anything():
    """Parts are written before they are read: the same bits whatever the workspace held."""
    b = ru.Batch([(1, 5000), (0, 9), (1, 1), (1, 900)], 128, 14)
    q = torch.randn((b.n_rows, 28, 128), generator=torch.Generator().manual_seed(15)).to(BF)
    pools = [ru.random_pool(b, 4, 128, s) for s in (27, 28)]
    got = []
    for fill in (0, 255, 127):
        ws = torch.full((1 << 25,), fill, dtype=torch.uint8, device="cuda")
        got.append(_run(b, q, pools, 0.1, workspace=ws))
    for o, lse in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(lse, got[0][1])
    _verify(b, q, pools, 0.1, *got[0])


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("order", ["rising", "falling", "spikes"])
def test_logits_far_apart(dt, order):
    """Logits over a wide range, so that the reference of the softmax moves often, seldom or in jumps."""
    Hq, Hkv, D, P = 4, 2, 64, 16
    b = ru.Batch([(2, 600), (1, 77)], P, 3)
    q = torch.randn((b.n_rows, Hq, D), generator=torch.Generator().manual_seed(4)).to(dt)
    pools = [ru.random_pool(b, Hkv, D, s) for s in (17, 18)]
    direction = np.sign(q[0, 0].double().numpy())
    for s, (_, t) in enumerate(b.spans):
        for l in range(-(-t // P)):
            pos = l * P + np.arange(P)
            size = {"rising": pos / 8.0, "falling": (t - pos) / 8.0, "spikes": np.where(pos % 97 == 5, 30.0 + pos / 16.0, 0.1)}[order]
            code, byte = ru.quantise(np.repeat((size[:, None] * direction)[None], Hkv, 0))
            held = min(P, t - l * P)
            byte[:, held:] = 255
            pools[0][b.tables[s, l]] = ru.pack(code, byte)
    o, lse = _run(b, q, pools, 0.125)
    _verify(b, q, pools, 0.125, o, lse)


@pytest.mark.parametrize("dt,spans,Hq,Hkv,D", [(BF, [(6, 40), (1, 20)], 4, 2, 128), (F32, [(6, 40), (1, 20)], 4, 2, 64), (BF, [(30, 40), (9, 200)], 14, 2, 64)])
def test_values_that_are_not_finite(dt, spans, Hq, Hkv, D):
    """NaN blocks in K and V of tokens that some rows see, infinite and NaN queries: only the rows that see them change."""
    P = 16
    b = ru.Batch(spans, P, 4)
    q = torch.randn((b.n_rows, Hq, D), generator=torch.Generator().manual_seed(6)).to(dt)
    pools = [ru.random_pool(b, Hkv, D, s) for s in (19, 20)]

    def spoil(pool, s, pos, g, block):
        code, byte = ru.unpack(pool[b.tables[s, pos // P]], P, D)
        byte[g, pos % P, block] = 255
        pool[b.tables[s, pos // P]] = ru.pack(code, byte)

    n, t = spans[0]
    spoil(pools[1], 0, t - n + 2, 0, D // 32 - 1)    # seen by the rows from the third on
    spoil(pools[1], 0, t - 1, 1, 0)                  # by the last row alone
    spoil(pools[0], 0, t - 2, 0, 1)
    spoil(pools[1], 1, 3, 1, 1)                      # by every row of the second sequence
    q[1, 1, 3] = float("nan")
    q[2, Hq - 1, 0] = float("inf")
    o, lse = _run(b, q, pools, 0.125)
    wo, wl, to, tl = ru.attend(b, q, *pools, 0.125, None, 2.0 ** -22 if dt == F32 else 2.0 ** -8)
    # an infinite query's logits are infinite of either sign or NaN: its row holds nothing
    wo[2, Hq - 1], wl[Hq - 1, 2] = np.nan, np.nan
    live = slice(0, b.rows)
    assert np.isnan(wo[live]).any() and np.isfinite(wo[live]).mean() > 0.5
    ru.check("LSE", lse.cpu().double().numpy()[:, live], wl[:, live], tl[:, live])
    ru.check("O", o.cpu().double().numpy()[live], wo[live], to[live])


def test_pages_and_lengths_out_of_range_are_not_seen():
    Hq, Hkv, D, P = 4, 2, 64, 16
    b = ru.Batch([(2, 100), (3, 2), (1, 400), (4, 64)], P, 4)
    q = torch.randn((b.n_rows, Hq, D), generator=torch.Generator().manual_seed(7))
    pools = [ru.random_pool(b, Hkv, D, s) for s in (21, 22)]
    at = b.device()
    table = at.pop("page_tables")
    gp = [torch.tensor(x, device="cuda") for x in pools]
    table[0, 3] = b.n_phys          # pages that the pool does not have
    table[0, 0] = -5
    desc = api.make_rows_desc(q.cuda(), gp[0], table, 120, 0.125, max_rows=3)    # lengths are cut to 120, rows to 3
    o, lse = torch.full(q.shape, 5.0, device="cuda"), torch.full((Hq, b.n_rows), 5.0, device="cuda")
    sel = torch.tensor([[list(range(7)) + [9000, -3]] * Hkv] * 4, dtype=torch.int32, device="cuda")
    cnt = torch.full((4, Hkv), 9, dtype=torch.int32, device="cuda")
    cnt[3, 1] = 1000                # more than the list's row holds
    api.paged_attn_fwd_kvq(desc, q.cuda(), *gp, table, None, None, o, lse, **at)
    torch.cuda.synchronize()
    b.spans = [(2, 100), (3, 2), (1, 120), (4, 64)]
    lists = [[[l for l in range(8) if l not in (0, 3)] if s == 0 else list(range(8)) for _ in range(Hkv)] for s in range(4)]
    wo, wl, to, tl = ru.attend(b, q, *pools, 0.125, lists, 2.0 ** -22)
    keep = [r for r in range(b.rows) if r != b.rows - 1]    # the fourth row of the last sequence is beyond max_rows
    ru.check("O", o.cpu().double().numpy()[keep], wo[keep], to[keep])
    ru.check("LSE", lse.cpu().double().numpy()[:, keep], wl[:, keep], tl[:, keep])
    assert (o[b.rows - 1:] == 5.0).all() and (o[2] == 0).all() and (lse[:, 2] == -math.inf).all()
    o2, lse2 = torch.full_like(o, 5.0), torch.full_like(lse, 5.0)
    api.paged_attn_fwd_kvq(desc, q.cuda(), *gp, table, sel, cnt, o2, lse2, **at)
    torch.cuda.synchronize()
    lists = [[[l for l in x if l < 7] for x in s] for s in lists]
    wo, wl, to, tl = ru.attend(b, q, *pools, 0.125, lists, 2.0 ** -22)
    ru.check("O", o2.cpu().double().numpy()[keep], wo[keep], to[keep])


def test_pool_beyond_4_gib():
    """Offsets past 32 bits, in the append, the read and the attention."""
    Hq, Hkv, D, P, n_phys = 2, 4, 128, 128, 130000
    tile = api.kvq_tile_bytes(P, D)
    assert n_phys * Hkv * tile > 1 << 32
    pools = [torch.empty((n_phys, Hkv, tile), dtype=torch.uint8, device="cuda") for _ in range(2)]
    n = 200
    table = torch.tensor([n_phys - 1, n_phys - 7], dtype=torch.int32, device="cuda")
    gen = torch.Generator().manual_seed(8)
    q, k, v = (torch.randn((n, h, D), generator=gen) for h in (4, Hkv, Hkv))
    desc = api.make_rows_desc(q.cuda(), pools[0], table, n, 0.1)
    y = api.kvq_append_rope(desc, k.cuda(), v.cuda(), table, *pools, q=q.cuda())
    o, lse = api.paged_attn_fwd_kvq(desc, y, *pools, table)
    kh, vh = api.kvq_read(desc, *pools, table)
    torch.cuda.synchronize()
    kq, vq = (ru.values(*ru.quantise(x.double().numpy())) for x in (k, v))
    assert np.array_equal(kh.cpu().double().numpy(), kq) and np.array_equal(vh.cpu().double().numpy(), vq)
    s = 0.1 * np.einsum("ihd,thd->hit", q.double().numpy(), kq)
    s = np.where(np.tril(np.ones((n, n), bool))[None], s, -np.inf)
    p = np.exp(s - s.max(-1, keepdims=True))
    want = np.einsum("hit,thd->ihd", p / p.sum(-1, keepdims=True), vq)
    assert np.abs(o.cpu().double().numpy() - want).max() < 1e-5   # 200 values of up to 6, each 2^-20 off at most


def test_results_do_not_depend_on_the_run_or_the_stream():
    b = ru.Batch([(2, 9000), (1, 300)], 16, 4)
    q = torch.randn((b.n_rows, 14, 64), generator=torch.Generator().manual_seed(7)).to(BF).cuda()
    gp = [torch.tensor(ru.random_pool(b, 2, 64, s), device="cuda") for s in (23, 24)]
    at = b.device()
    table = at.pop("page_tables")
    desc = api.make_rows_desc(q, gp[0], table, b.max_len, 0.125, max_rows=2)
    assert api.kvq_workspace_bytes(desc) > 0
    first = api.paged_attn_fwd_kvq(desc, q, *gp, table, **at)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = api.paged_attn_fwd_kvq(desc, q, *gp, table, **at)
    third = api.paged_attn_fwd_kvq(desc, q, *gp, table, **at)
    torch.cuda.synchronize()
    for a, c in ((first, second), (first, third)):
        assert torch.equal(a[0][:b.rows], c[0][:b.rows]) and torch.equal(a[1][:, :b.rows], c[1][:, :b.rows])


def test_captured_generation_replays_like_eager_steps():
    """A step of generation (append, attention) captured once: lengths and tables are read on the device, so replays follow them."""
    Hq, Hkv, D, P, B, steps = 14, 2, 128, 16, 3, 20
    gen = torch.Generator().manual_seed(11)
    lens0 = [30, 1, 15]
    cols = 8
    table = torch.randperm(B * cols, generator=gen).to(torch.int32).view(B, cols).cuda()
    rope = api.rope_tables(cols * P, D)
    xs = [torch.randn((B, (Hq + 2 * Hkv) * D), generator=gen).to(BF).cuda() for _ in range(steps)]

    def fresh():
        g2 = torch.Generator().manual_seed(12)
        pools = [api.kvq_pool(B * cols, Hkv, P, D) for _ in range(2)]
        for x in pools:
            x.copy_(torch.randint(0, 256, x.shape, generator=g2, dtype=torch.uint8))
            x[:, :, P * D // 2:] = 120
        return pools, torch.tensor(lens0, dtype=torch.int32, device="cuda"), torch.zeros((B, cols, Hkv, D), device="cuda")

    def buffers():
        return torch.zeros((B, (Hq + 2 * Hkv) * D), dtype=BF, device="cuda"), torch.zeros((B, Hq, D), dtype=BF, device="cuda"), \
            torch.zeros((Hq, B), device="cuda")

    def step(x, pools, lens, kbar, o, lse, ws):
        lens += 1
        q, k, v = x.split([Hq * D, Hkv * D, Hkv * D], 1)
        q, k, v = q.unflatten(1, (Hq, D)), k.unflatten(1, (Hkv, D)), v.unflatten(1, (Hkv, D))
        desc = api.make_rows_desc(q, pools[0], table, cols * P, 0.09, max_rows=1)
        y = api.kvq_append_rope(desc, k, v, table, *pools, q=q, rope=rope, kbar_cache=kbar, seq_lens=lens)
        api.paged_attn_fwd_kvq(desc, y, *pools, table, o=o, lse=lse, workspace=ws, seq_lens=lens)

    x, o, lse = buffers()
    pools, lens, kbar = fresh()
    desc = api.make_rows_desc(o, pools[0], table, cols * P, 0.09, max_rows=1)
    ws = torch.empty(max(256, api.kvq_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
    want = []
    for i in range(steps):
        x.copy_(xs[i])
        step(x, pools, lens, kbar, o, lse, ws)
        torch.cuda.synchronize()
        want.append([t.clone() for t in (o, lse, *pools, kbar)])
    assert kbar.any()

    pools, lens, kbar = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step(x, pools, lens, kbar, o, lse, ws)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step(x, pools, lens, kbar, o, lse, ws)
    torch.cuda.current_stream().wait_stream(side)
    start = fresh()
    for a, c in zip((*pools, lens, kbar), (*start[0], start[1], start[2])):
        a.copy_(c)
    for i in range(steps):
        x.copy_(xs[i])
        o.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip((o, lse, *pools, kbar), want[i]):
            assert torch.equal(a, c), f"replay {i}"


def test_two_captured_graphs_share_a_workspace():
    """Nothing stays in a workspace from call to call: graphs of other shapes replayed in turn over one give the eager results."""
    ws = torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
    calls = []
    for seed, (spans, Hq, Hkv, D, P) in enumerate([([(1, 6000), (1, 40)], 28, 4, 128, 128), ([(5, 3000), (2, 900), (5, 5)], 14, 2, 64, 16)]):
        b = ru.Batch(spans, P, seed)
        q = torch.randn((b.n_rows, Hq, D), generator=torch.Generator().manual_seed(seed)).to(BF).cuda()
        gp = [torch.tensor(ru.random_pool(b, Hkv, D, 31 + 2 * seed + i), device="cuda") for i in range(2)]
        at = b.device()
        table = at.pop("page_tables")
        desc = api.make_rows_desc(q, gp[0], table, b.max_len, 0.1, max_rows=b.max_rows)
        assert 0 < api.kvq_workspace_bytes(desc) <= ws.numel()
        o, lse = torch.zeros_like(q), torch.zeros((Hq, b.n_rows), device="cuda")

        def call(desc=desc, q=q, gp=gp, table=table, at=at, o=o, lse=lse):
            api.paged_attn_fwd_kvq(desc, q, *gp, table, o=o, lse=lse, workspace=ws, **at)

        call()
        torch.cuda.synchronize()
        want = o.clone(), lse.clone()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            call()
        calls.append((graph, o, lse, want, call))   # (the call holds what its graph reads)
    for _ in range(3):
        for graph, o, lse, want, _call in calls:
            o.fill_(7.0)
            lse.fill_(7.0)
            o[-2:], lse[:, -2:] = 0.0, 0.0   # (rows of no sequence)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


def test_rows_in_front_of_the_first_sequence_are_left_alone():
    b = ru.Batch([(3, 50), (2, 7)], 16, 3, behind=4)
    q = torch.randn((b.n_rows, 4, 64), generator=torch.Generator().manual_seed(3)).cuda()
    gp = [torch.tensor(ru.random_pool(b, 2, 64, s), device="cuda") for s in (35, 36)]
    at = b.device()
    table = at.pop("page_tables")
    desc = api.make_rows_desc(q, gp[0], table, b.max_len, 0.1, max_rows=3)
    o, lse = api.paged_attn_fwd_kvq(desc, q, *gp, table, **at)
    moved = torch.cat([q[-2:], q[:-2]])
    at["row_starts"] += 2
    o2, lse2 = torch.full_like(o, 9.0), torch.full_like(lse, 9.0)
    api.paged_attn_fwd_kvq(desc, moved, *gp, table, o=o2, lse=lse2, **at)
    torch.cuda.synchronize()
    assert torch.equal(o2[2:7], o[:5]) and torch.equal(lse2[:, 2:7], lse[:, :5])
    assert (o2[:2] == 9.0).all() and (o2[7:] == 9.0).all() and (lse2[:, :2] == 9.0).all() and (lse2[:, 7:] == 9.0).all()


def test_prompt_in_chunks_then_generation():
    """A prompt goes through in chunks -- append with rotation and means, pages picked from the means, attention over the picked pages --
    and tokens are generated over all of the cache; every output against 64 bits over what the cache holds."""
    Hq, Hkv, D, P, C, n_chunks, top_k = 6, 2, 64, 16, 64, 4, 3
    n_pages = n_chunks * C // P + 2
    table_np = np.random.default_rng(3).permutation(n_pages + 2)[:n_pages].astype(np.int32)
    table = torch.tensor(table_np, device="cuda")
    pools = [api.kvq_pool(n_pages + 2, Hkv, P, D) for _ in range(2)]
    for x in pools:
        x.fill_(255)
    kbar = torch.zeros((n_pages, Hkv, D), device="cuda")
    rope = api.rope_tables(n_pages * P, D)
    scale = 1.0 / math.sqrt(D)
    gen = torch.Generator().manual_seed(21)

    def rows(n):
        return [torch.randn((n, h, D), generator=gen).to(BF).cuda() for h in (Hq, Hkv, Hkv)]

    def verify(o, lse, y, n, t, lists):
        class B:
            pass
        b = B()
        b.spans, b.P, b.starts, b.tables = [(n, t)], P, [0, n], table_np[None]
        wo, wl, to, tl = ru.attend(b, y.cpu(), *(x.cpu().numpy() for x in pools), scale, lists, 2.0 ** -8)
        ru.check("O", o.cpu().double().numpy(), wo, to)
        ru.check("LSE", lse.cpu().double().numpy(), wl, tl)

    for c in range(n_chunks):
        t = (c + 1) * C
        q, k, v = rows(C)
        desc = api.make_rows_desc(q, pools[0], table, t, scale)
        y = api.kvq_append_rope(desc, k, v, table, *pools, q=q, rope=rope, kbar_cache=kbar)
        pick = api.means_desc(y, Hkv, P, t, scale)
        sel, cnt = api.page_score_topk_cached(pick, y, kbar, top_k)
        o, lse = api.paged_attn_fwd_kvq(desc, y, *pools, table, sel, cnt)
        torch.cuda.synchronize()
        for l in range(t // P):
            keys = ru.values(*ru.unpack(pools[0][table_np[l]].cpu().numpy(), P, D))
            assert np.allclose(kbar[l].cpu().numpy(), keys.mean(1), rtol=0, atol=16 * 6 * 2.0 ** -24)
        lists = [[[int(x) for x in sel[g, :int(cnt[g])]] for g in range(Hkv)]]
        assert all(len(x) == min(top_k, c * C // P) + C // P for x in lists[0])
        verify(o, lse, y, C, t, lists)
    for i in range(5):
        t = n_chunks * C + 1 + i
        q, k, v = rows(1)
        desc = api.make_rows_desc(q, pools[0], table, t, scale)
        y = api.kvq_append_rope(desc, k, v, table, *pools, q=q, rope=rope, kbar_cache=kbar)
        o, lse = api.paged_attn_fwd_kvq(desc, y, *pools, table)
        torch.cuda.synchronize()
        verify(o, lse, y, 1, t, None)


def test_training_step_with_rotation_against_autograd():
    """Append with rotation, dense attention forward and backward over two chunks, the append's backward: the gradients of the un-rotated
    projections against autograd in 64 bits over the whole sequence."""
    Hq, Hkv, D, P, C, n_chunks = 4, 2, 64, 16, 32, 2
    N, scale = C * n_chunks, 0.125
    gen = torch.Generator().manual_seed(31)
    x = [torch.randn((N, h, D), generator=gen) for h in (Hq, Hkv, Hkv)]
    d_o = torch.randn((N, Hq, D), generator=gen)
    rope = api.rope_tables(N, D)
    n = N // P
    table = torch.randperm(n + 3, generator=gen)[:n].to(torch.int32).cuda()
    pools = [torch.zeros((n + 3, Hkv, P, D), device="cuda") for _ in range(4)]
    k_pool, v_pool, dk_pool, dv_pool = pools
    kept, outs = [], []
    for c in range(n_chunks):
        q, k, v = (t[c * C:(c + 1) * C].cuda() for t in x)
        rd = api.make_rows_desc(q, k_pool, table, (c + 1) * C)
        y = api.kv_append_rope(rd, k, v, table, k_pool, v_pool, q=q, rope=rope)
        desc = api.make_desc(y, k_pool, (c + 1) * C, scale)
        kept.append((rd, desc, y, *api.paged_attn_fwd(desc, y, k_pool, v_pool, table)))
        outs.append(kept[-1][3])
    grads = [None] * n_chunks
    for c in reversed(range(n_chunks)):
        rd, desc, y, o, lse = kept[c]
        dy = api.paged_attn_bwd(desc, y, k_pool, v_pool, table, o, lse, d_o[c * C:(c + 1) * C].cuda(), dk_pool, dv_pool)
        grads[c] = api.kv_append_rope_bwd(rd, dk_pool, dv_pool, table, d_q=dy, rope=rope)
    torch.cuda.synchronize()

    leaves = [t.double().requires_grad_() for t in x]
    cos, sin = rope.cos.cpu().double(), rope.sin.cpu().double()

    def turn(t):
        a, b = t[..., :D // 2], t[..., D // 2:]
        c, s = cos[:N, None], sin[:N, None]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    q, k, v = turn(leaves[0]), turn(leaves[1]), leaves[2]
    k, v = (t.repeat_interleave(Hq // Hkv, 1) for t in (k, v))
    s = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0)) * scale
    s = s.masked_fill(torch.ones((N, N), dtype=torch.bool).triu(1), -math.inf)
    o = torch.matmul(s.softmax(-1), v.transpose(0, 1)).transpose(0, 1)
    (o * d_o.double()).sum().backward()
    # fp32 throughout: sums of up to 64 tokens and 2 heads of values of size 1 to 10, 2^-24 each and a few dozen roundings
    assert (torch.cat(outs).cpu().double() - o).abs().max() < 2e-5
    for i, leaf in enumerate(leaves):
        got = torch.cat([g[i] for g in grads]).cpu().double()
        assert (got - leaf.grad).abs().max() < 1e-4 * max(1.0, leaf.grad.abs().max())
