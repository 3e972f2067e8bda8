"""GPU tests of the calls over packed rows at the edges of what the header allows."""
import math

import numpy as np
import pytest
import torch

from paper_2602_02108_amd import api

import rows_util as ru

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _batch(spans, P, Hq, Hkv, D, dt, seed, **kw):
    """(batch, queries on the CPU and the GPU, pools as numpy and on the GPU, page tables, the other device arrays)"""
    b = ru.Batch(spans, P, seed, **kw)
    q = torch.randn((b.n_rows, Hq, D), generator=torch.Generator().manual_seed(seed)).to(dt)
    pools = [ru.random_pool(b, Hkv, D, 100 * seed + i) for i in (1, 2)]
    at = b.device()
    return b, q, q.cuda(), pools, [torch.tensor(x, device="cuda") for x in pools], at.pop("page_tables"), at


def _check(b, q, pools, scale, o, lse, terms, lists=None):
    wo, wl, to, tl = ru.attend(b, q, *pools, scale, lists, terms)
    live = slice(0, b.rows)
    ru.check("LSE", lse.cpu().double().numpy()[:, live], wl[:, live], tl[:, live])
    ru.check("O", o.cpu().double().numpy()[live], wo[live], to[live])


# (spans, (Hq, Hkv), D, P): rows that share a cache below, at and past 64, alone and beside others, over few tokens, so that sums of
# weights of either sign come out small and a weight's rounding shows beside the output's own
@pytest.mark.parametrize("spans,heads,D,P", [
    ([(16, 90)], (4, 1), 128, 128), ([(64, 130)], (1, 1), 128, 32), ([(65, 130)], (1, 1), 128, 32), ([(64, 100)], (2, 2), 64, 16),
    ([(65, 100)], (2, 2), 64, 16), ([(9, 60), (1, 50)], (14, 2), 64, 16), ([(1, 100), (40, 170), (2, 64)], (14, 2), 128, 128),
    ([(200, 260), (1, 33)], (28, 4), 128, 128),
])
def test_weights_of_bf16_rows_hold_sixteen_bits_in_every_call(spans, heads, D, P):
    """Two bf16 terms of a weight: 2^-8 of it is left by the first rounding, 2^-8 of that by the second."""
    b, q, gq, pools, gp, table, at = _batch(spans, P, *heads, D, BF, 41)
    scale = 1.0 / math.sqrt(D)
    desc = api.make_rows_desc(gq, gp[0], table, b.max_len, scale, max_rows=b.max_rows)
    o, lse = api.paged_attn_fwd_kvq(desc, gq, *gp, table, **at)
    _check(b, q, pools, scale, o, lse, 2.0 ** -16)


@pytest.mark.parametrize("dt,spans,P", [(BF, [(1, 200), (3, 40)], 128), (F32, [(5, 77)], 16), (BF, [(1, 6000), (2, 50)], 128), (BF, [(80, 300)], 32)])
def test_lists_without_room_list_nothing(dt, spans, P):
    """sel_pages [n_seqs][Hkv][0]: no row sees a token, in a cache that is walked whole and in one that is split."""
    b, q, gq, pools, gp, table, at = _batch(spans, P, 4, 2, 128, dt, 42)
    desc = api.make_rows_desc(gq, gp[0], table, b.max_len, 0.1, max_rows=b.max_rows)
    sel = torch.empty((len(spans), 2, 0), dtype=torch.int32, device="cuda")
    for fill in (0, 3):   # (a count is cut to the row's room)
        cnt = torch.full((len(spans), 2), fill, dtype=torch.int32, device="cuda")
        o, lse = torch.full_like(gq, 5.0), torch.full((4, b.n_rows), 5.0, device="cuda")
        api.paged_attn_fwd_kvq(desc, gq, *gp, table, sel, cnt, o, lse, **at)
        assert (o[:b.rows] == 0).all() and (lse[:, :b.rows] == -math.inf).all()
        assert (o[b.rows:] == 5.0).all() and (lse[:, b.rows:] == 5.0).all()


@pytest.mark.parametrize("dt,Hq,Hkv,D,P", [(BF, 8, 2, 64, 16), (F32, 8, 4, 128, 32)])
def test_many_short_sequences_under_a_loose_bound(dt, Hq, Hkv, D, P):
    """A thousand sequences of a few rows each, max_rows the rows of all."""
    rng = np.random.default_rng(5)
    spans = [(int(n), int(n + rng.integers(0, 40))) for n in rng.integers(0, 7, 1000)]
    b, q, gq, pools, gp, table, at = _batch(spans, P, Hq, Hkv, D, dt, 43)
    desc = api.make_rows_desc(gq, gp[0], table, b.max_len, 0.1)
    assert desc.max_rows == b.n_rows and len(spans) * Hq * b.n_rows > 1 << 24
    o, lse = api.paged_attn_fwd_kvq(desc, gq, *gp, table, **at)
    _check(b, q, pools, 0.1, o, lse, 2.0 ** -22 if dt == F32 else 2.0 ** -16)
    close = api.make_rows_desc(gq, gp[0], table, b.max_len, 0.1, max_rows=b.max_rows)
    k, v = gq[:, :Hkv], gq[:, Hkv:2 * Hkv]
    got = []
    for d in (desc, close):
        x = [t.clone() for t in gp]
        y = api.kvq_append_rope(d, k, v, table, *x, q=gq, **at)
        got.append([y, *x, *api.kvq_read(d, *x, table, **at)])
    assert all(torch.equal(a, c) for a, c in zip(*got)) and not torch.equal(got[0][1], gp[0])


def _garbage(*tensors):
    """The memory that the allocator gives next to tensors of these shapes holds NaN."""
    held = [torch.full_like(t, math.nan) for t in tensors for _ in range(3)]
    torch.cuda.synchronize()
    del held


@pytest.mark.parametrize("lens", [True, False], ids=["lengths", "bound-alone"])
def test_new_tensors_hold_zeros_where_rows_do_not_exist(lens):
    """Equal rows, some sequences shorter than theirs: the surplus in front is written by no call, and is zero in a new tensor."""
    P, D, Hq, Hkv, n = 16, 64, 4, 2, 6
    b = ru.Batch([(n, 4), (n, 4), (n, 4)] if not lens else [(n, 20), (n, 4), (n, 0)], P, 3, behind=0)
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((3 * n, h, D), generator=gen).cuda() for h in (Hq, Hkv, Hkv))
    at = b.device()
    table, seq_lens = at["page_tables"], at["seq_lens"] if lens else None
    live = torch.zeros(3 * n, dtype=torch.bool)
    live[[r for r, _, _ in b.each_row()]] = True
    plain = [torch.randn((b.n_phys, Hkv, P, D), generator=gen).cuda() for _ in range(2)]
    codes = [api.kvq_pool(b.n_phys, Hkv, P, D) for _ in range(2)]
    desc = api.make_rows_desc(q, plain[0], table, b.max_len, max_rows=n)
    kvq = api.make_rows_desc(q, codes[0], table, b.max_len, max_rows=n)
    calls = [lambda: [api.kv_append_rope(desc, k, v, table, *plain, q=q, seq_lens=seq_lens)],
             lambda: [api.kvq_append_rope(kvq, k, v, table, *codes, q=q, seq_lens=seq_lens)],
             lambda: api.kv_append_rope_bwd(desc, *plain, table, d_q=q, seq_lens=seq_lens),
             lambda: api.kvq_read(kvq, *codes, table, seq_lens=seq_lens)]
    for call in calls:
        _garbage(q, k)
        for t in call():
            t = t.cpu()
            assert (t[~live] == 0).all() and (t[live] != 0).any(-1).all()
    _garbage(q, torch.empty(Hq, 3 * n, device="cuda"))
    o, lse = api.paged_attn_fwd_kvq(kvq, q, *codes, table, seq_lens=seq_lens)
    assert (o.cpu()[~live] == 0).all() and (lse.cpu()[:, ~live] == -math.inf).all() and lse.cpu()[:, live].isfinite().all()


@pytest.mark.parametrize("dt,n,t,Hq,Hkv,D,P", [(BF, 1, 60, 2, 2, 64, 16), (F32, 3, 60, 2, 1, 128, 16), (BF, 40, 90, 4, 2, 128, 32), (F32, 1, 3000, 1, 1, 64, 128)])
def test_logits_below_a_floats_range_have_no_weight(dt, n, t, Hq, Hkv, D, P):
    """Every second token's logits are about -2^140, minus infinity in fp32: their weight is zero as it is in 64 bits."""
    b = ru.Batch([(n, t)], P, 6, behind=0)
    q = torch.randn((b.n_rows, Hq, D), generator=torch.Generator().manual_seed(2)).to(dt)
    q[..., 0] = 2.0 ** 60
    pools = [ru.random_pool(b, Hkv, D, s) for s in (51, 52)]
    for l in range(b.cols):
        page = b.tables[0, l]
        x = ru.values(*ru.unpack(pools[0][page], P, D))
        low = (l * P + np.arange(P)) % 2 == 0
        x[:, low, 0], x[:, ~low, :32] = -2.0 ** 80, 0.0
        code, byte = ru.quantise(np.nan_to_num(x))
        pools[0][page] = ru.pack(code, byte)
    at = b.device()
    table, gp, gq = at.pop("page_tables"), [torch.tensor(x, device="cuda") for x in pools], q.cuda()
    desc = api.make_rows_desc(gq, gp[0], table, t, 0.125)
    o, lse = api.paged_attn_fwd_kvq(desc, gq, *gp, table, **at)
    # the seen logits as the definition has them: those of the other tokens, whose first block is zero
    keep = q.clone()
    keep[..., :32] = 0.0
    x, seen = keep.double().numpy(), np.arange(t) % 2 == 1
    for h in range(Hq):
        g = h // (Hq // Hkv)
        k, v = ru.sequence_values(b, pools[0], 0, g, D), ru.sequence_values(b, pools[1], 0, g, D)
        s = 0.125 * (x[:, h] @ k.T)
        s = np.where(seen & (np.arange(t) <= (t - n + np.arange(n))[:, None]), s, -np.inf)
        want = np.log(np.exp(s).sum(-1))
        p = np.exp(s - want[:, None])
        got, glse = o[:, h].cpu().double().numpy(), lse[h].cpu().double().numpy()
        # logits: D exact products summed in fp32 and three roundings; twice that and two terms of the weights; half a step of the output
        off = (D + 3) * 2.0 ** -24 * 0.125 * (np.abs(x[:, h]) @ np.abs(k).T)[:, seen].max() + t * 2.0 ** -24
        tol = (p @ np.abs(v)) * (2.0 ** -16 + 2 * off) + ru.HALF[dt] * np.abs(p @ v)
        assert (np.abs(got - p @ v) <= tol).all() and (np.abs(glse - want) <= off + 2.0 ** -20).all()


def _written(b, P, D, last=None, most=None):
    """Which bytes of a [n_phys][...][tile] pool the rows of a batch take: codes and scales of their tokens."""
    mask = np.zeros((b.n_phys, P * (D // 2 + D // 32)), bool)
    for r, s, pos in b.each_row():
        if pos >= (last or 1 << 40) or r - b.starts[s] >= (most or 1 << 40) or not 0 <= b.tables[s, pos // P] < b.n_phys:
            continue
        at = pos % P
        mask[b.tables[s, pos // P], at * (D // 2):(at + 1) * (D // 2)] = True
        mask[b.tables[s, pos // P], P * (D // 2) + at::P] = True
    return mask


@pytest.mark.parametrize("dt,Hq,Hkv,D,P,spans", [
    (BF, 28, 4, 128, 128, [(1, 1), (1, 128), (1, 129), (1, 300), (0, 77), (0, 0)]), (BF, 4, 2, 128, 32, [(64, 64), (95, 700)]),
    (F32, 2, 1, 64, 16, [(40, 43), (16, 32), (0, 5), (7, 7)]), (BF, 14, 2, 64, 16, [(33, 100), (1, 16), (17, 17), (5, 37)]),
    (F32, 2, 2, 128, 64, [(10, 6), (3, 65)]),
])
@pytest.mark.parametrize("means", [False, True])
def test_a_quantised_append_leaves_every_other_byte(dt, Hq, Hkv, D, P, spans, means):
    b = ru.Batch(spans, P, 8)
    rng = np.random.default_rng(9)
    before = [rng.integers(0, 256, (b.n_phys, Hkv, P * (D // 2 + D // 32)), dtype=np.uint8) for _ in range(2)]
    pools = [torch.tensor(x, device="cuda") for x in before]
    k, v = (torch.randn((b.n_rows, Hkv, D), generator=torch.Generator().manual_seed(s)).to(dt) for s in (1, 2))
    at = b.device()
    table = at.pop("page_tables")
    desc = api.make_rows_desc(k.cuda(), pools[0], table, b.max_len, max_rows=b.max_rows)
    kbar = torch.zeros((len(spans), b.cols, Hkv, D), device="cuda") if means else None
    api.kvq_append_rope(desc, k.cuda(), v.cuda(), table, *pools, kbar_cache=kbar, **at)
    mask = _written(b, P, D)[:, None]
    want = [x.copy() for x in before]
    for r, s, pos in b.each_row():
        for w, x in zip(want, (k, v)):
            codes, scales = ru.unpack(w[b.tables[s, pos // P]], P, D)
            codes[:, pos % P], scales[:, pos % P] = ru.quantise(x[r].double().numpy())
            w[b.tables[s, pos // P]] = ru.pack(codes, scales)
    for name, got, w, old in zip("KV", pools, want, before):
        got = got.cpu().numpy()
        assert np.array_equal(np.where(mask, 0, got), np.where(mask, 0, old)), f"{name}: bytes of no row were written"
        # (N(0, 1) values, none of them zero or infinite: the codes that a search finds, to the sign)
        assert np.array_equal(got, w), f"{name}: {int((got != w).sum())} bytes differ"


def test_bytes_of_rows_that_do_not_exist_stay():
    """Rows in front of the first token, past max_rows, past max_len and of pages that the pool does not have."""
    P, D = 16, 64
    b = ru.Batch([(10, 6), (20, 40), (4, 300)], P, 2)
    b.tables[1, 2] = b.n_phys
    at = b.device()
    table = at.pop("page_tables")
    k, v = (torch.randn((b.n_rows, 1, D), generator=torch.Generator().manual_seed(s)).cuda() for s in (1, 2))
    before = torch.randint(0, 256, (b.n_phys, 1, api.kvq_tile_bytes(P, D)), generator=torch.Generator().manual_seed(3), dtype=torch.uint8)
    pools = [before.cuda() for _ in range(2)]
    desc = api.make_rows_desc(k, pools[0], table, 48, max_rows=18)
    api.kvq_append_rope(desc, k, v, table, *pools, **at)
    b.spans = [(n, min(t, 48)) for n, t in b.spans]
    mask = _written(b, P, D, 48, 18)[:, None]
    assert mask.any()
    for got in pools:
        assert np.array_equal(np.where(mask, 0, got.cpu().numpy()), np.where(mask, 0, before.numpy()))


def test_codes_past_the_caches_give_the_same_bits():
    """A pool past the last cache's size under a bound to match is read past it: the same rows over a small pool, and over the large one."""
    b, q, gq, pools, gp, table, at = _batch([(1, 900), (2, 5000), (0, 3), (1, 1)], 128, 8, 4, 128, BF, 44)
    n_phys = 4000   # of 2 x 34 KiB
    large = [torch.full((n_phys, *x.shape[1:]), 255, dtype=torch.uint8, device="cuda") for x in gp]
    for x, y in zip(large, gp):
        x[:b.n_phys] = y
    assert 2 * large[0].numel() > 256 << 20
    room = torch.cat([table, torch.full((4, 8192 - table.shape[1]), -1, dtype=torch.int32, device="cuda")], 1)
    got = []
    for x in (gp, large):
        desc = api.make_rows_desc(gq, x[0], room, 1 << 20, 0.1, max_rows=2)
        got.append(api.paged_attn_fwd_kvq(desc, gq, *x, room, **at))
    assert all(torch.equal(a, c) for a, c in zip(*got))
    _check(b, q, pools, 0.1, *got[0], 2.0 ** -16)


@pytest.mark.parametrize("dt,Hq,Hkv,D,P,spans", [
    (BF, 14, 2, 128, 128, [(1, 9000), (300, 1000), (4, 5000), (0, 70), (1, 1)]), (F32, 4, 2, 64, 16, [(200, 200), (1, 7000), (1, 3)]),
    (BF, 4, 1, 64, 32, [(17, 20000), (130, 131)]),
])
def test_prompts_beside_long_single_tokens(dt, Hq, Hkv, D, P, spans):
    """One call with a prompt, drafted and single tokens over long caches: each as the definition has it, and the single ones as alone."""
    b, q, gq, pools, gp, table, at = _batch(spans, P, Hq, Hkv, D, dt, 45)
    desc = api.make_rows_desc(gq, gp[0], table, b.max_len, 0.1, max_rows=b.max_rows)
    o, lse = api.paged_attn_fwd_kvq(desc, gq, *gp, table, **at)
    terms = 2.0 ** -22 if dt == F32 else 2.0 ** -16
    _check(b, q, pools, 0.1, o, lse, terms)
    for s, (n, t) in enumerate(spans):
        if 0 < n < 20:
            r = slice(b.starts[s], b.starts[s] + n)
            one = api.make_rows_desc(gq[r], gp[0], table[s], t, 0.1)
            o1, l1 = o.clone(), lse.clone()
            o1[r], l1[:, r] = api.paged_attn_fwd_kvq(one, gq[r], *gp, table[s])
            _check(b, q, pools, 0.1, o1, l1, terms)


@pytest.mark.parametrize("flag", [1, np.bool_(True)])
def test_pairs_of_a_rope_are_neighbours_by_any_truth_value(flag):
    b = ru.Batch([(5, 9)], 16, 1, behind=0)
    x = torch.randn((5, 2, 64), generator=torch.Generator().manual_seed(1)).cuda()
    cos, sin = (t.cuda() for t in ru.tables(9, 64))
    pools = [torch.zeros((b.n_phys, 2, 16, 64), device="cuda") for _ in range(2)]
    at = b.device()
    table = at.pop("page_tables")
    desc = api.make_rows_desc(x, pools[0], table, 9)
    rope = api.Rope(cos, sin)
    halves = api.kv_append_rope(desc, x, x, table, *pools, q=x, rope=rope, **at)
    rope.interleaved = flag
    got = api.kv_append_rope(desc, x, x, table, *pools, q=x, rope=rope, **at)
    want = api.kv_append_rope(desc, x, x, table, *pools, q=x, rope=api.Rope(cos, sin, True), **at)
    assert torch.equal(got, want) and not torch.equal(got, halves)


@pytest.mark.parametrize("dt,spans,Hq,Hkv,D,P", [(BF, [(6, 40), (1, 20)], 4, 2, 128, 16), (BF, [(30, 40), (9, 200)], 14, 2, 64, 32), (BF, [(70, 150)], 3, 3, 128, 64),
                                                 (F32, [(20, 90), (2, 300)], 4, 1, 128, 16)])
def test_nan_blocks_leave_the_other_rows_their_bits(dt, spans, Hq, Hkv, D, P):
    """NaN blocks of K and V near the end of each sequence: the rows that see them are NaN where they should be, the others as exact as ever."""
    b, q, gq, pools, gp, table, at = _batch(spans, P, Hq, Hkv, D, dt, 46)
    for s, (n, t) in enumerate(spans):
        for pool, back, g, block in ((pools[1], n // 2 + 1, 0, D // 32 - 1), (pools[1], 1, Hkv - 1, 0), (pools[0], 2, Hkv - 1, 1)):
            pos = max(t - back, 0)
            pool[b.tables[s, pos // P], g, P * D // 2 + block * P + pos % P] = 255
            gp[0 if pool is pools[0] else 1].copy_(torch.tensor(pool))
    desc = api.make_rows_desc(gq, gp[0], table, b.max_len, 0.1, max_rows=b.max_rows)
    o, lse = api.paged_attn_fwd_kvq(desc, gq, *gp, table, **at)
    _check(b, q, pools, 0.1, o, lse, 2.0 ** -22 if dt == F32 else 2.0 ** -16)
    assert o[:b.rows].isnan().any() and o[:b.rows].isfinite().any()
