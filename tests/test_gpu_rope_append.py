"""GPU tests of the rotating append, its backward and the append into a cache of 4-bit codes, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_02108_amd import api

import rows_util as ru

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
# (type, (Hq, Hkv), D, P, spans, rot_dim, interleaved): whole chunks, single tokens, pages begun and left in the middle, idle and empty sequences
CASES = [
    (BF, (28, 4), 128, 128, [(256, 512)], 128, False),
    (BF, (28, 4), 128, 128, [(1, 1), (1, 128), (1, 129), (1, 300), (0, 77), (0, 0)], 128, False),
    (BF, (6, 2), 128, 64, [(70, 130), (3, 64), (129, 129), (65, 1000)], 64, True),
    (BF, (14, 2), 64, 16, [(33, 100), (1, 16), (17, 17), (5, 37)], 64, False),
    (F32, (2, 1), 64, 16, [(40, 43), (16, 32), (0, 5), (7, 7)], 32, True),
    (F32, (8, 2), 128, 128, [(130, 257), (128, 128)], 48, False),
    (F32, (3, 3), 128, 32, [(1, 1)], 16, False),
    (BF, (4, 4), 64, 128, [(200, 333)], 0, False),
    (BF, (4, 2), 128, 32, [(64, 64), (95, 700)], 112, False),
]
IDS = [f"{'bf16' if c[0] == BF else 'f32'}-h{c[1][0]}-{c[1][1]}-d{c[2]}-p{c[3]}-rot{c[5]}{'i' if c[6] else ''}" for c in CASES]


def _setup(case, seed=3):
    dt, (Hq, Hkv), D, P, spans, rot, inter = case
    b = ru.Batch(spans, P, seed)
    gen = torch.Generator().manual_seed(seed)
    packed = torch.randn((b.n_rows, (Hq + 2 * Hkv) * D), generator=gen).to(dt)   # the rows are views of one tensor
    cos, sin = ru.tables(b.max_len + 2, rot, seed) if rot else (None, None)
    rope = api.Rope(cos.cuda(), sin.cuda(), inter) if rot else None
    return b, packed, cos, sin, rope


def _split(packed, Hq, Hkv, D):
    q, k, v = packed.split([Hq * D, Hkv * D, Hkv * D], 1)
    return q.unflatten(1, (Hq, D)), k.unflatten(1, (Hkv, D)), v.unflatten(1, (Hkv, D))


def _turned(x, pos, cos, sin, inter, back=False):
    """float64 rotation of a row and the sizes of its terms"""
    return ru.rotate(x, cos[pos], sin[pos], inter, back) if cos is not None else (x.double(), x.double().abs())


def _bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == BF else torch.int32)


def _same(got, want, name):
    assert torch.equal(_bits(got.cpu()), _bits(want)), f"{name} differs in {int((_bits(got.cpu()) != _bits(want)).sum())} places"


def _check_queries(b, got, q, cos, sin, inter, back=False, before=None):
    """two rounded products and a rounded sum in fp32 (3 half steps of the terms), then one rounding to the type (below its normal
    values: half a step of 2^-133 or three of 2^-149)"""
    want, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    if before is not None:
        want.copy_(before.double())
    for r, _, pos in b.each_row():
        want[r], size = _turned(q[r], pos, cos, sin, inter, back)
        tol[r] = ru.HALF[q.dtype] * want[r].abs() + 3 * 2.0 ** -24 * size + (2.0 ** -134 if q.dtype == BF else 0.0) + 3 * 2.0 ** -150
    ru.check("q", got.cpu().double().numpy(), want.numpy(), tol.numpy())


def _mean(keys):
    """fp32 mean of [P][...], in the order of the tokens"""
    total = torch.zeros(keys.shape[1:], dtype=torch.float32)
    for row in keys.float():
        total = total + row
    return total * (1.0 / keys.shape[0])


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_append(case):
    dt, (Hq, Hkv), D, P, spans, rot, inter = case
    b, packed, cos, sin, rope = _setup(case)
    q, k, v = _split(packed, Hq, Hkv, D)
    gq, gk, gv = _split(packed.cuda(), Hq, Hkv, D)
    gen = torch.Generator().manual_seed(9)
    pools = [torch.randn((b.n_phys, Hkv, P, D), generator=gen).to(dt) for _ in range(2)]
    gpools = [x.cuda() for x in pools]
    kbar = torch.full((len(spans), b.cols, Hkv, D), 7.0)
    gbar, out = kbar.cuda(), torch.full((b.n_rows, Hq, D), 5.0, dtype=dt, device="cuda")
    at = b.device()
    desc = api.make_rows_desc(gq, gpools[0], at["page_tables"], b.max_len, max_rows=b.max_rows)
    got = api.kv_append_rope(desc, gk, gv, at.pop("page_tables"), *gpools, q=gq, q_out=out, rope=rope, kbar_cache=gbar, **at)
    torch.cuda.synchronize()
    assert got is out
    _check_queries(b, out, q, cos, sin, inter, before=torch.full(q.shape, 5.0))
    for r, s, pos in b.each_row():
        page = b.tables[s, pos // P]
        y, _ = _turned(k[r], pos, cos, sin, inter)
        pools[0][page, :, pos % P] = y.float().to(dt)   # rounded to float, then to the type
        pools[1][page, :, pos % P] = v[r]
    for r, s, pos in b.each_row():
        if pos % P == P - 1:
            kbar[s, pos // P] = _mean(pools[0][b.tables[s, pos // P]].transpose(0, 1))
    _same(gpools[0], pools[0], "K pool")
    _same(gpools[1], pools[1], "V pool")
    _same(gbar, kbar, "means")
    assert torch.equal(packed, torch.cat([x.flatten(1) for x in (gq, gk, gv)], 1).cpu()), "an input was written"
    # in place, without means and for keys and values alone: the same rows
    for x, y in zip(gpools, pools):
        x.copy_(torch.zeros_like(y))
    both = gq.clone()
    seqs = b.device()
    api.kv_append_rope(desc, gk, gv, seqs["page_tables"], *gpools, q=both, q_out=both, rope=rope, seq_lens=seqs["seq_lens"], row_starts=seqs["row_starts"])
    torch.cuda.synchronize()
    assert torch.equal(both[:b.rows], out[:b.rows]) and torch.equal(both[b.rows:], gq[b.rows:])
    held = [x.clone() for x in gpools]
    assert api.kv_append_rope(desc, gk, gv, seqs["page_tables"], *gpools, rope=rope, seq_lens=seqs["seq_lens"], row_starts=seqs["row_starts"]) is None
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(held, gpools))


@pytest.mark.parametrize("grad", [F32, BF], ids=["f32-pools", "bf16-pools"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_append_backward(case, grad):
    dt, (Hq, Hkv), D, P, spans, rot, inter = case
    b, packed, cos, sin, rope = _setup(case)
    dq, _, _ = _split(packed, Hq, Hkv, D)
    gen = torch.Generator().manual_seed(10)
    pools = [torch.randn((b.n_phys, Hkv, P, D), generator=gen).to(grad) for _ in range(2)]
    gpools = [x.cuda() for x in pools]
    gdq = _split(packed.cuda(), Hq, Hkv, D)[0]
    grads = torch.full_like(packed, 5.0, device="cuda")
    oq, ok, ov = _split(grads, Hq, Hkv, D)
    at = b.device()
    table = at.pop("page_tables")
    desc = api.make_rows_desc(gdq, gpools[0], table, b.max_len, max_rows=b.max_rows)
    api.kv_append_rope_bwd(desc, *gpools, table, d_q=gdq, rope=rope, d_q_out=oq, d_k=ok, d_v=ov, **at)
    torch.cuda.synchronize()
    _check_queries(b, oq, dq, cos, sin, inter, back=True, before=torch.full(dq.shape, 5.0))
    want = [torch.full((b.n_rows, Hkv, D), 5.0, dtype=torch.float64) for _ in range(2)]
    tol = [torch.zeros_like(x) for x in want]
    for r, s, pos in b.each_row():
        gk, gv = (x[b.tables[s, pos // P], :, pos % P] for x in pools)
        want[0][r], size = _turned(gk, pos, cos, sin, inter, back=True)
        want[1][r] = gv.double()
        tol[0][r] = ru.HALF[dt] * want[0][r].abs() + 3 * 2.0 ** -24 * size
        tol[1][r] = ru.HALF[dt] * want[1][r].abs()
    ru.check("d_k", ok.cpu().double().numpy(), want[0].numpy(), tol[0].numpy())
    ru.check("d_v", ov.cpu().double().numpy(), want[1].numpy(), tol[1].numpy())
    assert all(torch.equal(x.cpu(), y) for x, y in zip(gpools, pools)), "a gradient pool was written"
    # new tensors, in place for the queries, and without them
    same = gdq.clone()
    a1, a2, a3 = api.kv_append_rope_bwd(desc, *gpools, table, d_q=same, rope=rope, d_q_out=same, **at)
    n1, n2, n3 = api.kv_append_rope_bwd(desc, *gpools, table, rope=rope, **at)
    torch.cuda.synchronize()
    assert a1 is same and torch.equal(a1[:b.rows], oq[:b.rows]) and n1 is None
    live = [r for r, _, _ in b.each_row()]
    for x in (a2, n2):
        assert torch.equal(x[live], ok[live])
    for x in (a3, n3):
        assert torch.equal(x[live], ov[live])
    assert not a2[b.rows:].any() and not a3[b.rows:].any()


@pytest.mark.parametrize("inter", [False, True])
def test_backward_against_differences(inter):
    """L = <q_out, a> + <K rows, b> + <V rows, c> changes along a direction by the inner product of the direction and the
    gradients: L is linear, so a difference over steps of 1 is exact but for roundings."""
    spans, P, Hq, Hkv, D = [(37, 60), (5, 5)], 16, 4, 2, 64
    b = ru.Batch(spans, P, 4, behind=0)
    gen = torch.Generator().manual_seed(5)
    rope = api.Rope(*(x.cuda() for x in ru.tables(b.max_len, D, 6)), inter)
    at = b.device()
    table = at.pop("page_tables")

    def normal(*shape):
        return torch.randn(shape, generator=gen).cuda()

    x, step = [normal(b.n_rows, h, D) for h in (Hq, Hkv, Hkv)], [normal(b.n_rows, h, D) for h in (Hq, Hkv, Hkv)]
    a, gk, gv = normal(b.n_rows, Hq, D), normal(b.n_phys, Hkv, P, D), normal(b.n_phys, Hkv, P, D)

    def loss(q, k, v):
        pools = [torch.zeros((b.n_phys, Hkv, P, D), device="cuda") for _ in range(2)]
        desc = api.make_rows_desc(q, pools[0], table, b.max_len, max_rows=b.max_rows)
        y = api.kv_append_rope(desc, k, v, table, *pools, q=q, rope=rope, **at)
        return sum((u.double() * w.double()).sum() for u, w in ((y, a), (pools[0], gk), (pools[1], gv)))

    lost = [loss(*(u + s * w for u, w in zip(x, step))) for s in (1.0, -1.0)]
    desc = api.make_rows_desc(a, gk, table, b.max_len, max_rows=b.max_rows)
    grads = api.kv_append_rope_bwd(desc, gk, gv, table, d_q=a, rope=rope, **at)
    along = sum((g.double() * w.double()).sum() for g, w in zip(grads, step))
    # every one of the terms is rounded a few times to 2^-24 of its size
    size = sum((g.double() * w.double()).abs().sum() for g, w in zip(grads, step)) + \
        sum((u.double().abs() + w.double().abs()).sum() for u, w in zip(x, step)) * 8
    assert abs((lost[0] - lost[1]) / 2 - along) <= 8 * 2.0 ** -24 * size


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_quantised_append_and_read(case):
    dt, (Hq, Hkv), D, P, spans, rot, inter = case
    b, packed, cos, sin, rope = _setup(case)
    packed[:, 3] *= 2.0 ** 40      # blocks of unlike sizes, and tiny, zero and huge ones
    packed[0] *= 2.0 ** -126
    packed[b.n_rows // 2, Hq * D:Hq * D + 32] = 0.0
    packed[b.n_rows - 3 if b.n_rows > 3 else 0, -40:] *= 2.0 ** 120
    q, k, v = _split(packed, Hq, Hkv, D)
    gq, gk, gv = _split(packed.cuda(), Hq, Hkv, D)
    pools = [ru.random_pool(b, Hkv, D, seed) for seed in (1, 2)]
    gpools = [torch.tensor(x, device="cuda") for x in pools]
    kbar = torch.full((len(spans), b.cols, Hkv, D), 7.0)
    gbar, out = kbar.cuda(), torch.full((b.n_rows, Hq, D), 5.0, dtype=dt, device="cuda")
    at = b.device()
    table = at.pop("page_tables")
    desc = api.make_rows_desc(gq, gpools[0], table, b.max_len, max_rows=b.max_rows)
    assert desc.page_size == P
    api.kvq_append_rope(desc, gk, gv, table, *gpools, q=gq, q_out=out, rope=rope, kbar_cache=gbar, **at)
    held = [torch.full((b.n_rows, Hkv, D), 5.0, dtype=dt, device="cuda") for _ in range(2)]
    api.kvq_read(desc, *gpools, table, k_out=held[0], v_out=held[1], **at)
    torch.cuda.synchronize()
    _check_queries(b, out, q, cos, sin, inter, before=torch.full(q.shape, 5.0))
    want = [np.full((b.n_rows, Hkv, D), 5.0) for _ in range(2)]
    before = [x.copy() for x in pools]
    for r, s, pos in b.each_row():
        page = b.tables[s, pos // P]
        y, _ = _turned(k[r], pos, cos, sin, inter)
        for pool, x, w in zip(pools, (y, v[r].double()), want):
            code, byte = ru.quantise(x.numpy())
            w[r] = ru.values(code, byte)
            codes, bytes_ = ru.unpack(pool[page], P, D)
            codes[:, pos % P], bytes_[:, pos % P] = code, byte
            pool[page] = ru.pack(codes, bytes_)
    for x, w, name in zip(held, want, ("K", "V")):
        assert np.array_equal(x.cpu().double().numpy(), w), f"{name}: {np.sum(x.cpu().double().numpy() != w)} values differ"
    for x, w, old, name in zip(gpools, pools, before, ("K", "V")):   # (a zero's sign may differ: compared as values where written, as bytes elsewhere)
        x = x.cpu().numpy()
        assert np.array_equal(ru.values(*ru.unpack(x, P, D)), ru.values(*ru.unpack(w, P, D)), equal_nan=True), f"{name} pool"
        same = old == w
        assert np.array_equal(ru.unpack(x, P, D)[1], ru.unpack(w, P, D)[1]) and (x[same] == w[same]).mean() > 0.99, f"{name} pool"
    for r, s, pos in b.each_row():
        if pos % P == P - 1:
            keys = ru.values(*ru.unpack(pools[0][b.tables[s, pos // P]], P, D))
            kbar[s, pos // P] = _mean(torch.tensor(keys, dtype=torch.float32).transpose(0, 1))
    assert torch.equal(gbar.cpu().isnan(), kbar.isnan()) and torch.equal(gbar.cpu().nan_to_num(), kbar.nan_to_num())


@pytest.mark.parametrize("D", [64, 128])
def test_values_that_are_not_finite_make_their_block_nan(D):
    b = ru.Batch([(3, 3)], 16, behind=0)
    x = torch.randn((3, 1, D), generator=torch.Generator().manual_seed(1))
    x[0, 0, 5], x[1, 0, 40], x[2, 0, D - 1] = float("nan"), float("inf"), -float("inf")
    g = x.cuda()
    pools = [api.kvq_pool(b.n_phys, 1, 16, D) for _ in range(2)]
    at = b.device()
    table = at.pop("page_tables")
    desc = api.make_rows_desc(g, pools[0], table, 3)
    api.kvq_append_rope(desc, g, g, table, *pools, **at)
    k, v = api.kvq_read(desc, *pools, table, **at)
    want = np.stack([ru.values(*ru.quantise(r.numpy().astype(np.float64))) for r in x])
    assert np.isnan(want).sum() == 96
    for y in (k, v):
        assert np.array_equal(y.cpu().double().numpy(), want, equal_nan=True)


def test_largest_and_smallest_values():
    """The scale's ends: past 6 2^125 values stay at it, below 2^-127 they vanish."""
    x = torch.zeros((4, 1, 64))
    x[0, 0, :4] = torch.tensor([3.4e38, -3.0e38, 2.0 ** 125, 2.0 ** 123])
    x[1, 0, :4] = torch.tensor([2.0 ** -126, 2.0 ** -127, 2.0 ** -128, -2.0 ** -149])
    x[2, 0, :3] = torch.tensor([7.0, 6.9, -5.0])
    x[3, 0, :3] = torch.tensor([7.0 + 2.0 ** -20, 6.9, -5.0])
    b = ru.Batch([(4, 20)], 16, behind=0)
    g = x.cuda()
    pools = [api.kvq_pool(b.n_phys, 1, 16, 64) for _ in range(2)]
    at = b.device()
    table = at.pop("page_tables")
    desc = api.make_rows_desc(g, pools[0], table, 20)
    api.kvq_append_rope(desc, g, g, table, *pools, **at)
    k, _ = api.kvq_read(desc, *pools, table, **at)
    want = np.stack([ru.values(*ru.quantise(r.numpy().astype(np.float64))) for r in x])
    assert want[0, 0, 0] == 6 * 2.0 ** 125 and want[2, 0, 0] == 6 and want[3, 0, 0] == 8
    assert np.array_equal(k.cpu().double().numpy(), want)


@pytest.mark.parametrize("kvq", [False, True])
def test_rows_that_do_not_exist_and_pages_out_of_range(kvq):
    """More rows than tokens (the surplus in front is left alone), a page id outside the pool, lengths beyond the bound, rows beyond
    max_rows: nothing outside the sequences' pages and rows is touched."""
    P, D, dt = 16, 64, F32
    b = ru.Batch([(10, 6), (20, 40), (4, 300)], P, 2)
    b.tables[1, 2] = b.n_phys      # the second sequence's last page
    at = b.device()
    table = at.pop("page_tables")
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((b.n_rows, h, D), generator=gen).cuda() for h in (2, 1, 1))
    make = (lambda: torch.full((b.n_phys, 1, kvq_tile), 17, dtype=torch.uint8, device="cuda")) if kvq else \
        (lambda: torch.full((b.n_phys, 1, P, D), 17.0, device="cuda"))
    kvq_tile = api.kvq_tile_bytes(P, D)
    pools = [make(), make()]
    desc = api.make_rows_desc(q, pools[0], table, 48, max_rows=18)   # max_len 48 < 300, max_rows 18 < 20
    out = torch.full_like(q, 5.0)
    append = api.kvq_append_rope if kvq else api.kv_append_rope
    append(desc, k, v, table, *pools, q=q, q_out=out, **at)
    torch.cuda.synchronize()
    written = {}
    for s, (n, t) in enumerate(b.spans):
        t = min(t, 48)
        for i in range(min(n, 18)):
            pos = t - n + i
            if pos >= 0:
                written[b.starts[s] + i] = (s, pos)
    want = torch.full_like(q, 5.0)
    for r in written:
        want[r] = q[r]
    assert torch.equal(out, want)
    ref = make()
    for r, (s, pos) in written.items():
        page = b.tables[s, pos // P]
        if page < b.n_phys and not kvq:
            ref[page, :, pos % P] = k[r]
    if not kvq:
        assert torch.equal(pools[0], ref)
        dk, dv = torch.full_like(k, 5.0), torch.full_like(v, 5.0)
        desc = api.make_rows_desc(q, pools[0], table, 48, max_rows=18)
        api.kv_append_rope_bwd(desc, *pools, table, d_k=dk, d_v=dv, **at)
        torch.cuda.synchronize()
        want = torch.full_like(k, 5.0)
        for r, (s, pos) in written.items():
            want[r] = k[r] if b.tables[s, pos // P] < b.n_phys else 0.0
        assert torch.equal(dk, want)
        return
    touched = {int(b.tables[s, pos // P]) for s, pos in written.values()}
    for page in range(b.n_phys):
        if page not in touched:
            assert (pools[0][page] == 17).all() and (pools[1][page] == 17).all()
    kh, _ = api.kvq_read(desc, *pools, table, k_out=torch.full_like(k, 5.0), v_out=torch.full_like(v, 5.0), **at)
    torch.cuda.synchronize()
    for r in range(b.n_rows):
        if r not in written:
            assert (kh[r] == 5.0).all()
        else:
            s, pos = written[r]
            w = ru.values(*ru.quantise(k[r].cpu().double().numpy())) if b.tables[s, pos // P] < b.n_phys else np.zeros((1, D))
            assert np.array_equal(kh[r].cpu().double().numpy(), w)


def test_without_arrays_of_starts_and_lengths():
    """row_starts None: equal rows each; seq_lens None: max_len each; a 1-D table: one sequence."""
    P, D = 16, 64
    b = ru.Batch([(3, 40), (3, 40)], P, 7, behind=0)
    gen = torch.Generator().manual_seed(2)
    k, v = (torch.randn((6, 1, D), generator=gen).cuda() for _ in range(2))
    at = b.device()
    table = at.pop("page_tables")
    pools = [torch.zeros((b.n_phys, 1, P, D), device="cuda") for _ in range(4)]
    desc = api.make_rows_desc(k, pools[0], table, 40, max_rows=3)
    api.kv_append_rope(desc, k, v, table, pools[0], pools[1], **at)
    api.kv_append_rope(desc, k, v, table, pools[2], pools[3])
    torch.cuda.synchronize()
    assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3]) and pools[0].any()
    one = api.make_rows_desc(k[:3], pools[0], table[0], 40)
    api.kv_append_rope(one, k[:3] + 1, v[:3], table[0], pools[0], pools[1])
    torch.cuda.synchronize()
    assert torch.equal(pools[0][b.tables[0, 2], 0, 5:8], k[:3, 0] + 1) and torch.equal(pools[0][b.tables[1, 2]], pools[2][b.tables[1, 2]])
