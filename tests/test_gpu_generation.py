"""GPU tests of generation's steps: pages forked, copied and compacted, beam search's selection, and all of them with the attention together."""
import math

import numpy as np
import pytest
import torch

from paper_2602_02108_amd import api

import gen_util as gu

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _i(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _state(spans, P, cols, n_phys, shared, seed):
    """Tables of sequences of `spans` tokens of which the i-th shares its first shared[i] pages with the one before it; and their counts."""
    rng = np.random.default_rng(seed)
    order = [int(x) for x in rng.permutation(n_phys)]
    tables, refs, at = [], [0] * n_phys, 0
    for i, t in enumerate(spans):
        n = -(-t // P)
        row = tables[-1][:shared[i]] if shared[i] else []
        row += order[at:at + n - len(row)]
        at += n - (shared[i] if shared[i] else 0)
        for x in row:
            refs[x] += 1
        tables.append(row + [-1] * (cols - n))
    assert at <= n_phys
    return tables, refs


FORKS = [
    # spans, pages shared with the one before, P, cols, n_phys, parents, grow, out_cols
    ([40, 40, 40], [0, 2, 2], 16, 5, 12, [1, 1, 2], [1, 1, 1], 5),
    ([33, 32, 1, 0, 48], [0, 0, 0, 0, 0], 16, 4, 20, [0, 0, 0, 4, 1, 3, 3], [16, 15, 0, 1, 0, 17, 1], 4),
    ([500, 500, 77], [0, 30, 0], 16, 40, 80, [0, 1, 1, -1, -2, -2, 2, 9, -7], [1, 1, 100, 50, 33, 0, 1, 1, 1], 48),
    ([130], [0], 128, 3, 6, [0] * 4, [1] * 4, 3),
    ([130], [0], 128, 3, 4, [0] * 6, [1] * 6, 3),                      # pages run out at copies
    ([20, 20], [0, 0], 16, 8, 6, [0, 1, 0, -2], [60, 60, 5, 500], 8),  # and at growth
    ([300, 17], [0, 0], 16, 20, 30, [0, 1, 0], [5, 5, 5], 10),         # rows of the new tables are shorter: lengths are cut
    ([64, 64, 64, 64], [0, 4, 4, 4], 16, 6, 9, [3, 3, 3, 3], None, 6), # nothing partly filled, one page for all
    ([5], [0], 1, 40, 50, [0, 0], [3, 30], 40),                        # pages of one token
]


def _fork_case(case, in_place, held=0):
    spans, shared, P, cols, n_phys, parents, grow, out_cols = case
    tables, refs = _state(spans, P, cols, n_phys, shared, 3)
    refs += [1] * held      # pages that somebody else holds
    want = gu.fork(tables, spans, parents, grow, refs, P, out_cols)
    n_out = len(parents)
    t, ln, r = _i(tables), _i(spans), _i(refs)
    out = torch.full((n_out, out_cols + 3), 77, dtype=torch.int32, device="cuda")[:, :out_cols]
    got = api.page_fork(t, ln, _i(parents), r, P, grow=None if grow is None else _i(grow), tables_out=out, refs_out=None if in_place else torch.full_like(r, 55),
                        lens_out=ln if in_place and n_out == len(spans) else None)
    torch.cuda.synchronize()
    assert got.tables.tolist() == want[0] and got.lens.tolist() == want[1]
    assert got.refs.tolist() == want[2] and got.copies.tolist() == want[3] and got.status.tolist() == want[4]
    assert t.tolist() == tables and (in_place or r.tolist() == refs)
    base = out._base if out._base is not None else out
    assert (base[:, out_cols:] == 77).all()
    return got, want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("held", [0, 9000])   # (few pages: one workgroup; many: two launches)
@pytest.mark.parametrize("case", FORKS, ids=[str(i) for i in range(len(FORKS))])
def test_fork(case, held, in_place):
    _fork_case(case, in_place, held)


@pytest.mark.parametrize("held", [0, 9000])
def test_fork_of_entries_out_of_range_and_of_lengths_out_of_range(held):
    P, n_phys = 16, 30
    tables, refs = _state([40, 40, 35], P, 4, n_phys, [0, 0, 0], 5)
    refs += [1] * held
    for x in (tables[0][1], tables[1][2], tables[2][2]):
        refs[x] = 0
    tables[0][1], tables[1][2], tables[2][2] = 30 + held, -9, 1 << 30
    parents, grow = [0, 0, 1, 1, 2, 2], [1, 9, 1, 30, -5, 40]
    want = gu.fork(tables, [40, 900, -3], parents, grow, refs, P, 4)
    got = api.page_fork(_i(tables), _i([40, 900, -3]), _i(parents), _i(refs), P, grow=_i(grow))
    torch.cuda.synchronize()
    assert got.tables.tolist() == want[0] and got.lens.tolist() == want[1] and got.refs.tolist() == want[2]
    assert got.copies.tolist() == want[3] and got.status.tolist() == want[4]


@pytest.mark.parametrize("n_seqs,n_out,P,n_phys", [(1500, 2000, 16, 60000), (4096, 4096, 128, 9000), (3, 700, 32, 40000), (1024, 1024, 16, 8192), (1025, 3, 16, 8192)])
def test_fork_of_many(n_seqs, n_out, P, n_phys):
    """More sequences than a workgroup has threads, more pages than it counts at a time, rows of several pieces; then further steps in place."""
    rng = np.random.default_rng(6)
    cols = 1300 if n_seqs < 10 else 20
    spans = [int(x) for x in rng.integers(0, min(cols * P, n_phys * P // n_seqs // 3) + 1, n_seqs)]
    tables, refs = _state(spans, P, cols, n_phys, [0] * n_seqs, 7)
    t, ln, r = _i(tables), _i(spans), _i(refs)
    for step in range(3):
        parents = [int(x) for x in rng.integers(-2, len(spans), n_out)]
        grow = [int(x) for x in rng.integers(0, 3 * P, n_out)]
        want = gu.fork(tables, spans, parents, grow, refs, P, cols)
        got = api.page_fork(t, ln, _i(parents), r, P, grow=_i(grow))
        torch.cuda.synchronize()
        tables, spans, refs = want[0], want[1], want[2]
        assert got.tables.tolist() == tables and got.lens.tolist() == spans and got.refs.tolist() == refs
        assert got.copies.tolist() == want[3] and got.status.tolist() == want[4]
        t, ln = got.tables, got.lens


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("n_phys,free", [(32768, 90), (32769, 90), (150001, 90), (150001, 2), (150001, 0), (70000, 9000)])
def test_fork_of_large_pools(n_phys, free, in_place):
    """The free pages are the last ones, or fewer than needed, or none; two of the counts are negative, which frees nothing."""
    P, cols, n = 16, 8, 50
    spans = [5 + i for i in range(n)]
    tables = [[7 * i + l if l < -(-t // P) else -1 for l in range(cols)] for i, t in enumerate(spans)]
    refs = [1] * (n_phys - free) + [0] * free
    refs[n_phys // 2] = refs[n_phys - free - 1] = -1
    parents, grow = [(3 * b) % n for b in range(n)], [1] * n
    want = gu.fork(tables, spans, parents, grow, refs, P, cols)
    r = _i(refs)
    out = None if in_place else torch.full((n_phys,), 77, dtype=torch.int32, device="cuda")
    got = api.page_fork(_i(tables), _i(spans), _i(parents), r, P, grow=_i(grow), refs_out=out)
    torch.cuda.synchronize()
    assert got.tables.tolist() == want[0] and got.lens.tolist() == want[1] and got.refs.tolist() == want[2]
    assert got.copies.tolist() == want[3] and got.status.tolist() == want[4]
    assert (got.refs is r) if in_place else r.tolist() == refs


@pytest.mark.parametrize("more", [0, 9000])
def test_counts_of_pages_held_besides(more):
    """A page that somebody outside holds: the first child copies it too, and it does not become free."""
    P = 16
    tables, refs = _state([20, 18], P, 3, 8, [0, 0], 9)
    refs += [1] * more
    held = tables[0][1]
    refs[held] += 1
    want = gu.fork(tables, [20, 18], [0, -1], [1, 0], refs, P, 3)
    got = api.page_fork(_i(tables), _i([20, 18]), _i([0, -1]), _i(refs), P, grow=_i([1, 0]))
    torch.cuda.synchronize()
    assert got.copies.tolist() == want[3] and got.copies.tolist()[0][0] == held and got.refs.tolist() == want[2]
    assert got.refs[held] == 1 and sum(x > 0 for x in got.refs.tolist()) == 3 + more


@pytest.mark.parametrize("kind", ["bf16", "f32", "tokens_first", "kvq", "gradient"])
def test_copy(kind):
    """Every listed page, in every pool, up to its tokens; all other bytes as they were."""
    gen = torch.Generator().manual_seed(4)
    n, H, P, D = 23, 3, 16, 64

    def pool():
        if kind == "kvq":
            return torch.randint(0, 256, (n, H, api.kvq_tile_bytes(P, D)), generator=gen, dtype=torch.uint8)
        x = torch.randn((n, H, P, D), generator=gen).to(BF if kind != "f32" and kind != "gradient" else F32)
        return x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if kind == "tokens_first" else x
    pools = [pool() for _ in range(70 if kind == "bf16" else 5)]       # (more than a launch takes)
    copies = [[0, 22, 16], [3, 4, 1], [-1, -1, 0], [5, 6, 15], [7, 23, 4], [-3, 8, 4], [9, 10, 0], [11, 12, 99], [13, 13, 5], [1, 14, 16]]
    got = [x.cuda() for x in pools]
    if kind == "tokens_first":
        got = [x.cuda().permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for x in pools]
    api.page_copy(got, _i(copies))
    torch.cuda.synchronize()
    for x, y in zip(pools, got):
        for a, b, t in copies:
            if 0 <= a < n and 0 <= b < n and t > 0 and a != b:
                if kind == "kvq":
                    x[b] = x[a]
                else:
                    x[b, :, :t] = x[a, :, :t]
        assert torch.equal(x, y.cpu())


@pytest.mark.parametrize("limit", [0, 1, 2, 9, -4])
def test_copy_of_a_count_on_the_device(limit):
    x = torch.randn((12, 2, 32, 128), generator=torch.Generator().manual_seed(4))
    copies = [[0, 6, 32], [1, 7, 3], [2, 8, 5]]
    got = x.cuda()
    api.page_copy((got,), _i(copies), count=_i([limit]))
    torch.cuda.synchronize()
    for a, b, t in copies[:max(0, limit)]:
        x[b, :, :t] = x[a, :, :t]
    assert torch.equal(x, got.cpu())


@pytest.mark.parametrize("n_phys,spans,P,cols", [(1, [0], 16, 1), (2, [5], 16, 2), (40, [100, 33, 0, 16], 16, 9), (9000, [3000, 70000, 1], 16, 5000),
                                                 (20000, [150000], 16, 10000), (8192, [40000, 39999, 1], 16, 3000), (8191, [90000], 16, 6000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(n_phys, spans, P, cols, in_place):
    tables, refs = _state(spans, P, cols, n_phys, [0] * len(spans), 11)
    if n_phys == 40:
        refs[[i for i, r in enumerate(refs) if r][3]] += 4       # shared and held pages keep their counts
    want = gu.compact(tables, spans, refs, P)
    t, r = _i(tables), _i(refs)
    got = api.page_compact(t, _i(spans), r, P, tables_out=None if in_place else torch.full_like(t, 9), refs_out=None if in_place else torch.full_like(r, 9))
    pools = [torch.randn((n_phys, 1, P, 64), generator=torch.Generator().manual_seed(s)) for s in (1, 2)]
    dev = [x.cuda() for x in pools]
    api.page_copy(dev, got.moves, count=got.status[1:])
    torch.cuda.synchronize()
    assert got.tables.tolist() == want[0] and got.refs.tolist() == want[1] and got.page_map.tolist() == want[3] and got.status.tolist() == want[4]
    assert got.moves[:want[4][1]].tolist() == want[2]
    for x, y in zip(pools, dev):
        for a, b, _ in want[2]:
            x[b] = x[a]
        assert torch.equal(x, y.cpu())


def test_compact_of_nothing_and_of_everything():
    for refs in ([0] * 50, [1] * 50, [0] * 25 + [2] * 25, [3] * 25 + [0] * 25, [0] * 10000, [1] * 10000, [0] * 5000 + [2] * 5000):
        want = gu.compact([[-1] * 3], [0], refs, 16)
        got = api.page_compact(_i([[-1] * 3]), _i([0]), _i(refs), 16)
        torch.cuda.synchronize()
        assert got.refs.tolist() == want[1] and got.page_map.tolist() == want[3] and got.status.tolist() == want[4]


# ---- beam search's selection ----

def _logits(shape, dt, seed, scale=4.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dt)


def _beam(x, scores, n_out, done=None, pad=0, **kw):
    p, t, s = api.beam_topk(x.cuda() if not x.is_cuda else x, scores.cuda(), n_out, done=None if done is None else done.cuda(), pad_token=pad, **kw)
    torch.cuda.synchronize()
    return p.cpu().numpy(), t.cpu().numpy(), s.cpu().double().numpy()


def _verify_beam(x, scores, n_out, got, done=None, pad=0):
    want = gu.beam(x.double().numpy(), scores.numpy(), n_out, None if done is None else done.numpy(), pad)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    fine = np.isfinite(want[2])
    assert np.array_equal(fine, np.isfinite(got[2])) and (got[2][~fine] == -np.inf).all()
    # the log-sum: exponentials of one ulp (2^-23) and factors, in sums of at most 64 in fp32 (2^-18) of each thread, 64 bits beyond; one rounding to float
    tol = 2.0 ** -18 + 2.0 ** -24 * np.abs(want[2][fine])
    assert (np.abs(got[2][fine] - want[2][fine]) <= tol).all()


BEAMS = [
    # groups, beams, vocab, n_out, type
    (1, 1, 1, 1, F32), (1, 1, 7, 7, F32), (1, 4, 32000, 8, F32), (2, 3, 50, 64, BF), (5, 8, 1000, 16, BF), (3, 4, 100003, 8, BF), (2, 64, 777, 64, F32),
    (1, 2, 300001, 5, F32), (40, 1, 4097, 1, BF), (1, 64, 20001, 64, BF), (3, 5, 8192, 2, BF), (2, 1, 8193, 33, BF), (1, 3, 2, 64, F32), (600, 4, 260, 4, F32),
]


@pytest.mark.parametrize("case", BEAMS, ids=["-".join(str(y) for y in c[:4]) for c in BEAMS])
def test_beam(case):
    groups, W, V, n_out, dt = case
    x = _logits((groups, W, V), dt, 21)
    scores = -10.0 * torch.rand((groups, W), generator=torch.Generator().manual_seed(22))
    _verify_beam(x, scores, n_out, _beam(x, scores, n_out))
    done = (torch.rand((groups, W), generator=torch.Generator().manual_seed(23)) < 0.4).to(torch.int32)
    scores[:, W // 2] = -math.inf
    _verify_beam(x, scores, n_out, _beam(x, scores, n_out, done, 3), done, 3)


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("V", [3, 60, 240, 256, 500])
def test_beam_of_short_rows_and_many_beams(V, dt):
    """Rows that fill fewer lanes than candidates are asked for: a first bound that nothing sets, and more cells than its list holds."""
    for W in (5, 17, 64):
        x = _logits((3, W, V), dt, 25)
        scores = -10.0 * torch.rand((3, W), generator=torch.Generator().manual_seed(26))
        done = (torch.rand((3, W), generator=torch.Generator().manual_seed(27)) < 0.3).to(torch.int32)
        for n_out in (1, 33, 64):
            _verify_beam(x, scores, n_out, _beam(x, scores, n_out))
            _verify_beam(x, scores, n_out, _beam(x, scores, n_out, done, 2), done, 2)


def test_beam_of_equal_logits_takes_the_lowest():
    for V, dt in ((9000, BF), (5000, F32), (300, BF)):
        for W in (1, 3):
            x, s = torch.zeros((2, W, V), dtype=dt), torch.zeros((2, W))
            for n_out in (1, 16, 64):
                _verify_beam(x, s, n_out, _beam(x, s, n_out))
    x = _logits((1, 1, 9000), BF, 3).round()            # few different values, equal hypotheses
    x, s = x.expand(2, 4, 9000).contiguous(), torch.zeros((2, 4))
    _verify_beam(x, s, 33, _beam(x, s, 33))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [300, 5000, 131072])
@pytest.mark.parametrize("mask", [-1e4, "least"])
def test_beam_of_logits_masked_with_a_finite_value(dt, V, mask):
    """Fewer live tokens than candidates: the first masked ones, by score and place, fill up."""
    gen = torch.Generator().manual_seed(V)
    least = torch.finfo(dt).min if mask == "least" else mask
    x = torch.full((4, 5, V), least).to(dt)
    for g in range(4):
        for w in range(5):
            live = torch.randperm(V, generator=gen)[:int(torch.randint(1, 4, (1,), generator=gen))]
            x[g, w, live] = (torch.randn(len(live), generator=gen) * 4).to(dt)
    s = -20 * torch.rand((4, 5), generator=gen)
    done = torch.zeros((4, 5), dtype=torch.int32)
    done[1, 2] = done[3, 0] = done[3, 1] = 1
    for n_out in (1, 16, 64):
        _verify_beam(x, s, n_out, _beam(x, s, n_out, done, 1), done, 1)


def test_beam_of_few_cells_with_many_values_above_equal_ones():
    """More values above the common one than are ranked at a time, all in a few threads' places."""
    V = 400000
    v = torch.arange(V)
    for many in (1, 7):
        x = torch.where((v // 4) % 256 == 0, 1 + (v * many % 4001) / 4096.0, torch.tensor(0.25)).expand(1, 1, V).contiguous()
        for n_out in (1, 50, 64):
            _verify_beam(x, torch.zeros((1, 1)), n_out, _beam(x, torch.zeros((1, 1)), n_out))


@pytest.mark.parametrize("n_out", [1, 2, 3])
def test_beam_that_has_ended_stands_behind_equal_ones(n_out):
    """Scores so large that log-sums vanish in them: every candidate of a group is equal, and the lowest places win over those of beams that have ended."""
    scores, x = torch.full((2, 3), -1e20), torch.zeros((2, 3, 5000))
    done = torch.tensor([[0, 1, 1], [1, 0, 1]], dtype=torch.int32)
    _verify_beam(x, scores, n_out, _beam(x, scores, n_out, done, 7), done, 7)


def test_beam_of_zeros_of_either_sign():
    """They are equal: the lowest place wins."""
    for V in (200, 9000, 30000):
        x = torch.where(torch.arange(V) % 3 == 0, 0.0, -0.0).expand(2, 2, V).contiguous()
        x[1, :, ::7] = -1.0
        s = torch.zeros((2, 2))
        _verify_beam(x, s, 20, _beam(x, s, 20))


@pytest.mark.parametrize("order", ["rising", "falling", "steps"])
def test_beam_of_sorted_logits(order):
    """Every tile brings better ones, or none, or blocks of equal ones."""
    V = 40001
    i = torch.arange(V, dtype=torch.float32)
    x = {"rising": i / 512, "falling": -i / 512, "steps": (i / 1000).floor()}[order].expand(1, 2, V).contiguous()
    s = torch.tensor([[-0.5, -1.0]])
    _verify_beam(x, s, 40, _beam(x, s, 40))


def test_beam_with_logits_that_are_not_finite():
    x = _logits((6, 3, 9001), F32, 31)
    x[0, 1, 4000] = math.nan            # the row offers nothing
    x[1, 0, 17] = math.inf
    x[2, 2] = -math.inf
    x[3, 0, 5:] = -math.inf             # five tokens are left
    x[3, 1:] = -math.inf
    x[4] = math.nan
    x[5, 1] = 3.0e38
    x[5, 2] = -3.0e38
    s = torch.zeros((6, 3))
    s[5, 0] = math.nan
    got = _beam(x, s, 9)
    _verify_beam(x, s, 9, got)
    assert (got[0][4] == -1).all() and (got[0][3][5:] == -1).all() and not (got[0][0] == 1).any()


@pytest.mark.parametrize("dt,pad,offset", [(BF, 1, 0), (BF, 3, 5), (F32, 1, 2), (BF, 8, 8), (F32, 4, 4)])
def test_beam_rows_of_any_alignment(dt, pad, offset):
    """Rows that are views: what lies between them is not read into the result."""
    groups, W, V = 3, 5, 10007
    room = torch.full((groups * W * (V + pad) + offset + 7,), math.inf, dtype=dt, device="cuda")
    x = torch.as_strided(room, (groups * W, V), (V + pad, 1), offset)
    x.copy_(_logits((groups * W, V), dt, 41))
    s = -torch.rand((groups, W), generator=torch.Generator().manual_seed(1))
    _verify_beam(x.cpu().view(groups, W, V), s, 12, _beam(x, s, 12))


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("kind", ["equal", "rising"])
def test_beam_log_sums_of_very_long_rows(kind, dt):
    """More beams than half the lists, so that a thread walks hundreds of tiles of a row, and logits whose roundings do not average out: equal ones below the
    best one of every thread, or ones that rise a little from tile to tile.  Log-sums are off by 2^-18 at most: an exponential of a difference d of up to 32 takes half a step
    of d (2^-20), half a step of d log2(e) times ln 2 (2^-19 ln 2) and a step of the result (2^-23), a sum of 32 of them nine roundings (9 * 2^-24), together
    3.1 * 2^-20; terms further below are 2^23 e^-32 of a sum at most; and everything beyond is in 64 bits.  Then one rounding to float."""
    W, V = 33, 4000004
    x = torch.empty((W, V), dtype=dt, device="cuda")
    tile = torch.arange(V, device="cuda") // (4096 if dt == F32 else 8192)
    for w in range(W):
        if kind == "equal":
            x[w] = -(3 + w / 11.0)
            x[w, :2048] = 0.0
        else:
            x[w] = (tile * 2.0 ** -10 * (0.5 + w / 8.0)).to(dt)
        x[w, V - 1 - 1000 * w] = 8.0 if kind == "equal" else float(x[w, -1]) + 12
    want = np.array([float(x[w].max().double() - torch.logsumexp(x[w].double(), 0)) for w in range(W)])
    order = np.argsort(-want, kind="stable")
    got = _beam(x, torch.zeros((1, W)), W)
    assert np.array_equal(np.sort(got[0][0]), np.arange(W)) and np.array_equal(got[1][0], V - 1 - 1000 * got[0][0])
    assert (np.abs(got[2][0] - want[got[0][0]]) <= 2.0 ** -18 + 2.0 ** -24 * np.abs(want[got[0][0]])).all()
    assert (np.abs(want[got[0][0]] - want[order]) <= 2.0 ** -17).all()      # (closer ones may change places)


def test_beam_workspaces_hold_anything_on_any_stream():
    x, s = _logits((4, 3, 30000), BF, 51).cuda(), torch.zeros((4, 3))
    need = api.beam_workspace_bytes(x, 4, 7)
    first = _beam(x, s, 7)
    side = torch.cuda.Stream()
    for fill in (0, 255):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            got = _beam(x, s, 7, workspace=ws)
        assert all(np.array_equal(a, b) for a, b in zip(first, got))


# ---- together ----

class Toy:
    """One layer over cached rows: a token's rows come from tables, what it attends to goes to logits.  The same numbers in 64 bits."""

    def __init__(self, V, Hq, Hkv, D, dt, device, seed=3):
        gen = torch.Generator().manual_seed(seed)
        self.V, self.Hq, self.Hkv, self.D, self.dt = V, Hq, Hkv, D, dt
        self.emb = torch.randn((V, (Hq + 2 * Hkv) * D), generator=gen).to(dt).to(device)
        self.head = (torch.randn((Hq * D, V), generator=gen) / math.sqrt(Hq * D) * 6).to(device)

    def rows(self, tokens):
        q, k, v = self.emb[tokens.long()].split([self.Hq * self.D, self.Hkv * self.D, self.Hkv * self.D], 1)
        return q.unflatten(1, (self.Hq, self.D)), k.unflatten(1, (self.Hkv, self.D)), v.unflatten(1, (self.Hkv, self.D))

    def logits(self, o):
        return o.flatten(1).float() @ self.head

    def next_logits(self, tokens, rope):
        """Of one whole text, in 64 bits on the CPU: every key rotated and rounded as the cache keeps it."""
        q, k, v = self.rows(torch.tensor(tokens))
        n, half = len(tokens), rope.cos.shape[1]
        cos, sin = rope.cos[:n].double().cpu()[:, None], rope.sin[:n].double().cpu()[:, None]

        def turn(x):
            x = x.double()
            a, b = x[..., :half], x[..., half:2 * half]
            return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], -1).to(self.dt).double()
        q, k, v, G = turn(q)[-1], turn(k), v.double(), self.Hq // self.Hkv
        k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
        p = torch.softmax((q[None] * k).sum(-1) / math.sqrt(self.D), 0)
        return (p[..., None] * v).sum(0).flatten() @ self.head.double()


def _search_plain(toy, prompts, W, steps, rope):
    """Whole texts, no cache: [(score, tokens)] of every prompt, best first."""
    out = []
    for prompt in prompts:
        beams = [(0.0, list(prompt))]
        for _ in range(steps):
            cand = []
            for i, (s, text) in enumerate(beams):
                x = toy.next_logits(text, rope)
                x = x - torch.logsumexp(x, 0)
                cand += [(-(s + float(x[v])), i, v) for v in range(toy.V)]
            beams = [(-c, beams[i][1] + [v]) for c, i, v in sorted(cand)[:W]]
        out.append(beams)
    return out


@pytest.mark.parametrize("dt,D,P,graph", [(F32, 64, 16, False), (F32, 128, 16, True)])
def test_beam_search_over_a_paged_cache(dt, D, P, graph):
    """Prompts of odd lengths into the cache, then steps of selection, fork, copy, append and attention, eager or captured once and replayed: texts and
    scores are those of a search without a cache in 64 bits.  fp32, so that no choice of these hangs on a rounding."""
    W, V, steps, Hq, Hkv = 4, 40, 9, 4, 2
    prompts = [[3, 1, 4, 1, 5, 9, 2, 6, 5, 3, 5, 8, 9, 7, 9, 3, 2], [2, 7], [1] * 31]
    n = len(prompts)
    B, cols = n * W, 6
    n_phys = 90
    cpu, gpu = Toy(V, Hq, Hkv, D, dt, "cpu"), Toy(V, Hq, Hkv, D, dt, "cuda")
    rope = api.rope_tables(cols * P, D)
    pools = [torch.full((n_phys, Hkv, P, D), math.nan, dtype=dt, device="cuda") for _ in range(2)]
    refs = torch.zeros(n_phys, dtype=torch.int32, device="cuda")
    scale = 1.0 / math.sqrt(D)

    # the prompts: one sequence each, begun and filled
    start = api.page_fork(_i([[-1] * cols]), _i([0]), _i([api.FORK_BEGINS] * n), refs, P, grow=_i([len(p) for p in prompts]))
    tokens = _i(sum(prompts, []))
    q, k, v = gpu.rows(tokens)
    at = dict(seq_lens=start.lens, row_starts=_i([0] + list(np.cumsum([len(p) for p in prompts]))))
    desc = api.make_rows_desc(q, pools[0], start.tables, cols * P, scale, max_rows=31)
    y = api.kv_append_rope(desc, k, v, start.tables, *pools, q=q, rope=rope, **at)
    o, _ = api.paged_attn_fwd_rows(desc, y, *pools, start.tables, **at)
    last = at["row_starts"][1:].long() - 1
    # the first choice: one live hypothesis a text, the others hold nothing
    logits = torch.zeros((B, V), device="cuda")
    logits[::W] = gpu.logits(o[last])
    scores = torch.full((n, W), -math.inf, device="cuda")
    scores[:, 0] = 0.0
    tables = [torch.full((B, cols), -1, dtype=torch.int32, device="cuda") for _ in range(2)]
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    tables[0][::W], lens[::W] = start.tables, start.lens
    texts = torch.zeros((B, cols * P), dtype=torch.int32, device="cuda")
    grow = _i([1] * B)
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    par, tok, best = torch.zeros((n, W), dtype=torch.int32, device="cuda"), torch.zeros((n, W), dtype=torch.int32, device="cuda"), torch.zeros((n, W), device="cuda")
    copies = torch.zeros((B, 3), dtype=torch.int32, device="cuda")
    missing = torch.zeros((), dtype=torch.int32, device="cuda")
    wide = api.make_rows_desc(torch.zeros((B, Hq, D), dtype=dt, device="cuda"), pools[0], tables[0], cols * P, scale, max_rows=1)
    ws = [torch.zeros(max(16, x), dtype=torch.uint8, device="cuda") for x in (api.beam_workspace_bytes(logits, n, W), api.page_fork_workspace_bytes(B, B, n_phys),
                                                                             api.rows_workspace_bytes(wide))]
    yq, oo = (torch.zeros((B, Hq, D), dtype=dt, device="cuda") for _ in range(2))
    ll = torch.zeros((Hq, B), device="cuda")

    def step(a, b, i):
        api.beam_topk(logits, scores, W, parents=par, tokens=tok, scores_out=best, workspace=ws[0])
        api.page_fork(tables[a], lens, par.view(-1), refs, P, grow=grow, tables_out=tables[b], lens_out=lens, copies=copies, status=status, workspace=ws[1])
        api.page_copy(pools, copies)
        missing.add_(status[1])
        scores.copy_(best)
        q, k, v = gpu.rows(tok.view(-1))
        desc = api.make_rows_desc(q, pools[0], tables[b], cols * P, scale, max_rows=1)
        api.kv_append_rope(desc, k, v, tables[b], *pools, q=q, q_out=yq, rope=rope, seq_lens=lens)
        api.paged_attn_fwd_rows(desc, yq, *pools, tables[b], o=oo, lse=ll, workspace=ws[2], seq_lens=lens)
        logits.copy_(gpu.logits(oo))
        texts.copy_(texts[par.view(-1).long()])
        texts.scatter_(1, i.expand(B, 1), tok.view(-1, 1))

    where = torch.zeros((1, 1), dtype=torch.int64, device="cuda")
    if graph:
        gpu.logits(oo)      # (the library's handles and workspaces exist before the capture)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        graphs = []
        with torch.cuda.stream(side):
            gpu.logits(oo)
            side.synchronize()
            for a, b in ((0, 1), (1, 0)):
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=side):
                    step(a, b, where)
                graphs.append(g)
        torch.cuda.synchronize()
    for i in range(steps):
        where.fill_(i)
        if graph:
            graphs[i % 2].replay()
        else:
            step(i % 2, 1 - i % 2, where)
        torch.cuda.synchronize()
    assert int(missing) == 0
    want = _search_plain(cpu, prompts, W, steps, rope)
    got_texts, got_scores = texts.cpu()[:, :steps].view(n, W, steps), scores.cpu()
    for i, prompt in enumerate(prompts):
        for w in range(W):
            s, text = want[i][w]
            assert got_texts[i, w].tolist() == text[len(prompt):], (i, w)
            # attention and rotation off by 2^-18 of values of up to 4, a head of Hq D of them: under 1e-4 a step
            assert abs(float(got_scores[i, w]) - s) < 1e-4 * steps
    # every page is named as often as the counts say
    count = [0] * n_phys
    final = tables[steps % 2].tolist()
    for row, t in zip(final, lens.tolist()):
        for x in row[:-(-t // P)]:
            count[x] += 1
    assert count == refs.tolist()


def _search_plain_that_ends(toy, prompts, W, steps, rope, eos, pad):
    """_search_plain whose texts end: one that holds eos stays as it is and goes on with pad."""
    out = []
    for prompt in prompts:
        beams = [(0.0, list(prompt), False)]
        for _ in range(steps):
            cand = []
            for i, (s, text, over) in enumerate(beams):
                if over:
                    cand.append((-s, i, pad))
                    continue
                x = toy.next_logits(text, rope)
                x = x - torch.logsumexp(x, 0)
                cand += [(-(s + float(x[v])), i, v) for v in range(toy.V)]
            beams = [(-c, beams[i][1] + [v], beams[i][2] or v == eos) for c, i, v in sorted(cand)[:W]]
        out.append(beams)
    return out


@pytest.mark.parametrize("D,eos,steps,graph", [(64, 7, 12, False), (64, 7, 12, True), (128, 6, 6, False), (128, 6, 6, True)])
def test_beam_search_whose_texts_end(D, eos, steps, graph):
    """The loop of a program: who has ended, the texts and the page means follow the parents; hypotheses that have ended hold no pages, their rows do not exist, and their
    logits are NaN.  Some end and are beaten later, and some texts end in all their hypotheses.  (Candidates next to each other at the edge are 2e-3 apart at least.)"""
    W, V, Hq, Hkv, P, pad, cols, n_phys = 4, 40, 4, 2, 16, 11, 6, 90
    prompts = [[3, 1, 4, 1, 5, 9, 2, 6, 5, 3, 5, 8, 9, 7, 9, 3, 2], [2, 7], [1] * 31]
    n = len(prompts)
    B = n * W
    cpu, gpu = Toy(V, Hq, Hkv, D, F32, "cpu"), Toy(V, Hq, Hkv, D, F32, "cuda")
    rope = api.rope_tables(cols * P, D)
    pools = [torch.full((n_phys, Hkv, P, D), math.nan, device="cuda") for _ in range(2)]
    refs = torch.zeros(n_phys, dtype=torch.int32, device="cuda")
    scale = 1.0 / math.sqrt(D)
    start = api.page_fork(_i([[-1] * cols]), _i([0]), _i([api.FORK_BEGINS] * n), refs, P, grow=_i([len(p) for p in prompts]))
    q, k, v = gpu.rows(_i(sum(prompts, [])))
    starts = _i([0] + list(np.cumsum([len(p) for p in prompts])))
    first_means = torch.zeros((n, cols, Hkv, D), device="cuda")
    desc = api.make_rows_desc(q, pools[0], start.tables, cols * P, scale, max_rows=31)
    y = api.kv_append_rope(desc, k, v, start.tables, *pools, q=q, rope=rope, kbar_cache=first_means, seq_lens=start.lens, row_starts=starts)
    o, _ = api.paged_attn_fwd_rows(desc, y, *pools, start.tables, seq_lens=start.lens, row_starts=starts)
    logits = torch.full((B, V), math.nan, device="cuda")
    logits[::W] = gpu.logits(o[starts[1:].long() - 1])
    scores = torch.full((n, W), -math.inf, device="cuda")
    scores[:, 0] = 0.0
    done = torch.zeros((n, W), dtype=torch.int32, device="cuda")
    tables = torch.full((B, cols), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    tables[::W], lens[::W] = start.tables, start.lens
    means = torch.zeros((B, cols, Hkv, D), device="cuda")
    means[::W] = first_means
    texts = torch.zeros((B, steps), dtype=torch.int32, device="cuda")
    missing, at = torch.zeros((), dtype=torch.int32, device="cuda"), torch.zeros((1, 1), dtype=torch.int64, device="cuda")
    ones = _i([1] * B)

    def step():
        parents, tokens, best = api.beam_topk(logits, scores, W, done=done, pad_token=pad)
        rows = parents.flatten()
        came = rows.clamp(min=0)
        over = done.flatten()[came] | (tokens.flatten() == eos)
        new = api.page_fork(tables, lens, torch.where(over != 0, api.FORK_NONE, rows), refs, P, grow=ones)
        api.page_copy(pools, new.copies)
        missing.add_(new.status[1])
        means.copy_(means[came])
        q, k, v = gpu.rows(tokens.flatten())
        desc = api.make_rows_desc(q, pools[0], new.tables, cols * P, scale, max_rows=1)
        y = api.kv_append_rope(desc, k, v, new.tables, *pools, q=q, rope=rope, kbar_cache=means, seq_lens=new.lens)
        o, _ = api.paged_attn_fwd_rows(desc, y, *pools, new.tables, seq_lens=new.lens)
        logits.copy_(torch.where(over[:, None] != 0, math.nan, gpu.logits(o)))
        scores.copy_(best)
        done.copy_(over.view(n, W))
        tables.copy_(new.tables)
        lens.copy_(new.lens)
        texts.copy_(texts[came])
        texts.scatter_(1, at.expand(B, 1), tokens.view(-1, 1))

    if graph:
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            gpu.logits(torch.zeros((B, Hq, D), device="cuda"))     # (the library's handles and workspaces exist before the capture)
            side.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                step()
        torch.cuda.synchronize()
    for i in range(steps):
        at.fill_(i)
        if graph:
            g.replay()
        else:
            step()
        torch.cuda.synchronize()
    assert int(missing) == 0
    want = _search_plain_that_ends(cpu, prompts, W, steps, rope, eos, pad)
    over = [[b[2] for b in beams] for beams in want]
    assert any(all(x) for x in over) and not all(all(x) for x in over)
    assert done.tolist() == [[int(x) for x in y] for y in over]
    got, got_scores = texts.cpu().view(n, W, steps), scores.cpu()
    for i, prompt in enumerate(prompts):
        for w in range(W):
            assert got[i, w].tolist() == want[i][w][1][len(prompt):], (i, w)
            assert abs(float(got_scores[i, w]) - want[i][w][0]) < 1e-4 * steps      # (as above: under 1e-4 a step)
    # pages of ended hypotheses are free, the others counted; the means are those of the pages' keys
    assert lens.tolist() == [0 if over[b // W][b % W] else len(prompts[b // W]) + steps for b in range(B)]
    count = [0] * n_phys
    for b, (row, t) in enumerate(zip(tables.tolist(), lens.tolist())):
        for x in row[:-(-t // P)]:
            count[x] += 1
        for l in range(t // P):
            keys = pools[0][row[l]].double()
            tol = P * 2.0 ** -24 * keys.abs().mean(1)                               # (sums of P in fp32)
            assert ((means[b, l].double() - keys.mean(1)).abs() <= tol).all()
    assert count == refs.tolist()
