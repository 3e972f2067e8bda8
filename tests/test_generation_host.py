"""Host-side checks of generation's entry points that need no GPU: descriptors, workspaces, and every refusal before a launch."""
import ctypes
import math

import pytest
import torch

from paper_2602_02108_amd import api

FAKE = 0x100000   # never dereferenced: validation fails first
BAD, NO, ROOM = api.ERR_INVALID_ARG, api.ERR_UNSUPPORTED, api.ERR_WORKSPACE
r = ctypes.byref


def _vp(x):
    return ctypes.c_void_p(x)


# ---- attention over pools of bf16 / fp32 rows ----

def _rows_desc(**kw):
    d = api.RowsDesc(28, 4, 128, 128, api.BF16, 8, 64, 8, 0.1, 0, 4096, 32, 300, 4 * 128 * 128, 128 * 128, 128)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _rows(heads=28, data=FAKE, tok=None, head=128):
    return api.Rows(data, heads * 128 if tok is None else tok, head)


SEQS = api.Seqs(FAKE, FAKE, FAKE)


def _attn(d, seqs=SEQS, q=None, o=None, k_pool=FAKE, v_pool=FAKE, sel=None, cnt=None, stride=0, lse=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return api.lib().oomb_paged_attn_fwd_rows(r(d), r(seqs) if seqs else None, r(q or _rows()), _vp(k_pool), _vp(v_pool), sel, cnt, stride, r(o or _rows()),
                                              _vp(lse), _vp(ws), ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(n_kv_heads=5), BAD), (dict(n_q_heads=0), BAD), (dict(dtype=7), BAD), (dict(reserved=1), BAD), (dict(n_seqs=0), BAD), (dict(n_rows=0), BAD),
    (dict(max_rows=0), BAD), (dict(max_rows=65), BAD), (dict(max_len=0), BAD), (dict(max_len=4097), BAD), (dict(num_phys_pages=0), BAD),
    (dict(pool_head_stride=1001), BAD), (dict(pool_tok_stride=132), BAD), (dict(pool_tok_stride=64), BAD), (dict(sm_scale=0.0), BAD), (dict(sm_scale=-1.0), BAD),
    (dict(sm_scale=math.inf), BAD), (dict(sm_scale=math.nan), BAD),
    (dict(head_dim=96), NO), (dict(page_size=8), NO), (dict(page_size=48), NO), (dict(page_size=256), NO),
    (dict(max_len=1 << 31, table_stride=1 << 25), NO), (dict(n_rows=1 << 30, max_rows=1 << 29), NO),
    (dict(n_rows=1 << 27, max_rows=1 << 27), NO),                      # more workgroups than a launch holds
    (dict(pool_tok_stride=1 << 24), NO),                               # a page of a head spans more than 32-bit offsets reach
    (dict(pool_tok_stride=1 << 60), NO),
])
def test_attention_descriptors(kw, want):
    assert _attn(_rows_desc(**kw)) == want


def test_attention_tensors_and_workspaces():
    for t in (_rows(data=0), _rows(data=FAKE + 4), _rows(tok=64), _rows(tok=515), _rows(head=100)):
        assert _attn(_rows_desc(), q=t) == BAD and _attn(_rows_desc(), o=t) == BAD
    assert _attn(_rows_desc(), k_pool=0) == BAD and _attn(_rows_desc(), v_pool=FAKE + 8) == BAD and _attn(_rows_desc(), lse=0) == BAD
    assert _attn(_rows_desc(), seqs=None) == BAD and _attn(_rows_desc(), seqs=api.Seqs(None, FAKE, FAKE)) == BAD
    assert _attn(_rows_desc(n_rows=63), seqs=api.Seqs(FAKE, None, None)) == BAD
    assert _attn(_rows_desc(), sel=FAKE, cnt=None, stride=4) == BAD and _attn(_rows_desc(), sel=FAKE, cnt=FAKE, stride=-1) == BAD
    one = _rows_desc(n_seqs=1, n_rows=1, max_rows=1, max_len=1 << 20, table_stride=1 << 13, num_phys_pages=1 << 13)
    need = api.rows_workspace_bytes(one)
    assert need > 0 and _attn(one, ws=0, ws_bytes=0) == ROOM and _attn(one, ws_bytes=need - 1) == ROOM and _attn(one, ws=FAKE + 8) == ROOM
    assert api.rows_workspace_bytes(one, 4) <= need
    assert api.rows_workspace_bytes(_rows_desc(n_seqs=1, n_rows=1, max_rows=1, max_len=100)) == 0 and api.rows_workspace_bytes(_rows_desc(head_dim=32)) == 0


# ---- pages ----

def _pages(**kw):
    d = api.PagesDesc(8, 8, 16, 0, 100, 100, 100, 100, 500)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


AT = dict(tables=FAKE, lens=2 * FAKE, parents=3 * FAKE, grow=4 * FAKE, refs=5 * FAKE, tables_out=6 * FAKE, lens_out=7 * FAKE, refs_out=8 * FAKE, copies=9 * FAKE,
          status=10 * FAKE, map=11 * FAKE)


def _fork(d, ws=FAKE, ws_bytes=1 << 40, **kw):
    a = {**AT, **kw}
    names = ("tables", "lens", "parents", "grow", "refs", "tables_out", "lens_out", "refs_out", "copies", "status")
    return api.lib().oomb_page_fork(r(d) if d else None, *(_vp(a[n]) for n in names), _vp(ws), ws_bytes, None)


def _compact(d, ws=FAKE, ws_bytes=1 << 40, max_moves=250, **kw):
    a = {**AT, **kw}
    return api.lib().oomb_page_compact(r(d) if d else None, *(_vp(a[n]) for n in ("tables", "lens", "refs", "tables_out", "refs_out", "copies")), max_moves, _vp(a["map"]),
                                       _vp(a["status"]), _vp(ws), ws_bytes, None)


@pytest.mark.parametrize("call", [_fork, _compact])
@pytest.mark.parametrize("kw,want", [
    (dict(n_seqs=0), BAD), (dict(n_out=-1), BAD), (dict(page_size=0), BAD), (dict(reserved=3), BAD), (dict(table_cols=0), BAD), (dict(out_cols=0), BAD),
    (dict(table_stride=99), BAD), (dict(out_stride=99), BAD), (dict(num_phys_pages=0), BAD), (dict(page_size=24), NO), (dict(num_phys_pages=1 << 31), NO),
    (dict(table_cols=1 << 28, table_stride=1 << 28, out_cols=1 << 28, out_stride=1 << 28), NO),
    (dict(page_size=1, table_cols=1 << 30, table_stride=1 << 30, out_cols=1 << 30, out_stride=1 << 30), NO),
])
def test_pages_descriptors(call, kw, want):
    assert call(_pages(**kw)) == want and call(None) == BAD


def test_pages_arrays():
    for name in AT:
        if name not in ("grow", "map"):
            assert _fork(_pages(), **{name: 0}) == BAD
        if name not in ("parents", "grow", "lens_out"):
            assert _compact(_pages(), **{name: 0}) == BAD
    assert _fork(_pages(), tables_out=FAKE) == BAD and _fork(_pages(), tables_out=FAKE + 8 * 100 * 4 - 4) == BAD      # tables in each other's memory
    assert _fork(_pages(), refs_out=5 * FAKE + 4) == BAD and _compact(_pages(), refs_out=5 * FAKE - 4) == BAD
    assert _compact(_pages(), tables_out=FAKE + 4) == BAD and _compact(_pages(out_stride=128), tables_out=FAKE) == BAD
    assert _compact(_pages(n_out=7)) == BAD and _compact(_pages(out_cols=90)) == BAD and _compact(_pages(), max_moves=249) == BAD
    assert _fork(_pages(n_seqs=4097)) == NO and _fork(_pages(n_out=4097)) == NO
    need = api.page_fork_workspace_bytes(8, 8, 500)
    assert need > 0 and _fork(_pages(), ws=0) == ROOM and _fork(_pages(), ws_bytes=need - 1) == ROOM and _fork(_pages(), ws=FAKE + 4) == ROOM
    need = api.page_compact_workspace_bytes(500)
    assert need > 0 and _compact(_pages(), ws=0) == ROOM and _compact(_pages(), ws_bytes=need - 1) == ROOM
    assert api.page_fork_workspace_bytes(0, 1, 5) == 0 and api.page_fork_workspace_bytes(1, 5000, 5) == 0 and api.page_compact_workspace_bytes(-1) == 0


def _copy(pools=(FAKE, 2 * FAKE), copies=FAKE, **kw):
    d = api.CopyDesc(len(pools), 4, 16, 256, 500, 4 * 16 * 256, 16 * 256, 256, 8)
    for k, v in kw.items():
        setattr(d, k, v)
    return api.lib().oomb_page_copy(r(d), (ctypes.c_void_p * len(pools))(*pools), _vp(copies), None, None)


@pytest.mark.parametrize("kw,want", [
    (dict(n_pools=0), BAD), (dict(n_heads=0), BAD), (dict(page_size=0), BAD), (dict(row_bytes=0), BAD), (dict(row_bytes=250), BAD), (dict(num_phys_pages=0), BAD),
    (dict(page_stride=65544), BAD), (dict(head_stride=4104), BAD), (dict(tok_stride=264), BAD), (dict(tok_stride=240), BAD), (dict(page_stride=128), BAD),
    (dict(head_stride=128), BAD), (dict(max_copies=-1), BAD), (dict(max_copies=1 << 31), NO), (dict(num_phys_pages=1 << 31), NO),
    (dict(page_size=1 << 24, tok_stride=256), NO), (dict(max_copies=0), api.OK),
])
def test_copy_descriptors(kw, want):
    assert _copy(**kw) == want


def test_copy_pools():
    assert _copy(pools=(FAKE, 0)) == BAD and _copy(pools=(FAKE + 8, FAKE)) == BAD and _copy(copies=0) == BAD


# ---- beam search's selection ----

def _beam(logits=FAKE, scores=2 * FAKE, done=None, parents=3 * FAKE, tokens=4 * FAKE, out=5 * FAKE, ws=FAKE, ws_bytes=1 << 40, **kw):
    d = api.BeamDesc(3, 4, 1000, 8, api.BF16, 0, 1000)
    for k, v in kw.items():
        setattr(d, k, v)
    return api.lib().oomb_beam_topk(r(d), _vp(logits), _vp(scores), done, _vp(parents), _vp(tokens), _vp(out), _vp(ws), ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(n_groups=0), BAD), (dict(n_beams=0), BAD), (dict(vocab=0), BAD), (dict(n_out=0), BAD), (dict(dtype=4), BAD), (dict(row_stride=999), BAD),
    (dict(n_out=65), NO), (dict(n_beams=65), NO), (dict(vocab=(1 << 31) - 1, row_stride=1 << 31), NO), (dict(n_groups=1 << 30), NO), (dict(n_groups=1 << 23), NO),
    (dict(logits=0), BAD), (dict(logits=FAKE + 1), BAD), (dict(logits=FAKE + 2, dtype=api.F32), BAD), (dict(scores=0), BAD), (dict(parents=0), BAD), (dict(tokens=0), BAD),
    (dict(out=0), BAD), (dict(out=2 * FAKE + 44), BAD), (dict(ws=0), ROOM), (dict(ws=FAKE + 8), ROOM), (dict(ws_bytes=8), ROOM),
])
def test_beam_refusals(kw, want):
    assert _beam(**kw) == want


def test_structs_match_the_header():
    assert ctypes.sizeof(api.PagesDesc) == 56 and ctypes.sizeof(api.CopyDesc) == 56 and ctypes.sizeof(api.BeamDesc) == 32


def test_the_python_calls_say_which_tensor_does_not_fit():
    def refused(match, f, *a, **kw):
        with pytest.raises(api.OombError, match=match) as e:
            f(*a, **kw)
        assert e.value.status == BAD

    q, pool = torch.zeros((4, 8, 64)), torch.zeros((5, 2, 16, 64))
    table = torch.zeros((2, 3), dtype=torch.int32)
    d = api.make_rows_desc(q, pool, table, 48)
    refused("one GPU", api.paged_attn_fwd_rows, d, q, pool, pool, table)
    refused("k_pool must be", api.paged_attn_fwd_rows, d, q, api.kvq_pool(5, 2, 16, 64, "cpu"), pool, table)
    refused("v_pool must be", api.paged_attn_fwd_rows, d, q, pool, pool.bfloat16(), table)
    refused("o must be", api.paged_attn_fwd_rows, d, q, pool, pool, table, o=q.bfloat16())
    refused("lse must be", api.paged_attn_fwd_rows, d, q, pool, pool, table, lse=torch.zeros((4, 8)))
    refused("sel_pages", api.paged_attn_fwd_rows, d, q, pool, pool, table, sel_pages=torch.zeros((2, 2, 3), dtype=torch.int32))

    two, refs = torch.zeros(2, dtype=torch.int32), torch.zeros(9, dtype=torch.int32)
    refused("one GPU", api.page_fork, table, two, two, refs, 16)
    refused("seq_lens must be", api.page_fork, table, refs, two, refs, 16)
    refused("grow must be", api.page_fork, table, two, two, refs, 16, grow=refs)
    refused("tables_out must be", api.page_fork, table, two, two, refs, 16, tables_out=table[:1])
    refused("copies must be", api.page_fork, table, two, two, refs, 16, copies=table[:, :2])
    refused("refs_out must be", api.page_fork, table, two, two, refs, 16, refs_out=two)
    refused("page_tables", api.page_fork, two, two, two, refs, 16)
    refused("parents must be", api.page_fork, table, two, two.long(), refs, 16)
    refused("one GPU", api.page_compact, table, two, refs, 16)
    refused("moves must be", api.page_compact, table, two, refs, 16, moves=table[:, :2])
    refused("page_map must be", api.page_compact, table, two, refs, 16, page_map=two)
    refused("refs must be", api.page_compact, table, two, refs.long(), 16)
    copies = torch.zeros((4, 3), dtype=torch.int32)
    refused("one GPU", api.page_copy, (pool, pool), copies)
    refused("pools must be", api.page_copy, (pool, pool.bfloat16()), copies)
    refused("pools must be", api.page_copy, (), copies)
    refused("pools must be", api.page_copy, (pool[..., ::2],), copies)
    refused("copies must be", api.page_copy, pool, copies[:, :2])
    refused("count must be", api.page_copy, pool, copies, two)
    x, s = torch.zeros((6, 50)), torch.zeros((2, 3))
    refused("one GPU", api.beam_topk, x, s, 4)
    refused("logits must be", api.beam_topk, x[:5], s, 4)
    refused("logits must be", api.beam_topk, x.half(), s, 4)
    refused("equal distances", api.beam_topk, torch.zeros((2, 4, 50))[:, :3], s, 4)
    refused("scores must be", api.beam_topk, x, s[0], 4)
    refused("scores must be", api.beam_topk, x, s.double(), 4)
    refused("done must be", api.beam_topk, x, s, 4, done=s)
    refused("parents must be", api.beam_topk, x, s, 4, parents=torch.zeros((2, 5), dtype=torch.int32))
    refused("scores_out must be", api.beam_topk, x, s, 4, scores_out=torch.zeros((2, 4), dtype=torch.int32))
    refused("vocabulary", api.beam_topk, torch.zeros((6, 100))[:, ::2], s, 4)
