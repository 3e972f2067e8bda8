"""Host-side checks of the entry points over packed rows that need no GPU: descriptors, workspaces, and every refusal before a launch."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2602_02108_amd import api

import rows_util as ru

FAKE = 0x1000   # never dereferenced: validation fails first


def _desc(**kw):
    """A batch of 8 sequences over a pool of 4-bit codes"""
    tile = api.kvq_tile_bytes(128, 128)
    d = api.RowsDesc(28, 4, 128, 128, api.BF16, 8, 64, 8, 0.1, 0, 4096, 32, 300, 4 * tile, tile, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _plain(**kw):
    return _desc(**{**dict(pool_page_stride=4 * 128 * 128, pool_head_stride=128 * 128, pool_tok_stride=128), **kw})


def _rows(heads, data=FAKE, tok=None, head=128):
    return api.Rows(data, heads * 128 if tok is None else tok, head)


SEQS = api.Seqs(FAKE, FAKE, FAKE)
ROPE = api.RopeDesc(FAKE, FAKE, 4096, 128, 0)


def _call(name, d, seqs=SEQS, rope=ROPE, q=None, q_out=None, k=None, v=None, k_pool=FAKE, v_pool=FAKE + 16, grad=api.F32, sel=None, cnt=None, stride=0,
          lse=FAKE, ws=FAKE, ws_bytes=1 << 40):
    l = api.lib()
    r = ctypes.byref
    q, q_out, k, v = q or _rows(28), q_out or _rows(28), k or _rows(4), v or _rows(4)
    sq = r(seqs) if seqs else None
    rp = r(rope) if rope else None
    kp, vp = ctypes.c_void_p(k_pool), ctypes.c_void_p(v_pool)
    if name == "attn":
        return l.oomb_paged_attn_fwd_kvq(r(d), sq, r(q), kp, vp, sel, cnt, stride, r(q_out), ctypes.c_void_p(lse), ctypes.c_void_p(ws), ws_bytes, None)
    if name == "read":
        return l.oomb_kvq_read(r(d), sq, kp, vp, r(k), r(v), None)
    if name == "bwd":
        return l.oomb_kv_append_rope_bwd(r(d), sq, rp, r(q), r(q_out), kp, vp, grad, r(k), r(v), None)
    f = l.oomb_kvq_append_rope if name == "kvq" else l.oomb_kv_append_rope
    return f(r(d), sq, rp, r(q), r(q_out), r(k), r(v), kp, vp, None, None)


ALL = ["append", "bwd", "kvq", "read", "attn"]


def _for(name, **kw):
    return (_plain if name in ("append", "bwd") else _desc)(**kw)


def test_structs_match_the_header():
    assert ctypes.sizeof(api.RowsDesc) == 10 * 4 + 6 * 8 and api.RowsDesc.max_len.offset == 40
    assert ctypes.sizeof(api.Rows) == 24 and ctypes.sizeof(api.Seqs) == 24 and ctypes.sizeof(api.RopeDesc) == 32


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("kw,want", [
    (dict(n_kv_heads=5), api.ERR_INVALID_ARG), (dict(n_q_heads=0), api.ERR_INVALID_ARG), (dict(dtype=7), api.ERR_INVALID_ARG),
    (dict(reserved=1), api.ERR_INVALID_ARG), (dict(n_seqs=0), api.ERR_INVALID_ARG), (dict(n_rows=0), api.ERR_INVALID_ARG),
    (dict(max_rows=0), api.ERR_INVALID_ARG), (dict(max_rows=65), api.ERR_INVALID_ARG), (dict(max_len=0), api.ERR_INVALID_ARG),
    (dict(max_len=4097), api.ERR_INVALID_ARG),            # more than the tables hold
    (dict(num_phys_pages=0), api.ERR_INVALID_ARG), (dict(pool_head_stride=1001), api.ERR_INVALID_ARG),
    (dict(pool_page_stride=4 * 128 * 128 * 8 + 1), api.ERR_INVALID_ARG),
    (dict(head_dim=96), api.ERR_UNSUPPORTED), (dict(page_size=8), api.ERR_UNSUPPORTED), (dict(page_size=48), api.ERR_UNSUPPORTED),
    (dict(page_size=256), api.ERR_UNSUPPORTED),
    (dict(max_len=1 << 31, table_stride=1 << 25), api.ERR_UNSUPPORTED),
    (dict(n_rows=1 << 30, max_rows=1 << 29), api.ERR_UNSUPPORTED),
])
def test_bad_descriptors(name, kw, want):
    rope = api.RopeDesc(FAKE, FAKE, 1 << 40, 128, 0)
    assert _call(name, _for(name, **kw), rope=rope) == want


@pytest.mark.parametrize("name", ALL)
def test_bad_tensors(name):
    bad = api.ERR_INVALID_ARG
    kv = name in ("append", "bwd", "kvq", "read")
    for r in (_rows(4, data=0), _rows(4, data=0x1004), _rows(4, tok=64), _rows(4, tok=515), _rows(4, head=100)):
        if kv:
            assert _call(name, _for(name), k=r) == bad and _call(name, _for(name), v=r) == bad
        if name != "read":
            assert _call(name, _for(name), q=r) == bad and _call(name, _for(name), q_out=r) == bad
    assert _call(name, _for(name), k_pool=0) == bad and _call(name, _for(name), v_pool=0x1008) == bad
    assert _call(name, _for(name), seqs=None) == bad and _call(name, _for(name), seqs=api.Seqs(None, FAKE, FAKE)) == bad
    # without row_starts every sequence has the same rows, and max_rows holds them
    assert _call(name, _for(name, n_rows=63), seqs=api.Seqs(FAKE, None, None)) == bad
    assert _call(name, _for(name, max_rows=7), seqs=api.Seqs(FAKE, None, None)) == bad


@pytest.mark.parametrize("name", ["append", "bwd", "kvq"])
@pytest.mark.parametrize("rope", [api.RopeDesc(None, FAKE, 4096, 128, 0), api.RopeDesc(FAKE, 0x1004, 4096, 128, 0), api.RopeDesc(FAKE, FAKE, 4095, 128, 0),
                                  api.RopeDesc(FAKE, FAKE, 4096, 120, 0), api.RopeDesc(FAKE, FAKE, 4096, 144, 0), api.RopeDesc(FAKE, FAKE, 4096, -16, 0)])
def test_bad_rotations(name, rope):
    assert _call(name, _for(name), rope=rope) == api.ERR_INVALID_ARG


def test_what_only_one_of_them_refuses():
    l, r = api.lib(), ctypes.byref
    bad = api.ERR_INVALID_ARG
    assert _call("bwd", _plain(), grad=5) == bad
    assert _call("bwd", _plain(pool_tok_stride=132), grad=api.BF16) == bad       # (264 bytes: rows lose their alignment)
    assert _call("append", _plain(), v_pool=FAKE) == bad                         # K and V in one pool
    assert l.oomb_kv_append_rope(r(_plain()), r(SEQS), None, r(_rows(28)), None, r(_rows(4)), r(_rows(4)), FAKE, FAKE + 16, None, None) == bad
    assert l.oomb_kv_append_rope_bwd(r(_plain()), r(SEQS), None, None, r(_rows(28)), FAKE, FAKE, 0, r(_rows(4)), r(_rows(4)), None) == bad
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert _call("attn", _desc(sm_scale=scale)) == bad
    assert _call("attn", _desc(), lse=0) == bad
    assert _call("attn", _desc(), sel=FAKE, cnt=None, stride=4) == bad
    assert _call("attn", _desc(), sel=FAKE, cnt=FAKE, stride=-1) == bad


def test_workspaces():
    one = _desc(n_seqs=1, n_rows=1, max_rows=1, max_len=1 << 20, table_stride=1 << 13, num_phys_pages=1 << 13)
    need = api.kvq_workspace_bytes(one)
    assert need > 0
    assert _call("attn", one, ws=0, ws_bytes=0) == api.ERR_WORKSPACE
    assert _call("attn", one, ws_bytes=need - 1) == api.ERR_WORKSPACE
    assert _call("attn", one, ws=0x1008) == api.ERR_WORKSPACE
    assert api.kvq_workspace_bytes(one, 4) <= need                               # short lists are split less
    assert api.kvq_workspace_bytes(_desc(n_seqs=1, n_rows=1, max_rows=1, max_len=100)) == 0
    assert api.kvq_workspace_bytes(_desc(head_dim=32)) == 0
    assert api.kvq_workspace_bytes(_desc(), -1) == api.kvq_workspace_bytes(_desc(sm_scale=0.0), -1)


def test_the_python_calls_say_which_tensor_does_not_fit():
    q, k = torch.zeros((4, 8, 64)), torch.zeros((4, 2, 64))
    pool, kvq = torch.zeros((5, 2, 16, 64)), api.kvq_pool(5, 2, 16, 64, "cpu")
    table = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(api.OombError, match="make_rows_desc"):
        api.make_rows_desc(q.half(), pool, table, 48)
    with pytest.raises(api.OombError, match="make_rows_desc"):
        api.make_rows_desc(q, kvq[..., :-1], table, 48)
    d, dq = api.make_rows_desc(q, pool, table, 48), api.make_rows_desc(q, kvq, table, 48)
    assert (d.n_q_heads, d.n_kv_heads, d.head_dim, d.page_size, d.n_seqs, d.n_rows, d.max_rows, d.table_stride) == (8, 2, 64, 16, 2, 4, 4, 3)
    assert dq.page_size == 16 and dq.pool_page_stride == 2 * api.kvq_tile_bytes(16, 64) and dq.sm_scale == 1.0

    def refused(match, f, *a, **kw):
        with pytest.raises(api.OombError, match=match) as e:
            f(*a, **kw)
        assert e.value.status == api.ERR_INVALID_ARG

    refused("one GPU", api.kv_append_rope, d, k, k, table, pool, pool.clone())
    refused("one GPU", api.kvq_append_rope, dq, k, k, table, kvq, kvq.clone())
    refused("one GPU", api.kv_append_rope_bwd, d, pool, pool, table)
    refused("one GPU", api.kvq_read, dq, kvq, kvq, table)
    refused("one GPU", api.paged_attn_fwd_kvq, dq, q, kvq, kvq, table)
    refused("k must be", api.kv_append_rope, d, k[:3], k, table, pool, pool)
    refused("v must be", api.kv_append_rope, d, k, k.bfloat16(), table, pool, pool)
    refused("q_out must be", api.kv_append_rope, d, k, k, table, pool, pool, q=q, q_out=k)
    refused("q must be", api.kv_append_rope, d, k, k, table, pool, pool, q_out=q)
    refused("k_pool must be", api.kv_append_rope, d, k, k, table, kvq, kvq)
    refused("v_pool must be", api.kvq_append_rope, dq, k, k, table, kvq, kvq[:4])
    refused("dv_pool must be", api.kv_append_rope_bwd, d, pool, pool.bfloat16(), table)
    refused("page_tables", api.kvq_read, dq, kvq, kvq, table.long())
    refused("page_tables", api.kvq_read, dq, kvq, kvq, table[:, :2])
    refused("page_tables", api.kvq_read, dq, kvq, kvq, table[0])
    refused("seq_lens", api.kvq_read, dq, kvq, kvq, table, seq_lens=torch.zeros(3, dtype=torch.int32))
    refused("row_starts", api.kvq_read, dq, kvq, kvq, table, row_starts=torch.zeros(2, dtype=torch.int32))
    refused("rope", api.kv_append_rope, d, k, k, table, pool, pool, rope=api.Rope(torch.zeros(48, 32), torch.zeros(48, 16)))
    refused("kbar_cache", api.kv_append_rope, d, k, k, table, pool, pool, kbar_cache=torch.zeros((3, 2, 64)))
    refused("kbar_cache", api.kv_append_rope, d, k, k, table, pool, pool, kbar_cache=torch.zeros((2, 2, 2, 64)))
    refused("lse must be", api.paged_attn_fwd_kvq, dq, q, kvq, kvq, table, lse=torch.zeros((4, 8)))
    refused("o must be", api.paged_attn_fwd_kvq, dq, q, kvq, kvq, table, o=q.bfloat16())
    refused("sel_pages", api.paged_attn_fwd_kvq, dq, q, kvq, kvq, table, sel_pages=torch.zeros((2, 2, 3)), sel_count=torch.zeros((2, 2), dtype=torch.int32))
    refused("sel_pages", api.paged_attn_fwd_kvq, dq, q, kvq, kvq, table, sel_pages=torch.zeros((2, 2, 3), dtype=torch.int32))


def test_rope_tables_hold_far_angles():
    r = api.rope_tables(1 << 20, 16, 500000.0, True, "cpu")
    assert r.interleaved and r.cos.shape == r.sin.shape == (1 << 20, 8) and r.cos.dtype == torch.float32
    p, i = (1 << 20) - 1, 1
    a = p * 500000.0 ** (-2 * i / 16)
    assert abs(float(r.cos[p, i]) - math.cos(a)) < 1e-7 and abs(float(r.sin[p, i]) - math.sin(a)) < 1e-7


def test_means_desc_fits_the_selection_calls():
    d = api.means_desc(torch.zeros((32, 4, 64), dtype=torch.bfloat16), 2, 16, 160, 0.5)
    assert api.workspace_bytes(d, 3, api.OP_SCORE_TOPK) > 0 and d.ctx_len == 160 and d.n_kv_heads == 2


def test_the_tests_own_quantiser():
    """Against the grid by hand: halves to the even code, 7 stays with the smaller scale, the block's other values follow its scale."""
    x = np.zeros((1, 32))
    x[0, :10] = [7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.2500001, -4.9]
    code, byte = ru.quantise(x)
    assert byte[0, 0] == 127
    assert ru.values(code, byte)[0, :10].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -0.5, -4.0]
    x[0, 0] = 7.0000001
    code, byte = ru.quantise(x)
    assert byte[0, 0] == 128 and ru.values(code, byte)[0, :3].tolist() == [8.0, 0.0, 1.0]
    tiles = ru.pack(np.tile(code, (1, 16, 2)), np.tile(byte, (1, 16, 2)))
    back = ru.unpack(tiles, 16, 64)
    assert (back[0][0, 3, :32] == code[0]).all() and (back[1] == 128).all()
