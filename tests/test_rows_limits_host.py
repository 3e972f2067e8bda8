"""Host-side limits of the calls over packed rows, without a GPU: what a launch can hold, on both sides."""
import ctypes

import pytest

from paper_2602_02108_amd import api

FAKE = 0x1000   # never dereferenced: validation fails first


def _attend(n_seqs, max_rows, heads=(28, 4), D=128, dtype=api.BF16, max_len=1024, n_rows=None, lists=None):
    """Status of an attention call without a place for LSE: ERR_INVALID_ARG where everything before that fits, and nothing is launched."""
    Hq, Hkv = heads
    tile = api.kvq_tile_bytes(128, D)
    d = api.RowsDesc(Hq, Hkv, D, 128, dtype, n_seqs, n_rows or max(max_rows, n_seqs), max_rows, 0.1, 0, max_len, (max_len + 127) // 128, 1 << 20, Hkv * tile, tile, 0)
    q, r = api.Rows(FAKE, Hq * D, D), ctypes.byref
    sel = ctypes.c_void_p(FAKE) if lists is not None else None
    return api.lib().oomb_paged_attn_fwd_kvq(r(d), r(api.Seqs(FAKE, FAKE, FAKE)), r(q), FAKE, FAKE + 16, sel, sel, lists or 0, r(q), None, FAKE, 1 << 50, None)


FITS, TOO_MANY = api.ERR_INVALID_ARG, api.ERR_UNSUPPORTED


@pytest.mark.parametrize("kw,want", [
    (dict(n_seqs=64, max_rows=9400, max_len=9400), FITS),                    # one prompt beside single tokens
    (dict(n_seqs=1, max_rows=600000, max_len=1 << 20), FITS),                # one prompt at once
    (dict(n_seqs=128, max_rows=8192, max_len=32768), FITS),
    (dict(n_seqs=32, max_rows=32768, max_len=32768), FITS),                  # the bound of a call that gives none
    (dict(n_seqs=128, max_rows=8192, max_len=32768, lists=64), FITS),
    (dict(n_seqs=4096, max_rows=4676), FITS),                                # 4096 x 4 x 1023 row blocks of 32
    (dict(n_seqs=4096, max_rows=4681), TOO_MANY),                            # 1024
    (dict(n_seqs=1 << 21, max_rows=2), TOO_MANY),                            # 14 rows, eight waves: 2^21 x 4, each two workgroups of 256 threads
    (dict(n_seqs=(1 << 21) - 1, max_rows=2), FITS),
    (dict(n_seqs=1 << 22, max_rows=2), TOO_MANY),
    (dict(n_seqs=1 << 14, max_rows=16 * 255, heads=(4, 4), dtype=api.F32), TOO_MANY),      # fp32 rows of head dim 128: blocks of 16, eight waves
    (dict(n_seqs=1 << 13, max_rows=16 * 255, heads=(4, 4), dtype=api.F32), FITS),          # 2^13 x 4 x 255 x 2
    (dict(n_seqs=1 << 13, max_rows=16 * 256, heads=(4, 4), dtype=api.F32), TOO_MANY),
])
def test_attention_over_codes_takes_what_its_launch_holds(kw, want):
    assert _attend(**kw) == want
