"""Which form of its launch attention over pages takes, by the rules of the dispatch itself (host only)."""
import struct

import pytest

from test_host_packed_cache import DTYPE, NULL, SHAPE, cache, ha  # noqa: F401  (ha: a fixture)


def test_codes_go_past_the_caches_where_the_table_has_room_for_more_than_they_hold(ha):
    """256 MiB: with 8 heads of d = 128 and pages of 64, 3855 entries are below, 3856 above."""
    form = lambda n_seq, max_blocks, q_len=1: ha.ha_cache4_attn_form(1000, 64, 8, 128, n_seq, q_len, 32, max_blocks)  # noqa: E731
    assert form(4, 964) == (0, True) and form(1, 3856) == (0, True) and form(1, 3855) == (0, False)
    assert form(64, 256, q_len=3) == (0, True)
    assert form(4, 2048, q_len=4) == (0, True) and form(4, 2048, q_len=5) == (0, False)   # a second tile of rows reads the codes again


def test_small_tables_have_a_workgroup_per_sequence(ha):
    form = lambda n_seq, max_blocks, Hk=4, q_len=1: ha.ha_cache4_attn_form(100000, 16, Hk, 64, n_seq, q_len, 4 * Hk, max_blocks)  # noqa: E731
    assert form(1, 64) == (8, False) and form(1, 65) == (0, False)          # 1024 tokens
    assert form(16, 128) == (8, False) and form(16, 129) == (0, False)      # 64 workgroups: 2048
    assert form(15, 128) == (0, False) and form(64, 128) == (8, False) and form(65, 128) == (4, False) and form(128, 128) == (4, False)
    assert form(129, 128) == (0, False) and form(2000, 64) == (4, False)    # more than 512: 1024 again
    assert form(33, 64, q_len=8) == (4, False)                              # two tiles of rows
    assert ha.ha_cache4_attn_form(0, 16, 4, 64, 4, 1, 16, 1 << 20) == (8, False)   # no page: every sequence is empty


def test_refusals(ha):
    import ctypes
    call, x = ha.lib().ha_cache4_attn_form, ctypes.c_int32(0)
    q = struct.pack("5i", 2, 1, 4, 0, 8)
    assert call(cache(), q, None, x) == NULL and call(cache(), q, x, None) == NULL and call(None, q, x, x) == NULL and call(cache(), None, x, x) == NULL
    assert call(cache(page=24), q, x, x) == SHAPE and call(cache(), struct.pack("5i", 2, 65, 4, 0, 8), x, x) == SHAPE
    assert call(cache(), struct.pack("5i", 2, 1, 4, 7, 8), x, x) == DTYPE
    with pytest.raises(TypeError):
        import torch
        ha.ha_cache4_attn_form(8, 16, 2, 64, 2, 1, 4, 8, dtype=torch.float16)
