"""Refusals of the calls over chunks of new tokens that need no GPU.  (The addresses here are never dereferenced.)"""
import struct

import pytest

from test_host_packed_cache import ALIGN, DTYPE, NULL, OK, SHAPE, WORKSPACE, cache, ha  # noqa: F401  (ha: fixture)


def chunk(n_seq=2, rows=10, Hq=4, dtype=0, max_blocks=100):
    return struct.pack("5i", n_seq, rows, Hq, dtype, max_blocks)


def attn(ha, p=None, c=None, q=None, st=None, ws=OK, nbytes=1 << 40):
    return ha.lib().ha_cache4_attn_chunk(*(p or [OK] * 7), c or cache(), q or chunk(), st, ws, nbytes, None)


def weights(ha, p=None, c=None, q=None, st=None, ws=OK, nbytes=1 << 40, fresh=0):
    return ha.lib().ha_cache4_weights(*(p or [OK] * 7), c or cache(), q or chunk(), fresh, st, ws, nbytes, None)


BAD = [(dict(n_seq=-1), SHAPE), (dict(n_seq=(1 << 16) + 1), SHAPE), (dict(rows=-1), SHAPE), (dict(rows=(1 << 22) + 1), SHAPE), (dict(Hq=0), SHAPE), (dict(Hq=3), SHAPE),
       (dict(Hq=2048), SHAPE), (dict(rows=1 << 22, Hq=32), SHAPE), (dict(n_seq=1 << 16, Hq=128), SHAPE), (dict(max_blocks=-1), SHAPE), (dict(max_blocks=0x7FFFFFFF), SHAPE),
       (dict(n_seq=1 << 16, max_blocks=1 << 15), SHAPE), (dict(n_seq=1 << 15, max_blocks=1 << 17), SHAPE), (dict(dtype=2), DTYPE)]


@pytest.mark.parametrize("over,status", BAD)
def test_sizes(ha, over, status):
    assert attn(ha, q=chunk(**over)) == status
    assert ha.lib().ha_cache4_attn_chunk_workspace_bytes(cache(), chunk(**over)) == 0
    assert weights(ha, q=chunk(**over)) == status
    assert ha.lib().ha_cache4_weights_workspace_bytes(cache(), chunk(**over)) == 0


def test_nothing_to_do(ha):
    assert attn(ha, q=chunk(n_seq=0)) == 0 and attn(ha, q=chunk(rows=0)) == 0
    for nothing in (dict(q=chunk(n_seq=0)), dict(q=chunk(rows=0)), dict(q=chunk(max_blocks=0)), dict(c=cache(n_pages=0))):
        assert weights(ha, **nothing) == 0


def test_pointers_strides_and_workspace(ha):
    need = ha.lib().ha_cache4_attn_chunk_workspace_bytes(cache(), chunk())
    assert 0 < need <= 80 << 20
    for i in range(7):
        p = [OK] * 7
        p[i] = None
        assert attn(ha, p) == NULL, i
        p[i] = OK + 2
        assert attn(ha, p) == ALIGN, i
    assert attn(ha, c=struct.pack("4i", 8, 16, 2, 96)) == SHAPE and attn(ha, ws=None) == NULL
    assert attn(ha, nbytes=need - 1) == WORKSPACE and attn(ha, ws=OK + 128, nbytes=need) == WORKSPACE
    for bad, status in (((32, 64), SHAPE), ((1 << 23, 64), SHAPE), ((256, -8), SHAPE), ((260, 64), ALIGN), ((256, 4), ALIGN)):
        assert attn(ha, st=struct.pack("4q", *bad, 256, 64)) == status, bad
    for bad in ((256, 0), (256, 32), (128, 64), (64, 9 * 64)):   # rows of heads that overlap may be read, not written
        assert attn(ha, st=struct.pack("4q", 256, 64, *bad), nbytes=0) == SHAPE, bad
        assert attn(ha, st=struct.pack("4q", 256, 0, 256, 64), nbytes=0) == WORKSPACE
    # tables of few tokens need none; the most that any call needs
    assert ha.lib().ha_cache4_attn_chunk_workspace_bytes(cache(), chunk(max_blocks=4)) == 0
    assert ha.lib().ha_cache4_attn_chunk_workspace_bytes(cache(d=128, page=256), chunk(n_seq=1000, rows=1 << 20, Hq=64, max_blocks=10000)) <= 80 << 20


def test_pointers_strides_and_workspace_of_weights(ha):
    many = chunk(rows=1000)
    need = ha.lib().ha_cache4_weights_workspace_bytes(cache(), many)
    assert 0 < need <= 2 << 20 and ha.lib().ha_cache4_weights_workspace_bytes(cache(), chunk(rows=2)) == 0
    for i in range(7):
        p = [OK] * 7
        p[i] = None
        assert weights(ha, p, q=many) == NULL, i
        p[i] = OK + 2
        assert weights(ha, p, q=many) == ALIGN, i
    assert weights(ha, c=struct.pack("4i", 8, 16, 2, 96)) == SHAPE and weights(ha, q=many, ws=None) == NULL
    assert weights(ha, q=many, nbytes=need - 1) == WORKSPACE and weights(ha, q=many, ws=OK + 128, nbytes=need) == WORKSPACE
    for bad, status in (((32, 64), SHAPE), ((1 << 23, 64), SHAPE), ((256, -8), SHAPE), ((260, 64), ALIGN), ((256, 4), ALIGN)):
        assert weights(ha, q=many, st=struct.pack("2q", *bad)) == status, bad
    assert weights(ha, q=many, st=struct.pack("2q", 64, 0), nbytes=0) == WORKSPACE   # heads that share elements may be read


def test_binding_refuses_what_a_kernel_cannot_take(ha):
    """On tensors of the CPU every call raises before it reaches the library."""
    import torch
    i32 = torch.int32
    Q, cu, lens = torch.zeros(6, 4, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32)
    pages, table = torch.zeros(4, 2, 16 * 68, dtype=torch.uint8), torch.zeros(2, 5, dtype=i32)
    with pytest.raises(ValueError, match="Q has shape"):
        ha.ha_cache4_attn_chunk(Q[0], pages, cu, table, lens, 16)
    with pytest.raises(ValueError, match="cache has shape"):
        ha.ha_cache4_attn_chunk(Q, pages, cu, table, lens, 32)
    with pytest.raises(ValueError, match="n_seq"):
        ha.ha_cache4_attn_chunk(Q, pages, cu[:2], table, lens, 16)
    with pytest.raises(TypeError):
        ha.ha_cache4_attn_chunk(Q.half(), pages, cu, table, lens, 16)
    with pytest.raises(ValueError, match="device tensor"):
        ha.ha_cache4_attn_chunk(Q, pages, cu, table, lens, 16)
    lse, w = torch.zeros(4, 6), ha.alloc_cache4_weights(4, 16, 2, device="cpu")
    assert w.shape == (4, 2, 16) and (w == 0).all()
    with pytest.raises(ValueError, match="n_seq"):
        ha.ha_cache4_weights(Q, pages, cu[:2], table, lens, lse, w, 16)
    with pytest.raises(ValueError, match="device tensor"):
        ha.ha_cache4_weights(Q, pages, cu, table, lens, lse, w, 16)


@pytest.mark.gpu
def test_binding_refuses_tensors_that_do_not_fit(ha):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    i32 = torch.int32
    Q, cu, lens = torch.zeros(6, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=i32, device="cuda"), torch.zeros(2, dtype=i32, device="cuda")
    pages, table = torch.zeros(4, 2, 16 * 68, dtype=torch.uint8, device="cuda"), torch.zeros(2, 5, dtype=i32, device="cuda")
    lse, w = torch.zeros(4, 6, device="cuda"), ha.alloc_cache4_weights(4, 16, 2)
    for call, what in ((lambda: ha.ha_cache4_attn_chunk(Q, pages, cu, table, lens[:1], 16), "lens has shape"),
                       (lambda: ha.ha_cache4_attn_chunk(Q, pages, cu, table, lens, 16, lse=lse.T), "lse has shape"),
                       (lambda: ha.ha_cache4_attn_chunk(Q.cpu(), pages, cu, table, lens, 16), "Q is on"),
                       (lambda: ha.ha_cache4_attn_chunk(Q, pages, cu, table.T.contiguous().T, lens, 16), "contiguous"),
                       (lambda: ha.ha_cache4_weights(Q, pages, cu, table, lens, lse, w[:3], 16), "weights has shape"),
                       (lambda: ha.ha_cache4_weights(Q, pages, cu, table, lens, lse[:3], w, 16), "lse has shape"),
                       (lambda: ha.ha_cache4_weights(Q, pages, cu, table, lens, lse, w.cpu(), 16), "weights is on")):
        with pytest.raises(ValueError, match=what):
            call()
    with pytest.raises(TypeError):
        ha.ha_cache4_weights(Q, pages, cu, table, lens, lse, w.double(), 16)
    with pytest.raises(TypeError):
        ha.ha_cache4_attn_chunk(Q, pages, cu.long(), table, lens, 16)
    with pytest.raises(ha.HyperAttnError):
        ha.ha_cache4_attn_chunk(Q, pages, cu, torch.zeros(2, 500, dtype=i32, device="cuda"), lens, 16, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


def evict(ha, p=None, c=None, e=(2, 100, 4), ws=OK, nbytes=1 << 40):
    return ha.lib().ha_cache4_evict(*(p or [OK + 64 * i for i in range(10)]), c or cache(), struct.pack("3i", *e), ws, nbytes, None)


def test_eviction(ha):
    for e in ((-1, 4, 0), (8193, 4, 0), (2, -1, 0), (2, 4, -1), (2, (1 << 26) + 1, 0), (8192, 1 << 18, 0)):
        assert evict(ha, e=e) == SHAPE, e
        assert ha.lib().ha_cache4_evict_workspace_bytes(cache(), struct.pack("3i", *e)) == 0
    assert evict(ha, c=cache(Hk=1024), e=(1025, 4, 0)) == SHAPE and evict(ha, c=cache(page=24)) == SHAPE
    assert ha.lib().ha_cache4_evict(*[OK + 64 * i for i in range(10)], cache(), None, OK, 1 << 40, None) == NULL
    need = ha.lib().ha_cache4_evict_workspace_bytes(cache(), struct.pack("3i", 2, 100, 4))
    assert 2 * 2 * 1600 * 4 <= need <= 2 * 2 * 1600 * 4 + 512
    for i in range(10):
        p = [OK + 64 * j for j in range(10)]
        p[i] = None
        assert evict(ha, p) == NULL, i
        p[i] = OK + 2
        assert evict(ha, p) == ALIGN, i
    for i, j in ((8, 4), (8, 5), (9, 7)):   # lens_out over lens or keep, free_count_out over free_count
        p = [OK + 64 * x for x in range(10)]
        p[i] = p[j]
        assert evict(ha, p) == SHAPE, (i, j)
    for i in (4, 5):                        # overlapping by one of their two numbers
        for by in (-4, 4):
            p = [OK + 64 * i for i in range(10)]
            p[8] = p[i] + by
            assert evict(ha, p) == SHAPE, (i, by)
    assert evict(ha, ws=None) == NULL and evict(ha, nbytes=need - 1) == WORKSPACE and evict(ha, ws=OK + 128, nbytes=need) == WORKSPACE


def test_binding_of_eviction(ha):
    import torch
    i32 = torch.int32
    pages, w, table = torch.zeros(4, 2, 16 * 68, dtype=torch.uint8), torch.zeros(4, 2, 16), torch.zeros(2, 5, dtype=i32)
    two, free, one = torch.zeros(2, dtype=i32), torch.zeros(4, dtype=i32), torch.zeros(1, dtype=i32)
    with pytest.raises(ValueError, match="block_table has shape"):
        ha.ha_cache4_evict(pages, w, table[0], two, two, free, one, 16)
    with pytest.raises(ValueError, match="cache has shape"):
        ha.ha_cache4_evict(pages, w, table, two, two, free, one, 32)
    with pytest.raises(ValueError, match="device tensor"):
        ha.ha_cache4_evict(pages, w, table, two, two, free, one, 16)


@pytest.mark.gpu
def test_binding_of_eviction_refuses_tensors_that_do_not_fit(ha):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    zeros = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    pages, w, table, two, free, one = zeros(4, 2, 16 * 68, dtype=torch.uint8), ha.alloc_cache4_weights(4, 16, 2), zeros(2, 5), zeros(2), zeros(4), zeros(1)
    for call, what in ((lambda: ha.ha_cache4_evict(pages, w[:2], table, two, two, free, one, 16), "weights has shape"),
                       (lambda: ha.ha_cache4_evict(pages, w, table, two, two[:1], free, one, 16), "keep has shape"),
                       (lambda: ha.ha_cache4_evict(pages, w, table, two, two, free[:3], one, 16), "free_pages has shape"),
                       (lambda: ha.ha_cache4_evict(pages, w, table, two, two, free, one, 16, weights_out=w.cpu()), "weights_out is on")):
        with pytest.raises(ValueError, match=what):
            call()
    with pytest.raises(ha.HyperAttnError):
        ha.ha_cache4_evict(pages, w, table, two, two, free, one, 16, recent=-1)


def test_the_most_workspace_is_what_the_header_says(ha):
    """Over head counts, sequences, rows and tables up to the limits; the number is read from the header, which callers reserve by."""
    import pathlib
    import re
    header = (pathlib.Path(__file__).parent.parent / "include" / "hyperattn.h").read_text()
    for call in ("ha_cache4_attn_chunk", "ha_cache4_weights"):
        stated, = re.findall(call + r"_workspace_bytes\(\) \(at most (\d+) MiB", header)
        need = getattr(ha.lib(), call + "_workspace_bytes")
        most = 0
        for Hk in (1, 2, 8, 64, 300, 512, 513, 768, 944, 945, 1024):
            for group in (1, 2, 16, 17, 129, 1024):
                for n_seq in (1, 4, 64, 4096, 1 << 16):
                    for rows in (1, 4096, 1 << 16, 1 << 22):
                        for blocks in (1, 100, 10000):   # (sizes past a limit have no workspace: 0)
                            most = max([most] + [need(cache(Hk=Hk, d=128, page=page), chunk(n_seq, rows, Hk * group, 0, blocks)) for page in (16, 256)])
        assert 0 < most <= int(stated) << 20, (call, stated, most)


def test_weights_of_a_batch_of_many_rows_go_by_every_sequence(ha):
    """The host knows the batch's rows alone: on average few of a sequence, in all as many as a prompt's, they may be one's.  (The form for few rows alone needs no workspace.)"""
    need = ha.lib().ha_cache4_weights_workspace_bytes
    for n_seq, rows, most in ((512, 511 + 2048, 400), (200, 199 + 600, 1000), (64, 64 * 8, 256)):
        assert need(cache(Hk=8, d=128, page=64), chunk(n_seq, rows, 64, 0, most)) > 0, (n_seq, rows)
    assert need(cache(Hk=8, d=128, page=64), chunk(64, 64, 32, 0, 256)) == 0   # a decoding step
    assert need(cache(Hk=8, d=128, page=64), chunk(1000, 1000, 32, 0, 4)) == 0   # (no sequence of 256 tokens can have more new ones)


def test_numbers_that_eviction_writes_lie_apart_from_those_it_reads(ha):
    """Order of the pointers: 4 lens, 5 keep, 7 free_count, 8 lens_out, 9 free_count_out; two sequences."""
    for i, j, by in ((8, 7, 0), (8, 7, -4), (9, 4, 0), (9, 4, 4), (9, 5, 0), (9, 5, 4), (9, 8, 0), (9, 8, 4)):
        p = [OK + 64 * x for x in range(10)]
        p[i] = p[j] + by
        assert evict(ha, p) == SHAPE, (i, j, by)
