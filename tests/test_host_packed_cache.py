"""Refusals of the packed and the cache calls that need no GPU: sizes, types, strides, alignment and workspaces are checked on the host before anything
is enqueued, and the binding checks what a kernel assumes of a tensor.  (The addresses here are never dereferenced.)"""
import os
import struct

import pytest

OK = 0x7F0000000000
NULL, DTYPE, SHAPE, WORKSPACE, ALIGN = -1, -2, -3, -4, -6


@pytest.fixture(scope="module")
def ha():
    import paper_2310_05869_amd as mod
    if not os.path.exists(mod.binding.LIB_PATH):
        from paper_2310_05869_amd import build
        build.build_library()
    mod.lib()
    return mod


def packed(n_seq=3, rows=100, Hq=4, Hk=2, d=64, dtype=0, causal=1):
    return struct.pack("7i", n_seq, rows, Hq, Hk, d, dtype, causal)


def strides(**over):
    s = dict(q=(256, 64), k=(128, 64), v=(128, 64), out=(256, 64), d_out=(256, 64), dq=(256, 64), dk=(128, 64), dv=(128, 64))
    s.update(over)
    return struct.pack("16q", *(x for name in ("q", "k", "v", "out", "d_out", "dq", "dk", "dv") for x in s[name]))


def forward(ha, shape=None, st=None, q=OK, k=OK, v=OK, cu=OK, out=OK, lse=OK, f32=None):
    return ha.lib().exact_attn_packed_forward(q, k, v, cu, out, lse, f32, shape or packed(), st, None)


def backward(ha, shape=None, st=None, ws=OK, nbytes=1 << 40, f32=None, **p):
    a = {**dict(q=OK, k=OK, v=OK, cu=OK, out=OK, lse=OK, d_out=OK, dq=OK, dk=OK, dv=OK), **p}
    return ha.lib().exact_attn_packed_backward(a["q"], a["k"], a["v"], a["cu"], a["out"], f32, a["lse"], a["d_out"], a["dq"], a["dk"], a["dv"],
                                               shape or packed(), st, ws, nbytes, None)


@pytest.mark.parametrize("over,status", [
    (dict(dtype=2), DTYPE), (dict(n_seq=-1), SHAPE), (dict(rows=-1), SHAPE), (dict(Hk=0), SHAPE), (dict(Hq=3), SHAPE), (dict(Hq=2048, Hk=1), SHAPE),
    (dict(d=96), SHAPE), (dict(rows=(1 << 24) + 1), SHAPE), (dict(rows=1 << 24, Hq=16), SHAPE), (dict(n_seq=1 << 21), SHAPE), (dict(rows=0), 0), (dict(n_seq=0), 0)])
def test_packed_shapes(ha, over, status):
    assert forward(ha, packed(**over)) == status
    assert backward(ha, packed(**over)) == status
    assert (ha.lib().exact_attn_packed_backward_workspace_bytes(packed(**over)) == 0) == (status != 0 or over.get("rows") == 0)


def test_packed_pointers_strides_and_workspace(ha):
    assert forward(ha, q=None) == NULL and forward(ha, cu=None) == NULL and forward(ha, lse=None) == NULL
    assert ha.lib().exact_attn_packed_forward(OK, OK, OK, OK, OK, OK, None, None, None, None) == NULL
    assert forward(ha, k=OK + 8) == ALIGN and forward(ha, lse=OK + 2) == ALIGN and forward(ha, cu=OK + 1) == ALIGN and forward(ha, f32=OK + 4) == ALIGN
    assert forward(ha, packed(dtype=1), f32=OK) == DTYPE      # the unrounded copy is for bf16 tensors
    for bad, status in (((32, 64), SHAPE), ((-64, 64), SHAPE), ((1 << 23, 64), SHAPE), ((256, -8), SHAPE), ((260, 64), ALIGN), ((256, 4), ALIGN)):
        assert forward(ha, st=strides(q=bad)) == status, bad
    assert forward(ha, st=strides(out=(256, 0))) == SHAPE     # heads that share elements may be read, not written
    # rows of heads that overlap may not be written: 4 heads over 100 rows, head stride within the row's and across it
    for bad in ((64, 64), (192, 64), (248, 64), (256, 72), (64, 99 * 64)):
        assert forward(ha, st=strides(out=bad)) == SHAPE and backward(ha, st=strides(dq=bad), nbytes=0) == SHAPE, bad
    for good in ((256, 64), (264, 64), (64, 6400), (72, 99 * 72 + 64)):
        assert backward(ha, st=strides(dq=good), nbytes=0) == WORKSPACE, good
    assert backward(ha, packed(rows=1), strides(dq=(64, 64)), nbytes=0) == WORKSPACE and backward(ha, packed(Hq=1, Hk=1), strides(dq=(64, 0)), nbytes=0) == WORKSPACE
    assert backward(ha, st=strides(dk=(128, 0))) == SHAPE and backward(ha, st=strides(d_out=(8, 64))) == SHAPE
    assert backward(ha, d_out=None) == NULL and backward(ha, ws=None) == NULL and backward(ha, dq=OK + 8) == ALIGN
    need = ha.exact_attn_packed_backward_workspace_bytes(100, 3, 4, 2, 64)
    assert need >= 100 * 4 * 4
    assert backward(ha, nbytes=need - 1) == WORKSPACE and backward(ha, ws=OK + 128, nbytes=need) == WORKSPACE
    # rows of delta and, at most, a row of sums per query head and gradient
    for Hq, Hk in ((4, 1), (12, 4), (8, 8)):
        assert ha.exact_attn_packed_backward_workspace_bytes(1000, 7, Hq, Hk, 128) <= 4 * 1000 * Hq * (1 + 2 * 128) + 1024


def cache(n_pages=8, page=16, Hk=2, d=64):
    return struct.pack("4i", n_pages, page, Hk, d)


@pytest.mark.parametrize("over", [dict(page=8), dict(page=48), dict(page=512), dict(d=96), dict(Hk=0), dict(Hk=1025), dict(n_pages=-1), dict(n_pages=1 << 27)])
def test_cache_shapes(ha, over):
    assert ha.lib().ha_cache4_bytes(cache(**over)) == 0
    assert ha.lib().ha_cache4_write(OK, OK, OK, OK, cache(**over), 4, 0, None, None) == SHAPE
    assert ha.lib().ha_cache4_read(OK, OK, OK, OK, cache(**over), 4, 0, None, None) == SHAPE
    q = struct.pack("5i", 2, 1, 4, 0, 8)
    assert ha.lib().ha_cache4_attn(OK, OK, OK, OK, OK, OK, cache(**over), q, None, OK, 1 << 40, None) == SHAPE
    assert ha.lib().ha_cache4_attn_workspace_bytes(cache(**over), q) == 0


def test_cache_bytes_and_rows(ha):
    assert ha.ha_cache4_bytes(10, 64, 8, 128) == 10 * 8 * 64 * 136 and ha.ha_cache4_bytes(3, 16, 1, 64) == 3 * 16 * 68
    write, read = ha.lib().ha_cache4_write, ha.lib().ha_cache4_read
    assert write(OK, OK, OK, OK, cache(), 4, 3, None, None) == DTYPE and write(OK, OK, OK, OK, cache(), -1, 0, None, None) == SHAPE
    assert write(None, OK, OK, OK, cache(), 4, 0, None, None) == NULL and read(None, OK, OK, OK, cache(), 4, 0, None, None) == NULL
    assert write(OK, OK, OK + 2, OK, cache(), 4, 0, None, None) == ALIGN and read(OK + 8, OK, OK, OK, cache(), 4, 0, None, None) == ALIGN
    assert write(OK, OK, OK, OK, cache(), 0, 0, None, None) == 0 and write(OK, OK, OK, None, cache(n_pages=0), 4, 0, None, None) == 0
    assert write(OK, OK, OK, OK, cache(), 4, 0, struct.pack("4q", 128, 64, 32, 64), None) == SHAPE
    assert read(OK, OK, OK, OK, cache(), 4, 0, struct.pack("4q", 128, 0, 128, 64), None) == SHAPE
    assert read(OK, OK, OK, OK, cache(), 4, 0, struct.pack("4q", 64, 64, 128, 64), None) == SHAPE
    assert write(OK, OK, OK, OK, cache(), 1 << 26, 0, None, None) == SHAPE and write(OK, OK, OK, OK, cache(), (1 << 26) + 1, 0, None, None) == SHAPE
    assert read(OK, OK, OK, OK, cache(), 4, 0, struct.pack("4q", 132, 64, 128, 64), None) == ALIGN


@pytest.mark.parametrize("q,status", [((2, 0, 4, 0, 8), SHAPE), ((2, 65, 4, 0, 8), SHAPE), ((2, 1, 3, 0, 8), SHAPE), ((2, 1, 0, 0, 8), SHAPE), ((-1, 1, 4, 0, 8), SHAPE),
                                      ((2, 1, 4, 0, -1), SHAPE), ((1 << 16, 1, 128, 0, 8), SHAPE), ((2, 64, 1024, 0, 8), SHAPE), ((2, 1, 4, 5, 8), DTYPE),
                                      ((1 << 16, 1, 4, 0, 1 << 17), SHAPE), ((2, 1, 4, 0, 0x7FFFFFFF), SHAPE), ((0, 1, 4, 0, 8), 0)])
def test_cache_queries(ha, q, status):
    query = struct.pack("5i", *q)
    assert ha.lib().ha_cache4_attn(OK, OK, OK, OK, OK, OK, cache(), query, None, OK, 1 << 40, None) == status
    assert (ha.lib().ha_cache4_attn_workspace_bytes(cache(), query) == 0) == (status != 0)


def test_cache_attention_pointers_and_workspace(ha):
    query = struct.pack("5i", 2, 1, 4, 0, 8)
    attn = ha.lib().ha_cache4_attn
    need = ha.lib().ha_cache4_attn_workspace_bytes(cache(), query)
    for i in range(6):
        p = [OK] * 6
        p[i] = None
        assert attn(*p, cache(), query, None, OK, need, None) == NULL
        p[i] = OK + 2
        assert attn(*p, cache(), query, None, OK, need, None) == ALIGN
    assert attn(*[OK] * 6, cache(), query, None, OK, need - 1, None) == WORKSPACE
    assert attn(*[OK] * 6, cache(), query, None, OK + 64, need, None) == WORKSPACE
    assert attn(*[OK] * 6, cache(), query, struct.pack("4q", 256, 64, 256, 32), OK, need, None) == SHAPE
    assert attn(*[OK] * 6, cache(), query, struct.pack("4q", 256, 64, 128, 64), OK, need, None) == SHAPE


def test_plan(ha):
    plan = ha.lib().ha_page_plan

    def call(shape, p=None):
        return plan(*(p or [OK + 64 * i for i in range(9)]), struct.pack("5i", *shape), None)

    for shape in ((-1, 4, 16, 8, 4), (8193, 4, 16, 8, 4), (2, -1, 16, 8, 4), (2, 4, 20, 8, 4), (2, 4, 16, -1, 4), (2, 4, 16, 1 << 28, 4), (2, 4, 16, 8, -1),
                  (2, 4, 16, 8, (1 << 26) + 1), (8192, 1 << 18, 16, 8, 4)):
        assert call(shape) == SHAPE, shape
    for i in range(9):
        p = [OK + 64 * j for j in range(9)]
        p[i] = None
        assert call((2, 4, 16, 8, 4), p) == NULL, i
        p[i] = OK + 1
        assert call((2, 4, 16, 8, 4), p) == ALIGN, i
    p = [OK + 64 * j for j in range(9)]
    p[5] = p[0]      # lens_out over lens
    assert call((2, 4, 16, 8, 4), p) == SHAPE
    p = [OK + 64 * j for j in range(9)]
    p[8] = p[4]      # free_count_out over free_count
    assert call((2, 4, 16, 8, 4), p) == SHAPE


def test_binding_refuses_what_a_kernel_cannot_take(ha):
    """On tensors of the CPU, and on a machine without a GPU, every call raises before it reaches the library."""
    import torch
    i32 = torch.int32
    Q, K = torch.zeros(6, 4, 64, dtype=torch.bfloat16), torch.zeros(6, 2, 64, dtype=torch.bfloat16)
    cu, slots = torch.zeros(3, dtype=i32), torch.zeros(6, dtype=i32)
    pages = torch.zeros(4, 2, 16 * 68, dtype=torch.uint8)
    with pytest.raises(ValueError):
        ha.exact_attn_packed_forward(Q[0], K, K, cu)
    with pytest.raises(ValueError):
        ha.exact_attn_packed_forward(Q, K, K, cu[:, None])
    with pytest.raises(TypeError):
        ha.exact_attn_packed_forward(Q.half(), K.half(), K.half(), cu)
    with pytest.raises(TypeError):
        ha.ha_cache4_write(K, K, slots, pages.int(), 16)
    with pytest.raises(ValueError, match="heads"):
        ha.ha_cache4_write(K[:, :1], K[:, :1], slots, pages, 16)
    with pytest.raises(ValueError, match="cache has shape"):
        ha.ha_cache4_write(K, K, slots, pages, 32)
    with pytest.raises(ValueError, match="cache has shape"):
        ha.ha_cache4_read(pages[:, :, :100], slots, 16)
    with pytest.raises(ValueError, match="q_len"):
        ha.ha_cache4_attn(Q, pages, torch.zeros(6, 2, dtype=i32), slots, 16, q_len=2)
    with pytest.raises(ValueError, match="rows or slots"):
        ha.ha_page_plan(slots, slots, torch.zeros(6, 2, dtype=i32), slots, slots[:1], 16)
    with pytest.raises(ha.HyperAttnError):
        ha.alloc_cache4(4, 24, 2, 64, device="cpu")
    assert ha.alloc_cache4(4, 16, 2, 64, device="cpu").shape == pages.shape


@pytest.mark.gpu
def test_binding_refuses_tensors_that_do_not_fit(ha):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    i32 = torch.int32
    Q, K = torch.zeros(6, 4, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(6, 2, 64, device="cuda", dtype=torch.bfloat16)
    cu, slots = torch.zeros(3, dtype=i32, device="cuda"), torch.zeros(6, dtype=i32, device="cuda")
    pages = torch.zeros(4, 2, 16 * 68, dtype=torch.uint8, device="cuda")
    table = torch.zeros(6, 2, dtype=i32, device="cuda")
    for call, what in ((lambda: ha.exact_attn_packed_forward(Q, K, K[:5], cu), "V has shape"),
                       (lambda: ha.exact_attn_packed_forward(Q, K, K.cpu(), cu), "V is on"),
                       (lambda: ha.exact_attn_packed_forward(Q.cpu(), K, K, cu), "device tensor"),
                       (lambda: ha.exact_attn_packed_forward(Q.transpose(1, 2).contiguous().transpose(1, 2), K, K, cu), "last dimension"),
                       (lambda: ha.exact_attn_packed_forward(Q, K, K, cu, lse=torch.zeros(6, 4, device="cuda")), "lse has shape"),
                       (lambda: ha.exact_attn_packed_forward(Q, K, K, torch.zeros(6, dtype=i32, device="cuda")[::2]), "contiguous"),
                       (lambda: ha.ha_cache4_write(K, K, slots[:5], pages, 16), "slots has shape"),
                       (lambda: ha.ha_cache4_attn(Q, pages, table, slots[:5], 16), "lens has shape"),
                       (lambda: ha.ha_cache4_attn(Q, pages.transpose(0, 1).contiguous().transpose(0, 1), table, slots, 16), "contiguous"),
                       (lambda: ha.ha_page_plan(slots, slots, table, slots, slots[:2], 16, rows=4), "free_count has shape")):
        with pytest.raises(ValueError, match=what):
            call()
    with pytest.raises(TypeError):
        ha.exact_attn_packed_forward(Q, K.float(), K, cu)
    with pytest.raises(TypeError):
        ha.ha_cache4_write(K, K, slots.long(), pages, 16)
    with pytest.raises(ha.HyperAttnError):   # rows that share elements
        ha.exact_attn_packed_forward(Q, K, K, cu, out=torch.zeros(1, 4, 64, device="cuda", dtype=torch.bfloat16).expand(6, 4, 64))
    with pytest.raises(ha.HyperAttnError):
        ha.ha_cache4_attn(Q, pages, table, slots, 16, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    # nothing to do: nothing is touched
    ha.ha_cache4_write(K[:0], K[:0], slots[:0], pages, 16)
    out, lse = ha.ha_cache4_attn(Q[:0], pages, table[:0], slots[:0], 16)
    assert out.shape == (0, 4, 64) and lse.shape == (4, 0)
    out, lse = ha.exact_attn_packed_forward(Q[:0], K[:0], K[:0], cu)
    assert out.shape == (0, 4, 64)
    lens, cu2, s2, count = ha.ha_page_plan(slots[:0], slots[:0], table[:0], slots, torch.tensor([3], dtype=i32, device="cuda"), 16, rows=0)
    assert cu2.tolist() == [0] and count.tolist() == [3]
