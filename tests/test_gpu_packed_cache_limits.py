"""The packed and the cache calls at the far ends of what include/hyperattn.h allows: offsets past 32 bits, the most queries and heads, empty pools.  References and
tolerances are those of test_gpu_packed.py and test_gpu_cache4.py."""
import numpy as np
import pytest

import test_gpu_cache4 as cached
import test_gpu_packed as packed
from ha_testutil import have_gpu
from test_gpu_packed import ha, host, torch  # noqa: F401  (ha and torch: fixtures)

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]
DTYPES = ["bf16", "fp32"]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page,d", [(16, 64), (256, 128)])
def test_a_cache_of_more_than_4_gib(ha, torch, page, d, dtype):
    """Rows of the last pages and of the first, written, read and attended to."""
    Hk, Hq, dt = 4, 8, cached.dtypes(torch, dtype)
    nbytes = Hk * page * (d + d // 16)
    N = (1 << 32) // nbytes + 40
    cache = ha.alloc_cache4(N, page, Hk, d)
    cache.fill_(255)
    rng = np.random.default_rng(1)
    lens = [5 * page + 3, 1, 3 * page]
    pages = [[N - 1, 0, N - 2, 1, N - 3, N // 2], [N - 4], [2, N - 5, N // 2 + 1]]
    table = np.full((3, 6), -1, np.int32)
    for s, p in enumerate(pages):
        table[s, :len(p)] = p
    slots = np.concatenate([[table[s, t // page] * page + t % page for t in range(n)] for s, n in enumerate(lens)]).astype(np.int32)
    K, V = (torch.from_numpy(rng.standard_normal((len(slots), Hk, d))).to(dt).cuda() for _ in range(2))
    S = torch.from_numpy(slots).cuda()
    ha.ha_cache4_write(K, V, S, cache, page)
    k, v = ha.ha_cache4_read(cache, S, page, dtype=dt)
    kq, vq = cached.quantised(host(K))[0], cached.quantised(host(V))[0]
    np.testing.assert_array_equal(host(k), kq)
    np.testing.assert_array_equal(host(v), vq)
    assert int((cache == 255).sum(dtype=torch.int64)) > cache.numel() - 3 * len(slots) * Hk * (d + d // 16)   # nothing else was touched
    for q_len in (1, 2):
        Q = torch.from_numpy(d ** -0.25 * rng.standard_normal((3 * q_len, Hq, d))).to(dt).cuda()
        out, lse = ha.ha_cache4_attn(Q, cache, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), page, q_len=q_len)
        cut = np.cumsum(lens)[:-1]
        ref, rl, absv, werr = cached.attention64(host(Q), np.split(kq, cut), np.split(vq, cut), q_len)
        cached.check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, max(lens))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,q_len,Hq,Hk,d", [([10, 64, 0, 100, 700, 63, 65], 64, 8, 2, 64), ([5, 1500, 64], 64, 6, 3, 128), ([200], 64, 512, 2, 64), ([90, 3], 16, 1024, 1024, 64)])
@pytest.mark.parametrize("tokens", [0, 8192])
def test_the_most_queries_and_heads(ha, torch, lens, q_len, Hq, Hk, d, dtype, tokens):
    """64 queries a sequence, Hq * q_len of 2^15, 1024 key heads."""
    page, rng = 16, np.random.default_rng(2)
    cache, table, ks, vs = cached.filled_cache(ha, torch, rng, lens, Hk, d, page, tokens=tokens)
    Q = torch.from_numpy(2 * d ** -0.25 * rng.standard_normal((len(lens) * q_len, Hq, d))).to(cached.dtypes(torch, dtype)).cuda()
    out, lse = ha.ha_cache4_attn(Q, cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), page, q_len=q_len)
    ref, rl, absv, werr = cached.attention64(host(Q), ks, vs, q_len)
    cached.check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, max(lens))


def test_an_empty_pool_and_an_empty_table(ha, torch):
    Q = torch.randn(2, 4, 64, device="cuda").bfloat16()
    lens = torch.tensor([20, 3], dtype=torch.int32, device="cuda")
    for n_pages, blocks in ((0, 4), (3, 0), (0, 0), (0, 1000)):
        cache = ha.alloc_cache4(n_pages, 16, 2, 64)
        table = torch.zeros(2, blocks, dtype=torch.int32, device="cuda")
        out, lse = ha.ha_cache4_attn(Q, cache, table, lens, 16)
        assert (out == 0).all() and (lse == -float("inf")).all()
        slots = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
        if n_pages == 0:
            K = Q[:, :2]
            ha.ha_cache4_write(K, K, slots, cache, 16)
            k, v = ha.ha_cache4_read(cache, slots, 16)
            assert (k == 0).all() and (v == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_packed_rows_far_apart(ha, torch, dtype):
    """Row strides of 2^22 elements, head strides past 2^31: slices of large tensors, read and written where they lie."""
    T, Hq, Hk, d, dt = 300, 4, 2, 64, cached.dtypes(torch, dtype)
    lens = [100, 0, 170, 30]
    cu = np.concatenate([[0], np.cumsum(lens)])
    c = torch.from_numpy(cu.astype(np.int32)).cuda()
    rng = np.random.default_rng(3)
    Q, K, V, dO = packed.inputs(torch, rng, T, Hq, Hk, d, dtype, False)
    want = packed.run_all(ha, torch, Q, K, V, dO, c, True, dtype)

    big = torch.zeros((T - 1) * (1 << 22) + 4096, dtype=dt, device="cuda")   # rows of all tensors, 2^22 apart: past 2^30
    far = torch.zeros(3 * (1 << 30) + T * d, dtype=dt, device="cuda")        # heads 2^30 apart: the fourth past 2^31
    by_row = lambda at, H: torch.as_strided(big, (T, H, d), (1 << 22, d, 1), at)   # noqa: E731
    by_head = lambda H: torch.as_strided(far, (T, H, d), (d, 1 << 30, 1), 0)        # noqa: E731
    q, k, v, do = by_row(0, Hq), by_row(256, Hk), by_row(512, Hk), by_row(1024, Hq)
    for to, x in ((q, Q), (k, K), (v, V), (do, dO)):
        to.copy_(x)
    f32 = torch.zeros(T, Hq, d, device="cuda") if dtype == "bf16" else None
    out = by_head(Hq)
    lse = torch.zeros(Hq, T, device="cuda")
    ha.exact_attn_packed_forward(q, k, v, c, causal=True, out=out, lse=lse, out_f32=f32)
    assert torch.equal(out, want["out"]) and torch.equal(lse, want["lse"])
    grads = by_row(2048, Hq), by_row(2560, Hk), by_row(2816, Hk)
    ha.exact_attn_packed_backward(q, k, v, c, out, lse, do, causal=True, out_f32=f32, grads=grads)
    for name, g in zip(("dQ", "dK", "dV"), grads):
        assert torch.equal(g, want[name]), name
    q2, o2 = by_head(Hq), torch.zeros(T, Hq, d, dtype=dt, device="cuda")
    q2.copy_(Q)
    ha.exact_attn_packed_forward(q2, k, v, c, causal=True, out=o2, lse=lse, out_f32=f32)
    assert torch.equal(o2, want["out"])


@pytest.mark.parametrize("dtype", DTYPES)
def test_packed_tensors_of_more_than_2_31_numbers(ha, torch, dtype):
    """2^22 + 77 rows of 8 query heads, d = 64, in sequences of 8 rows and some long ones: the first, the last and some between against 64 bits."""
    T, Hq, Hk, d, dt = (1 << 22) + 77, 8, 1, 64, cached.dtypes(torch, dtype)
    lens = np.full((T - 700) // 8, 8)
    lens[[0, 1000, len(lens) - 2]] = [216, 308, 108]
    cu = np.concatenate([[0], np.cumsum(lens)])
    assert T - 100 < cu[-1] <= T
    torch.manual_seed(4)
    Q, K, V = (torch.randn(T, H, d, device="cuda", dtype=dt).mul_(d ** -0.25) for H in (Hq, Hk, Hk))
    dO = torch.randn(T, Hq, d, device="cuda", dtype=dt)
    c = torch.from_numpy(cu.astype(np.int32)).cuda()
    got = packed.run_all(ha, torch, Q, K, V, dO, c, True, dtype)
    n = len(lens)
    for first, last in ((0, 3), (998, 1003), (n // 2, n // 2 + 4), (n - 4, n)):
        rows = slice(int(cu[first]), int(cu[last]))
        ref, mag = packed.attention64(*(host(t[rows]) for t in (Q, K, V, dO)), cu[first:last + 1] - cu[first], True)
        for name, roundings in (("out", 1), ("lse", 0), ("dV", 1), ("dQ", 2), ("dK", 2)):
            x = got[name][:, rows] if name == "lse" else got[name][rows]
            packed.check(host(x), ref[name], mag[name], dtype, name, roundings)
    assert all((got[name][int(cu[-1]):] == 0).all() for name in ("out", "dQ", "dK", "dV"))


def test_a_plan_of_the_largest_table(ha, torch):
    """8192 sequences of 2^17 blocks (a table of 4 GiB), 2^26 slots, 2^27 - 1 pages: the last sequences' entries and rows too."""
    n, most, page, N, rows = 8192, 1 << 17, 16, (1 << 27) - 1, 1 << 26
    rng = np.random.default_rng(5)
    lens = np.zeros(n, np.int64)
    lens[[0, 17, n - 2, n - 1]] = [1600 * page, 33, most * page - 20, 5000]
    add = np.zeros(n, np.int64)
    add[rng.integers(0, n, 300)] = rng.integers(1, 300, 300)
    add[[0, 17, n - 2, n - 1]] = [-1, 200000, 20, 40000]
    table = torch.full((n, most), -1, dtype=torch.int32, device="cuda")
    at, held = 0, {}
    for s in np.flatnonzero(lens):
        b = -(-int(lens[s]) // page)
        held[s] = np.arange(N - 1 - at, N - 1 - at - b, -1, dtype=np.int32)
        table[int(s), :b] = torch.from_numpy(held[s].copy()).cuda()
        at += b
    left = N - at
    free = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    free[:left] = torch.arange(left, dtype=torch.int32, device="cuda")
    dev = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()  # noqa: E731
    lens_out, cu, slots, count = ha.ha_page_plan(dev(lens), dev(add), table, free, dev([left]), page, rows=rows)
    more = np.maximum(add, 0)
    start = np.concatenate([[0], np.cumsum(more)])
    np.testing.assert_array_equal(cu.cpu().numpy(), start)
    np.testing.assert_array_equal(lens_out.cpu().numpy(), np.where(add < 0, 0, lens + more))
    stack = np.concatenate([np.arange(left, dtype=np.int64), held[0]])   # sequence 0 ended
    need = np.where(add < 0, 0, -(-(lens + more) // page) - -(-lens // page))
    taken = stack[::-1][:need.sum()]
    assert count.item() == len(stack) - need.sum()
    np.testing.assert_array_equal(free[left - 5:count.item()].cpu().numpy(), stack[left - 5:count.item()])
    got = slots[:int(start[-1])].cpu().numpy()
    first = np.concatenate([[0], np.cumsum(need)])
    for s in np.flatnonzero(more):
        have = -(-int(lens[s]) // page)
        new = taken[first[s]:first[s + 1]]
        np.testing.assert_array_equal(table[int(s), have:have + len(new)].cpu().numpy(), new)
        pages = np.concatenate([held.get(s, np.zeros(0, np.int64)), new])
        pos = lens[s] + np.arange(more[s])
        np.testing.assert_array_equal(got[start[s]:start[s + 1]], pages[pos // page] * page + pos % page)
    assert (slots[int(start[-1]):] == -1).all()
