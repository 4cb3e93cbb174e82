"""What attention weight cached tokens got (ha_cache4_weights) against 64 bits.

Tolerance, from the arithmetic.  The reference takes the lse that the call was given (fp32).  A weight is exp(s - lse), s a sum in fp32 of d exact products, off by at most
e_s = d 2^-24 sum_c |q_c k_c|; the exponent's argument is formed in the unit of the exponential with two roundings (lse, and the difference), relative 2^-24 each of |lse| and of
|s - lse|, and the exponential adds 2^-22: a weight is off by p (e_s + 2^-22 (1 + |s| + |lse|)) (fp32 queries enter with 24 bits: e_s (1 + 1 / d), and their parts
below 2^-126 count as 0).  A token's sum of n weights in fp32 is off by n 2^-24 of it at worst (min(n, 4096): partial sums lie apart), and what was there is added with one
rounding."""
import numpy as np
import pytest

from ha_testutil import have_gpu
from test_gpu_cache4 import ha, host, torch  # noqa: F401  (ha and torch: fixtures)
from test_gpu_cache4_chunk import CASES, DTYPES, LONG, WIDE, a_case, ints

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


def weights64(q, lse, ks, new):
    """Per sequence: sums [len, Hk] and their bounds."""
    sums, bounds, at = [], [], 0
    Hq, d = q.shape[1:]
    for k, n_new in zip(ks, new):
        n, Hk = len(k), k.shape[1]
        got, off = np.zeros((n, Hk)), np.zeros((n, Hk))
        seen = np.arange(n)[None, :] <= (n - n_new + np.arange(n_new))[:, None]
        for x in range(Hq if n and n_new else 0):
            h = x * Hk // Hq
            S, L = q[at:at + n_new, x] @ k[:, h].T, lse[x, at:at + n_new, None]
            with np.errstate(invalid="ignore", over="ignore"):
                p = np.where(seen & (L != -np.inf), np.exp(S - L), 0)
                e = (d + 1) * 2.0 ** -24 * (np.abs(q[at:at + n_new, x]) @ np.abs(k[:, h]).T) + 2.0 ** -22 * (1 + np.abs(S) + np.abs(L))
                got[:, h] += p.sum(0)
                off[:, h] += np.where(p > 0, p * (e + 2.0 ** -24 * min(n_new * Hq // Hk, 4096)), 0).sum(0)
        sums.append(got)
        bounds.append(off)
        at += n_new
    return sums, bounds


def places(table, s, n, page):
    t = np.arange(n)
    return table[s, t // page], t % page


def check(torch, weights, before, q, lse, ks, new, table, page, fresh):
    """All of `weights` after a call that found `before`."""
    sums, bounds = weights64(host(q), host(lse), ks, new)
    got, want, tol, table = host(weights), host(before), np.zeros(before.shape), table.cpu().numpy()
    for s, (w, b, n_new) in enumerate(zip(sums, bounds, new)):
        n = len(w)
        pg, tok = places(table, s, n, page)
        there = (pg >= 0) & (pg < got.shape[0])
        pg, tok, w, b = pg[there], tok[there], w[there], b[there]
        old = np.where((np.arange(n)[there] < n - n_new)[:, None] & (not fresh), want[pg, :, tok], 0)
        want[pg, :, tok] = old + w
        tol[pg, :, tok] = b + 2.0 ** -24 * np.abs(old + w)
    err = np.abs(got - want)
    assert np.isfinite(got).all() and (err <= tol).all(), f"{(err > tol).sum()} of {err.size} off, worst {np.max(err / np.maximum(tol, 1e-300)):.2f} of what is allowed"


@pytest.mark.parametrize("fresh", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(CASES) + len(LONG)))
def test_weights(ha, torch, dtype, case, fresh):
    both, Hq, Hk, d, page = (CASES + LONG)[case]
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, both, Hq, Hk, d, page, dtype, pad=3, seed=case)
    _, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page, lse=torch.full((Hq, Q.shape[0]), 7.0, device="cuda"))
    before = torch.rand(cache.shape[0], Hk, page, device="cuda")
    weights = before.clone()
    assert ha.ha_cache4_weights(Q, cache, cu, table, L, lse, weights, page, fresh=fresh) is weights
    check(torch, weights, before, Q, lse, ks, new, table, page, fresh)
    again = before.clone()
    ha.ha_cache4_weights(Q, cache, cu, table, L, lse, again, page, fresh=fresh)
    assert torch.equal(weights, again)
    # a row's weights add up to 1: all of them to the rows that see something, times the query heads
    if fresh:
        total = sum(host(weights)[places(table.cpu().numpy(), s, n, page)[0], :, np.arange(n) % page].sum() for s, n in enumerate(lens))
        assert abs(total - sum(new) * Hq) <= 1e-3 * max(1, sum(new) * Hq)


@pytest.mark.parametrize("dtype", DTYPES)
def test_more_new_tokens_than_the_cache_holds(ha, torch, dtype):
    """The first rows see nothing and give nothing."""
    page = 16
    Q, cache, cu, table, _, ks, vs, new, _ = a_case(ha, torch, [(70, 0), (5, 30), (40, 0), (90, 300)], 4, 2, 64, page, dtype)
    lens = [50, 35, 0, 3]
    _, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, ints(torch, lens), page)
    assert (lse == -float("inf")).any()
    before = torch.rand(cache.shape[0], 2, page, device="cuda")
    weights = before.clone()
    ha.ha_cache4_weights(Q, cache, cu, table, ints(torch, lens), lse, weights, page)
    check(torch, weights, before, Q, lse, [k[:n] for k, n in zip(ks, lens)], new, table, page, False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_scores(ha, torch, dtype):
    page = 16
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, [(70, 700), (5, 250)], 4, 2, 64, page, dtype, scale=6.0)
    _, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    assert lse.max() > 100
    before = torch.zeros(cache.shape[0], 2, page, device="cuda")
    weights = before.clone()
    ha.ha_cache4_weights(Q, cache, cu, table, L, lse, weights, page)
    sums, bounds = weights64(host(Q), host(lse), ks, new)
    got = host(weights)
    for s, (w, b) in enumerate(zip(sums, bounds)):
        pg, tok = places(table.cpu().numpy(), s, len(w), page)
        # (weights below 2^-126 are 0 in fp32: at most that much a row and head)
        assert (np.abs(got[pg, :, tok] - w) <= b + 2.0 ** -24 * w + 2.0 ** -126 * new[s] * 2).all()


def test_a_decoding_step_by_either_attention(ha, torch):
    """One query each: the lse of ha_cache4_attn serves as well."""
    page, lens = 32, [300, 1, 0, 77, 1900]
    Q, cache, _, table, _, ks, vs, _, _ = a_case(ha, torch, [(1, max(n - 1, 0)) for n in lens], 12, 2, 128, page, "bf16")
    L, cu, ks = ints(torch, lens), torch.arange(6, dtype=torch.int32, device="cuda"), [k[:n] for k, n in zip(ks, lens)]
    _, lse = ha.ha_cache4_attn(Q, cache, table, L, page)
    before = torch.rand(cache.shape[0], 2, page, device="cuda")
    weights = before.clone()
    ha.ha_cache4_weights(Q, cache, cu, table, L, lse, weights, page)
    check(torch, weights, before, Q, lse, ks, [1] * 5, table, page, False)


@pytest.mark.parametrize("fresh", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,Hq,Hk", [(64, 8, 2), (128, 3, 1), (128, 70, 1)])
def test_few_rows_and_many_side_by_side(ha, torch, d, Hq, Hk, dtype, fresh):
    """Up to 64 rows of a key head and more, in one call, and sequences without any."""
    few = max(1, 64 // (Hq // Hk))
    both = [(few, 600), (few + 1, 90), (0, 70), (few, 0), (40, 700), (1, 511), (0, 0), (few + 1, 0), (1, 0), (300, 3)] + [(0, n) for n in range(0, 130, 19)]
    page = 16
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, both, Hq, Hk, d, page, dtype, pad=2)
    _, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    before = torch.rand(cache.shape[0], Hk, page, device="cuda")
    weights = before.clone()
    ha.ha_cache4_weights(Q, cache, cu, table, L, lse, weights, page, fresh=fresh)
    check(torch, weights, before, Q, lse, ks, new, table, page, fresh)


def test_no_rows_at_all(ha, torch):
    """Nothing is added; fresh: what the sequences hold is 0, and nothing else."""
    page = 16
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, [(0, 300), (0, 0), (0, 77)], 4, 2, 64, page, "bf16")
    Q = Q.new_empty(0, 4, 64)   # (numpy's has other strides)
    before = torch.rand(cache.shape[0], 2, page, device="cuda")
    for fresh in (False, True):
        weights = before.clone()
        ha.ha_cache4_weights(Q, cache, cu, table, L, torch.zeros(4, 0, device="cuda"), weights, page, fresh=fresh)
        check(torch, weights, before, Q, torch.zeros(4, 0, device="cuda"), ks, new, table, page, fresh)


def test_the_last_rows_alone(ha, torch):
    """A prompt's last 20 rows decide: their part of Q and lse, as a call of its own."""
    page, Hq = 16, 4
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, [(200, 500)], Hq, 2, 64, page, "bf16")
    _, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    before = torch.rand(cache.shape[0], 2, page, device="cuda")
    weights = before.clone()
    q, l = Q[180:], lse[:, 180:].contiguous()
    ha.ha_cache4_weights(q, cache, ints(torch, [0, 20]), table, L, l, weights, page, fresh=True)
    check(torch, weights, before, q, l, ks, [20], table, page, True)


def test_pages_that_are_not_there_and_nan(ha, torch):
    """Tokens of page numbers outside the cache have no place; NaN of K and of a row's lse go where the formula takes them."""
    page, Hk, Hq = 16, 2, 4
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, [(40, 160), (30, 70)], Hq, Hk, 128, page, "bf16")
    table[0, 2], table[0, 11], table[1, :] = -1, cache.shape[0], 2 ** 31 - 1
    _, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    before = torch.rand(cache.shape[0], Hk, page, device="cuda")
    weights = before.clone()
    ha.ha_cache4_weights(Q, cache, cu, table, L, lse, weights, page)
    check(torch, weights, before, Q, lse, ks, new, table, page, False)
    slot = ints(torch, [int(table[0, 3]) * page + 5])
    k, v = ha.ha_cache4_read(cache, slot, page, dtype=torch.float32)
    k[:, 1, 70] = float("nan")
    ha.ha_cache4_write(k, v, slot, cache, page)
    want = weights.clone()
    want[table[0, 3], 1, 5] = float("nan")
    again = before.clone()
    ha.ha_cache4_weights(Q, cache, cu, table, L, lse, again, page)
    assert torch.equal(torch.nan_to_num(again, nan=-1.0), torch.nan_to_num(want, nan=-1.0))
    lse[3, 20] = float("nan")   # row 20, the second key head: tokens up to 180
    again = before.clone()
    ha.ha_cache4_weights(Q, cache, cu, table, L, lse, again, page)
    pg, tok = places(table.cpu().numpy(), 0, 200, page)
    there = (pg >= 0) & (pg < cache.shape[0])
    got, same = host(again)[pg[there], :, tok[there]], host(want)[pg[there], :, tok[there]]
    late = np.arange(200)[there] > 180
    assert np.isnan(got[~late, 1]).all()
    np.testing.assert_array_equal(got[:, 0], same[:, 0])
    np.testing.assert_array_equal(got[late], same[late])


def test_strides_streams_senseless_starts_and_a_graph(ha, torch):
    page, Hq, Hk, d = 16, 4, 2, 64
    Q, cache, cu, table, L, *_ = a_case(ha, torch, [(150, 300), (2, 3000), (30, 0)], Hq, Hk, d, page, "bf16")
    _, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    T = Q.shape[0]
    ref = ha.ha_cache4_weights(Q, cache, cu, table, L, lse, ha.alloc_cache4_weights(cache.shape[0], page, Hk), page)
    x = torch.randn(T, Hq + 3, d, device="cuda").bfloat16()
    x[:, 1:1 + Hq] = Q
    ws = torch.empty(ha.ha_cache4_weights_workspace_bytes(cache, page, 3, T, Hq, table.shape[1]), dtype=torch.uint8, device="cuda")
    ws.fill_(255)
    s = torch.cuda.Stream()
    a, b = (ha.alloc_cache4_weights(cache.shape[0], page, Hk) for _ in range(2))
    s.wait_stream(torch.cuda.current_stream())
    ha.ha_cache4_weights(x[:, 1:1 + Hq], cache, cu, table, L, lse, a, page, workspace=ws, stream=s)
    ha.ha_cache4_weights(Q, cache, cu, table, L, lse, b, page, stream=s)
    s.synchronize()
    assert torch.equal(a, ref) and torch.equal(b, ref)
    room = torch.zeros(cache.shape[0] + 2, Hk, page, device="cuda")
    for bad in ([0, 1000, 1000, 2 ** 31 - 1], [-5, 20, 10, 59], [40, 30, 20, 10], [-2 ** 31, -1, -1, 5], [0, 182, 0, 182]):
        ha.ha_cache4_weights(Q, cache, ints(torch, bad), table, L, lse, room[1:-1], page)
        assert (room[0] == 0).all() and (room[-1] == 0).all()
    g, w = torch.cuda.CUDAGraph(), torch.zeros_like(ref)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        ha.ha_cache4_weights(Q, cache, cu, table, L, lse, w, page, workspace=ws)
    for rows, lens in (([0, 150, 152, 182], [450, 3002, 30]), ([0, 1, 2, 182], [100, 501, 30]), ([0, 0, 180, 181], [7, 480, 1])):
        cu.copy_(ints(torch, rows))
        L.copy_(ints(torch, lens))
        ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page, lse=lse)
        want = ha.ha_cache4_weights(Q, cache, cu, table, L, lse, ref.clone(), page, workspace=ws)
        w.copy_(ref)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("both", [[(200, 700), (3, 90)], [(300, 2000), (2, 60), (1, 300), (40, 7), (1, 1)], [(9, 300)]])   # many rows, with few beside them, few alone
def test_rows_left_out_give_nothing_whatever_they_hold(ha, torch, both, d, dtype):
    """lse -inf and a row of Q of NaN, or of infinities: as if the row were zeros, in every form and wherever it lies."""
    Hq, Hk, page = 4, 2, 16
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, both, Hq, Hk, d, page, dtype, WIDE, seed=11)
    lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)[1]
    T = Q.shape[0]
    for left_out in ([0], [T - 1], [T // 2, T // 2 + 1], list(range(0, T, 5)), list(range(T // 3, T))):
        for heads in ([1], [0, 1, 2, 3]):
            q, le = Q.clone(), lse.clone()
            for x in heads:
                le[x, left_out] = -float("inf")
                q[left_out, x] = 0
            want = ha.ha_cache4_weights(q, cache, cu, table, L, le, torch.zeros(cache.shape[0], Hk, page, device="cuda"), page, fresh=True)
            check(torch, want, torch.zeros_like(want), q, le, ks, new, table, page, True)
            for value in (float("nan"), float("inf"), -float("inf")):
                for x in heads:
                    q[left_out, x] = value
                got = ha.ha_cache4_weights(q, cache, cu, table, L, le, torch.zeros_like(want), page, fresh=True)
                assert torch.equal(got, want), (left_out[:3], heads, value)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_prompt_among_many_that_decode(ha, torch, dtype):
    """Rows that are few of a sequence on average, most of them one sequence's."""
    Hq, Hk, d, page = 8, 2, 64, 16
    for both in ([(1, n % 50) for n in range(120)] + [(300, 500)] + [(1, n) for n in range(30)], [(1, 70)] * 60 + [(170, 30)] + [(20, 5)]):
        Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, both, Hq, Hk, d, page, dtype, pad=2, seed=12)
        _, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
        before = torch.rand(cache.shape[0], Hk, page, device="cuda")
        weights = before.clone()
        ha.ha_cache4_weights(Q, cache, cu, table, L, lse, weights, page)
        check(torch, weights, before, Q, lse, ks, new, table, page, False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [200, 30])
def test_the_last_rows_alone_without_fresh(ha, torch, rows, dtype):
    """Without the others' rows, the others' tokens count as old: what lies at their places is added to.  With them, their lse -inf, they start from 0."""
    page, Hq, Hk, last = 16, 4, 2, 20
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, [(rows, 500)], Hq, Hk, 64, page, dtype)
    _, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    before = torch.rand(cache.shape[0], Hk, page, device="cuda")
    weights = before.clone()
    q, l = Q[rows - last:], lse[:, rows - last:].contiguous()
    ha.ha_cache4_weights(q, cache, ints(torch, [0, last]), table, L, l, weights, page)
    check(torch, weights, before, q, l, ks, [last], table, page, False)
    lse[:, :rows - last] = -float("inf")
    weights = before.clone()
    ha.ha_cache4_weights(Q, cache, cu, table, L, lse, weights, page)
    check(torch, weights, before, Q, lse, ks, new, table, page, False)
