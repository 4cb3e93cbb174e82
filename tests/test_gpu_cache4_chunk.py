"""Attention of chunks of new tokens over the paged 4-bit cache (ha_cache4_attn_chunk) against 64 bits.  Tolerances are those of test_gpu_cache4.py, whose
arithmetic this is: the weights of bf16 queries enter the product in bf16, scores and sums are fp32."""
import numpy as np
import pytest

from ha_testutil import have_gpu
from test_gpu_cache4 import check_attention, dtypes, filled_cache, ha, host, torch  # noqa: F401  (ha and torch: fixtures)

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]
DTYPES = ["bf16", "fp32"]
WIDE = 4096   # tokens of a table in which work is shared out


def chunks64(q, ks, vs, new, pad=0):
    """q [rows, Hq, d] of sum(new) + pad rows -> out, lse, and the bounds' parts absv [rows, Hq, d], weight error [rows, Hq]; rows behind the last sequence: zeros."""
    rows, Hq, d = q.shape
    out, absv, lse, werr = np.zeros(q.shape), np.zeros(q.shape), np.full((Hq, rows), -np.inf), np.zeros((rows, Hq))
    at = 0
    for k, v, n_new in zip(ks, vs, new):
        n, Hk = len(k), k.shape[1]
        sees = n - n_new + 1 + np.arange(n_new)
        live = sees > 0
        if live.any():
            for h in range(Hq):
                kk, vv, x = k[:, h * Hk // Hq], v[:, h * Hk // Hq], q[at:at + n_new, h][live]
                hidden = np.arange(n)[None, :] >= sees[live][:, None]
                S = np.where(hidden, -np.inf, x @ kk.T)
                m = S.max(1, keepdims=True)
                p = np.exp(S - m)
                L = p.sum(1, keepdims=True)
                p /= L
                r = np.arange(at, at + n_new)[live]
                out[r, h], absv[r, h], lse[h, r] = p @ vv, p @ np.abs(vv), (m + np.log(L))[:, 0]
                size = np.where(hidden, 0, np.abs(x) @ np.abs(kk).T).max(1)
                werr[r, h] = 2 * (d * 2.0 ** -24 * size + 2.0 ** -22 * (1 + np.where(hidden, 0, np.abs(S)).max(1)))
        at += n_new
    return out, lse, absv, werr


def starts(torch, new):
    return torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")


def ints(torch, x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def a_case(ha, torch, both, Hq, Hk, d, page, dtype, tokens=0, pad=0, seed=1, scale=1.0):
    rng = np.random.default_rng(seed)
    new, lens = [n for n, _ in both], [n + h for n, h in both]
    cache, table, ks, vs = filled_cache(ha, torch, rng, lens, Hk, d, page, tokens=tokens, scale=scale)
    Q = torch.from_numpy(2 * scale * d ** -0.25 * rng.standard_normal((sum(new) + pad, Hq, d))).to(dtypes(torch, dtype)).cuda()
    return Q, cache, starts(torch, new), table, ints(torch, lens), ks, vs, new, lens


CASES = [
    # (new, held) of every sequence, Hq, Hk, d, page
    ([(1, 0)], 1, 1, 64, 16),
    ([(0, 5)], 2, 1, 128, 16),
    ([(1, 14), (2, 14), (17, 0), (63, 0), (64, 1), (65, 64)], 4, 2, 128, 16),
    ([(0, 0), (3, 297), (0, 9), (1, 0), (40, 0), (129, 200)], 8, 2, 64, 32),
    ([(300, 477)], 8, 4, 64, 16),
    ([(700, 300), (1, 900)], 3, 3, 128, 64),          # a head of keys for each of queries
    ([(50, 300), (7, 0), (33, 60)], 15, 3, 64, 256),   # five query heads a key head: 25 tokens a tile, three rows of it empty
    ([(9, 70), (1, 64)], 14, 2, 128, 128),             # seven
    ([(3, 100), (20, 2)], 260, 2, 64, 16),             # 130 query heads a key head: two runs of 65
    ([(2, 30)], 128, 1, 128, 16),                      # a tile holds one token
    ([(1, 63)] * 70 + [(0, 0)] * 5 + [(30, 170)] * 3, 2, 2, 64, 64),   # more sequences than lanes
]


@pytest.mark.parametrize("tokens", [0, WIDE])   # of the table: small ones have a workgroup per tile, in larger ones the work is shared out
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_chunks(ha, torch, dtype, case, tokens):
    both, Hq, Hk, d, page = CASES[case]
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, both, Hq, Hk, d, page, dtype, tokens, pad=3, seed=case)
    out, lse = torch.full_like(Q, 7.0), torch.full((Hq, Q.shape[0]), 7.0, device="cuda")
    ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page, out=out, lse=lse)
    T = sum(new)
    assert (out[T:] == 7).all() and (lse[:, T:] == 7).all()   # rows of no sequence
    ref, rl, absv, werr = chunks64(host(Q)[:T], ks, vs, new)
    check_attention(host(out)[:T], host(lse)[:, :T], ref, rl, absv, werr, dtype, max(lens))
    o2, l2 = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    assert torch.equal(out[:T], o2[:T]) and torch.equal(lse[:, :T], l2[:, :T])


LONG = [
    ([(200, 20000)], 8, 2, 128, 64),                       # one tile or two, many parts
    ([(1, 30000), (500, 3000), (2, 9000), (0, 700), (1, 1)], 8, 2, 128, 64),
    ([(1500, 2000), (64, 5000)], 4, 4, 64, 32),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", range(len(LONG)))
def test_long_sequences(ha, torch, dtype, case):
    both, Hq, Hk, d, page = LONG[case]
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, both, Hq, Hk, d, page, dtype, seed=20 + case)
    out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    ref, rl, absv, werr = chunks64(host(Q), ks, vs, new)
    check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, max(lens))


@pytest.mark.parametrize("tokens", [0, WIDE])
@pytest.mark.parametrize("dtype", DTYPES)
def test_large_scores(ha, torch, dtype, tokens):
    """Scores of hundreds, in either direction."""
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, [(70, 700), (5, 250)], 4, 2, 64, 16, dtype, tokens, scale=6.0)
    out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, 16)
    ref, rl, absv, werr = chunks64(host(Q), ks, vs, new)
    assert np.abs(rl).max() > 100
    # Channels in which every token of some weight holds a zero: what is left of them are weights below 2^-126 of the largest, which fp32 and bf16 have as zeros (the
    # exponentials are taken against a reference that is no larger than the largest score, their sum is at least 1), and so have parts of fp32 weights, three
    # each: at most 3 n 2^-126 max |v| in all.  (28 of the 19200 elements lie below 6 2^-126.)  Half a step of absv stands for it below.
    absv = absv + 2.0 ** 24 * 3 * max(lens) * 2.0 ** -126 * max(np.abs(v).max() for v in vs)
    check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, max(lens))


@pytest.mark.parametrize("tokens", [0, WIDE])
def test_one_token_each_is_a_decoding_step(ha, torch, tokens):
    """The same queries by ha_cache4_attn: the same to the tolerance of both."""
    lens = [300, 1, 0, 77, 900]
    Q, cache, cu, table, L, ks, vs, new, _ = a_case(ha, torch, [(1, max(n - 1, 0)) for n in lens], 8, 2, 128, 16, "bf16", tokens)
    L, ks, vs = ints(torch, lens), [k[:n] for k, n in zip(ks, lens)], [v[:n] for v, n in zip(vs, lens)]
    out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, 16)
    want, wl = ha.ha_cache4_attn(Q, cache, table, L, 16)
    ref, rl, absv, werr = chunks64(host(Q), ks, vs, new)
    check_attention(host(out), host(lse), ref, rl, absv, werr, "bf16", 900)
    check_attention(host(want), host(wl), ref, rl, absv, werr, "bf16", 900)


@pytest.mark.parametrize("tokens", [0, WIDE])
@pytest.mark.parametrize("dtype", DTYPES)
def test_more_new_tokens_than_the_cache_holds(ha, torch, dtype, tokens):
    """The first rows see nothing: out 0, lse -inf."""
    Q, cache, cu, table, _, ks, vs, new, _ = a_case(ha, torch, [(70, 0), (5, 30), (40, 0), (90, 10)], 4, 2, 64, 16, dtype, tokens)
    lens = [50, 35, 0, 3]
    out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, ints(torch, lens), 16)
    ref, rl, absv, werr = chunks64(host(Q), [k[:n] for k, n in zip(ks, lens)], [v[:n] for v, n in zip(vs, lens)], new)
    assert np.isinf(rl).any()
    check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, 50)


@pytest.mark.parametrize("tokens", [0, WIDE])
def test_pages_that_are_not_there(ha, torch, tokens):
    """Tokens of page numbers outside the cache count as absent; lens past the table as its capacity; negative ones as none."""
    page, Hk = 16, 2
    Q, cache, cu, table, _, ks, vs, new, _ = a_case(ha, torch, [(40, 160), (30, 70), (5, 45)], 4, Hk, 128, page, "bf16", tokens)
    table[0, 2], table[0, 11], table[1, :] = -1, cache.shape[0], 2 ** 31 - 1   # (the second in the middle of the new tokens)
    out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, ints(torch, [200, 100, -3]), page)
    q, k, v = host(Q), ks[0], vs[0]
    there = np.ones(200, bool)
    there[2 * page:3 * page] = there[11 * page:12 * page] = False
    none = np.zeros((0, Hk, 128))
    parts = []
    for i in range(40):   # row by row: what is there of what it sees, its own token last or not
        see = there & (np.arange(200) <= 160 + i)
        parts.append(chunks64(q[i:i + 1], [k[see]], [v[see]], [1]))
    rest = chunks64(q[40:], [none, none], [none, none], [30, 5])
    ref, absv, werr = (np.concatenate([p[j] for p in parts] + [rest[j]]) for j in (0, 2, 3))
    rl = np.concatenate([p[1] for p in parts] + [rest[1]], 1)
    check_attention(host(out), host(lse), ref, rl, absv, werr, "bf16", 200)
    cache.fill_(120)
    full = table[:1].clamp(0, cache.shape[0] - 1)
    a, b = (ha.ha_cache4_attn_chunk(Q[:40], cache, cu[:2], full, ints(torch, [n]), page) for n in (2 ** 30, full.shape[1] * page))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("few", [False, True])   # rows of a sequence: the form for few takes them where there can be several sequences
@pytest.mark.parametrize("tokens", [0, WIDE])
@pytest.mark.parametrize("byte", [252, 253, 254, 255])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_scales_of_other_writers_count_for_the_queries_that_see_them(ha, torch, d, dtype, byte, tokens, few):
    """V of a token in the middle of the new ones with channels 32 ... 63 at a scale of 2^125 ... 2^127 or NaN: for the rows from its own on, and no other.  (Its K is
    0, so that its weight is at most 1.)"""
    from test_gpu_cache4 import STEPS
    from test_gpu_cache4_forms import put_v
    Hq, Hk, page = 4, 2, 16
    both, at = ([(6, 60), (3, 30), (8, 150), (1, 20)], [62, 20, 155, 20]) if few else ([(50, 27), (140, 30)], [27 + 20, 30 + 90])
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, both, Hq, Hk, d, page, dtype, tokens)
    for s, pos in enumerate(at):
        slot = ints(torch, [int(table[s, pos // page]) * page + pos % page])
        k, v = ha.ha_cache4_read(cache, slot, page, dtype=torch.float32)
        ha.ha_cache4_write(torch.zeros_like(k), v, slot, cache, page)
        ks[s][pos] = 0
    want, wl = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    codes = np.arange(d) % 16
    with np.errstate(over="ignore"):
        values = np.full(d, np.nan) if byte == 255 else (STEPS[codes] * 2.0 ** (byte - 127)).astype(np.float32).astype(np.float64)
    bytes_ = cache.cpu().numpy()
    sees = np.zeros((sum(new), Hq), bool)
    for s, pos in enumerate(at):
        scales = np.full(d // 32, 127, np.uint8)
        scales[1] = byte
        put_v(bytes_[int(table[s, pos // page]), 1], page, pos % page, np.where(np.arange(d) // 32 == 1, codes, 2), scales)
        vs[s][pos, 1] = 1.0
        vs[s][pos, 1, 32:64] = np.where(np.isfinite(values[32:64]), values[32:64], 0.0)
        first = sum(new[:s]) + max(pos - both[s][1], 0)
        sees[first:sum(new[:s + 1]), Hq // Hk:] = True
    cache.copy_(torch.from_numpy(bytes_))
    out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    assert torch.equal(lse, wl)
    got = host(out)
    np.testing.assert_array_equal(got[~sees], host(want)[~sees])
    ref, _, absv, werr = chunks64(host(Q), ks, vs, new)
    far = np.zeros(got.shape, bool)
    far[sees] = np.arange(d) // 32 == 1
    far &= ~np.isfinite(values)
    expected = np.broadcast_to(values, got.shape)   # NaN or an infinity
    np.testing.assert_array_equal(got[far], expected[far])
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tol = absv * (half + werr[..., None] + 2.0 ** -24 * max(lens)) + half * np.abs(ref)
    err = np.abs(np.where(far, 0, got - ref))
    assert (err[~far] <= tol[~far]).all(), np.max(err[~far] / tol[~far])


def test_a_nan_query_and_a_nan_key_stay_theirs(ha, torch):
    """A NaN in a row of Q: its own results.  A NaN in a token's K: the rows that see the token.  (Other rows of a wave may be taken against other references.)"""
    Hq, Hk, d, page = 4, 2, 128, 16
    for tokens in (0, WIDE):
        Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, [(60, 100), (20, 5)], Hq, Hk, d, page, "bf16", tokens)
        ref, rl, absv, werr = chunks64(host(Q), ks, vs, new)

        def check(hit):
            got, gl = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
            assert torch.isnan(got[hit]).all() and torch.isnan(gl.T[hit]).all()
            keep = ~hit.cpu().numpy()
            check_attention(host(got)[keep][:, None], host(gl).T[keep][None], ref[keep][:, None], rl.T[keep][None], absv[keep][:, None], werr[keep][:, None], "bf16", max(lens))

        hit = torch.zeros(Q.shape[:2], dtype=torch.bool, device="cuda")
        hit[17, 2] = True
        was = Q[17, 2, 5].clone()
        Q[17, 2, 5] = float("nan")
        check(hit)
        Q[17, 2, 5] = was
        slot = ints(torch, [int(table[0, 130 // page]) * page + 130 % page])
        k, v = ha.ha_cache4_read(cache, slot, page, dtype=torch.float32)
        k[:, 0, 70] = float("nan")
        ha.ha_cache4_write(k, v, slot, cache, page)
        hit[:] = False
        hit[30:60, :Hq // Hk] = True
        check(hit)


def test_strides_streams_and_a_workspace_kept(ha, torch):
    Hq, Hk, d, page = 4, 2, 64, 16
    Q, cache, cu, table, L, *_ = a_case(ha, torch, [(30, 300), (2, 3000)], Hq, Hk, d, page, "bf16")
    ref, rl = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    T = Q.shape[0]
    x = torch.randn(T, Hq + 3, d, device="cuda").bfloat16()
    x[:, 1:1 + Hq] = Q
    ws = torch.empty(ha.ha_cache4_attn_chunk_workspace_bytes(cache, page, 2, T, Hq, table.shape[1]), dtype=torch.uint8, device="cuda")
    ws.fill_(255)
    wide = torch.zeros(T, 2 * Hq, d, device="cuda", dtype=torch.bfloat16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, lse = ha.ha_cache4_attn_chunk(x[:, 1:1 + Hq], cache, cu, table, L, page, out=wide[:, ::2], workspace=ws, stream=s)
    o2, l2 = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page, workspace=ws, stream=s)
    o3, l3 = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page, stream=s)
    s.synchronize()
    assert torch.equal(out, ref) and torch.equal(lse, rl) and (wide[:, 1::2] == 0).all()
    assert torch.equal(o2, ref) and torch.equal(l2, rl) and torch.equal(o3, ref) and torch.equal(l3, rl)


@pytest.mark.parametrize("tokens", [0, WIDE])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,Hq,Hk", [(64, 8, 2), (128, 3, 1), (128, 32, 2)])
def test_few_rows_and_many_side_by_side(ha, torch, d, Hq, Hk, dtype, tokens):
    """Sixteen rows of a key head and one more, many sequences of either, empty ones between."""
    G = Hq // Hk
    few = 16 // G
    both = [(few, 200), (few + 1, 90), (0, 70), (few, 0), (40, 300), (1, 511), (0, 0), (few + 1, 0), (1, 0), (60, 3)] + [(1, n) for n in range(0, 130, 9)]
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, both, Hq, Hk, d, 16, dtype, tokens, pad=2)
    T = sum(new)
    out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, 16)
    ref, rl, absv, werr = chunks64(host(Q)[:T], ks, vs, new)
    check_attention(host(out)[:T], host(lse)[:, :T], ref, rl, absv, werr, dtype, max(lens))


@pytest.mark.parametrize("d", [64, 128])
def test_few_rows_behind_long_sequences(ha, torch, d):
    """Rows whose tokens many workgroups share, in either form: joined by a group of threads, by all of a workgroup, by workgroups of several runs."""
    for both, Hq, Hk in (([(2, 40000), (1, 3000), (1, 60), (3, 9000)], 4, 1), ([(1, 60000)] * 4, 2, 2), ([(30, 50000)], 4, 1), ([(5, 30000), (90, 20000)], 4, 2)):
        Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, both, Hq, Hk, d, 128, "bf16", seed=33)
        out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, 128)
        ref, rl, absv, werr = chunks64(host(Q), ks, vs, new)
        check_attention(host(out), host(lse), ref, rl, absv, werr, "bf16", max(lens))


def test_two_graphs_share_a_workspace(ha, torch):
    """Nothing is kept in it: calls of other sizes, captured one by one and replayed in turn."""
    a, b = (a_case(ha, torch, both, 8, 2, 128, 16, "bf16", seed=s) for both, s in (([(40, 2000), (1, 500), (1, 30), (1, 900)], 1), ([(3, 3000), (100, 1500)], 2)))
    need = max(ha.ha_cache4_attn_chunk_workspace_bytes(x[1], 16, x[3].shape[0], x[0].shape[0], 8, x[3].shape[1]) for x in (a, b))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    want = [ha.ha_cache4_attn_chunk(*x[:5], 16) for x in (a, b)]
    out = [(torch.zeros_like(x[0]), torch.zeros(8, x[0].shape[0], device="cuda")) for x in (a, b)]
    torch.cuda.synchronize()
    graphs = []
    for x, (o, l) in zip((a, b), out):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            ha.ha_cache4_attn_chunk(*x[:5], 16, out=o, lse=l, workspace=ws)
    for which in (0, 1, 1, 0, 1):
        for o, l in out:
            o.zero_(), l.zero_()
        graphs[which].replay()
        torch.cuda.synchronize()
        assert torch.equal(out[which][0], want[which][0]) and torch.equal(out[which][1], want[which][1])


def test_senseless_row_starts_stay_inside(ha, torch):
    """cu_seqlens past the rows, negative, decreasing: nothing outside the outputs is touched."""
    Hq, Hk, d, page = 4, 2, 64, 16
    for tokens in (0, WIDE):
        Q, cache, cu, table, L, *_ = a_case(ha, torch, [(30, 40), (20, 100), (9, 9)], Hq, Hk, d, page, "bf16", tokens)
        T = Q.shape[0]
        room = torch.full((T + 64, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
        for bad in ([0, 1000, 1000, 2 ** 31 - 1], [-5, 20, 10, 59], [40, 30, 20, 10], [-2 ** 31, -1, -1, 5], [0, 59, 0, 59]):
            ha.ha_cache4_attn_chunk(Q, cache, ints(torch, bad), table, L, page, out=room[32:32 + T])
            assert (room[:32] == 7).all() and (room[32 + T:] == 7).all()


def test_large_values_stay_finite(ha, torch):
    """The largest |V| times the tokens just below 2^120 (a scale changes no result but by itself: compared after it is taken out again)."""
    page = 64
    for dtype in DTYPES:
        for tokens in (0, WIDE):
            Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, [(50, 400), (1, 900)], 4, 2, 64, page, dtype, tokens)
            top = max(np.abs(v).max() for v in vs)
            up = 119 - int(np.ceil(np.log2(top * max(lens))))
            scales = cache[:, :, page * 66:]   # V's scale bytes lie last in a block
            scales[scales != 255] += up
            out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
            ref, rl, absv, werr = chunks64(host(Q), ks, vs, new)
            check_attention(host(out) * 2.0 ** -up, host(lse), ref, rl, absv, werr, dtype, max(lens))


def test_an_empty_pool_table_or_batch(ha, torch):
    Q = torch.randn(5, 4, 64, device="cuda").bfloat16()
    cu, lens = ints(torch, [0, 2, 5]), ints(torch, [20, 3])
    for n_pages, blocks in ((0, 4), (3, 0), (0, 0), (0, 1000)):
        out, lse = ha.ha_cache4_attn_chunk(Q, ha.alloc_cache4(n_pages, 16, 2, 64), cu, torch.zeros(2, blocks, dtype=torch.int32, device="cuda"), lens, 16)
        assert (out == 0).all() and (lse == -float("inf")).all()
    cache, table = ha.alloc_cache4(3, 16, 2, 64), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    out, lse = ha.ha_cache4_attn_chunk(Q[:0], cache, cu, table, lens, 16)
    assert out.shape == (0, 4, 64) and lse.shape == (4, 0)
    kept = torch.full_like(Q, 3.0)
    ha.ha_cache4_attn_chunk(Q, cache, cu[:1], table[:0], lens[:0], 16, out=kept)
    assert (kept == 3).all()


def test_a_captured_call_replays(ha, torch):
    """Replayed with other queries, lengths and row starts, with eager calls on the same workspace between: each against the eager result."""
    Hq, Hk, d, page = 8, 2, 128, 16
    Q, cache, cu, table, L, *_ = a_case(ha, torch, [(40, 2000), (1, 500), (20, 30)], Hq, Hk, d, page, "bf16")
    ws = torch.empty(ha.ha_cache4_attn_chunk_workspace_bytes(cache, page, 3, Q.shape[0], Hq, table.shape[1]), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(Q), torch.zeros(Hq, Q.shape[0], device="cuda")
    ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page, out=out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page, out=out, lse=lse, workspace=ws)
    for rows, lens in (([0, 40, 41, 61], [2040, 501, 50]), ([0, 1, 2, 61], [100, 501, 50]), ([0, 0, 60, 61], [7, 480, 1])):
        Q.copy_(torch.randn_like(Q))
        cu.copy_(ints(torch, rows))
        L.copy_(ints(torch, lens))
        want, wl = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page, workspace=ws)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wl)
