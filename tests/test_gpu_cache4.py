"""The paged 4-bit cache on the GPU: rows written and read back, attention over pages, the page plan, and a run of them together, each against a
plain implementation in 64 bits written from the format's and the operators' definitions (include/hyperattn.h).

Tolerances, derived from the arithmetic.
Rows: none: a scale is a power of two, so dividing by it and the values themselves are exact, and the rounding to sixteen values has one result.
Attention, |got - ref| per element, with p the softmax weights and absv = sum_j p_j |v_j| of the row:
  bf16 queries: the weights enter the product in bf16, each off by at most half a step, relative 2^-8 (eight significant bits: in [1, 2) the step is
    2^-7), their sum does not: 2^-8 absv.  Scores are sums in fp32 of d
    exact products: off by at most d 2^-24 sum_c |q_c k_c| =: e_s, and the exponential adds 2^-22 (the hardware's 2^x and its argument's rounding, which is
    |s| 2^-23): a weight is off by 2 (e_s + 2^-22 (1 + |s|)) relative, the factor two for the weight and the sum.  The sum of n products in
    fp32: sqrt(n) 2^-24 absv at random, n 2^-24 at worst; 2^-24 min(n, 4096) is allowed.  The result is rounded once: half a step, 2^-8 |ref|.
  fp32 queries: as above without the two roundings to bf16; queries and weights enter with 24 bits (2^-24 each), the result is rounded to 2^-24.
lse: the same error of a weight, absolute, and one rounding of the result."""
import numpy as np
import pytest

from ha_testutil import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]

STEPS = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])


@pytest.fixture(scope="module")
def ha():
    import paper_2310_05869_amd as mod
    mod.lib()
    return mod


@pytest.fixture(scope="module")
def torch():
    import torch as t
    return t


# ---------------------------------------------------------------- the format in 64 bits
def quantised(x):
    """x [..., d] as the cache holds it: values and scale bytes."""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    most = np.abs(g).max(-1, keepdims=True)
    fine = np.isfinite(most)
    m, e = np.frexp(np.where(fine, most, 1.0))
    e = np.clip(e - np.where(m <= 0.75, 3, 2), -125, 125)
    y = np.where(fine, g, 0.0) / 2.0 ** e
    a = np.abs(y)
    edges, even = [.25, .75, 1.25, 1.75, 2.5, 3.5, 5.], [False, True, False, True, False, True, False]
    code = sum(((a >= t) if up else (a > t)).astype(int) for t, up in zip(edges, even))
    v = np.sign(y) * STEPS[code] * 2.0 ** e
    v = np.where(fine, v, np.nan)
    return v.reshape(x.shape), np.where(fine, e + 127, 255).astype(np.uint8)[..., 0]


def page_values(block, page, d):
    """K, V [page, d] of one page's block (bytes) of a head, by the header's description, channel by channel."""
    G = d // 32
    K, V = np.empty((page, d)), np.empty((page, d))

    def scale(byte):
        return np.nan if byte == 255 else 2.0 ** (int(byte) - 127)

    kw = block[:page * d // 2].view(np.uint32).reshape(page, d // 8)
    vw = block[page * d // 2:page * d].view(np.uint32).reshape(page // 4, d // 8, 4)
    ks = block[page * d:page * (d + G)].reshape(page, G)
    vs = block[page * (d + G):].reshape(page, G)
    for t in range(page):
        for c in range(d):
            g, cc = divmod(c, 32)
            K[t, c] = STEPS[(int(kw[t, cc // 8 * G + g]) >> (4 * (cc % 8))) & 15] * scale(ks[t, g])
            m = cc // 2
            word, byte = (m, g) if d == 128 else (m // 2, 2 * g + m % 2)
            V[t, c] = STEPS[(int(vw[t // 4, word, t % 4]) >> (8 * byte + 4 * (c % 2))) & 15] * scale(vs[t, g])
    return K, V


def dtypes(torch, name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def host(t):
    return t.detach().double().cpu().numpy()


# ---------------------------------------------------------------- rows
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,Hk,d,page,n_pages", [(1, 1, 64, 16, 1), (5, 3, 128, 16, 2), (37, 2, 64, 32, 3), (130, 8, 128, 64, 4), (300, 1, 128, 256, 2)])
def test_rows_written_lie_as_described_and_come_back(ha, torch, dtype, rows, Hk, d, page, n_pages):
    rng = np.random.default_rng(rows + d)
    dt = dtypes(torch, dtype)
    x = rng.standard_normal((2, rows, Hk, d)) * 2.0 ** rng.integers(-20, 20, (2, rows, Hk, 1))
    x[0, 0, 0, :32] = 0                       # a group of zeros
    x[1, rows - 1, Hk - 1, 32:64] = np.arange(32) / 8 * np.where(np.arange(32) % 2, 1, -1)   # half-way points
    K, V = (torch.from_numpy(a).to(dt).cuda() for a in x)
    order = rng.permutation(n_pages * page)[:rows].astype(np.int32)
    slots = torch.from_numpy(order).cuda()
    cache = torch.full((n_pages, Hk, page * (d + d // 16)), 0x5A, dtype=torch.uint8, device="cuda")
    ha.ha_cache4_write(K, V, slots, cache, page)
    want_k, want_v = quantised(host(K))[0], quantised(host(V))[0]
    bytes_ = cache.cpu().numpy()
    for h in range(Hk):
        got = [page_values(bytes_[p, h], page, d) for p in range(n_pages)]
        gk, gv = (np.concatenate([g[i] for g in got])[order] for i in range(2))
        np.testing.assert_array_equal(gk, want_k[:, h])
        np.testing.assert_array_equal(gv, want_v[:, h])
    # nothing else was touched: unused slots hold what was there
    untouched = np.setdiff1d(np.arange(n_pages * page), order)
    fresh = page_values(np.full(page * (d + d // 16), 0x5A, np.uint8), page, d)
    for h in range(Hk):
        for i in range(2):   # (every token of a page of these bytes holds the same row)
            kept = np.concatenate([page_values(bytes_[p, h], page, d)[i] for p in range(n_pages)])[untouched]
            np.testing.assert_array_equal(kept, np.broadcast_to(fresh[i][0], kept.shape))
    k2, v2 = ha.ha_cache4_read(cache, slots, page, dtype=dt)
    np.testing.assert_array_equal(host(k2), want_k)
    np.testing.assert_array_equal(host(v2), want_v)


def test_rows_of_extreme_numbers(ha, torch):
    """Infinities and NaN make their 32 channels NaN and no others; the largest numbers stay finite; tiny ones take the least scale."""
    d, page = 64, 16
    x = np.ones((6, 1, d))
    x[0, 0, 3] = np.inf
    x[1, 0, 40] = np.nan
    x[2, 0, 5] = 3.0e38
    x[3, 0, :] = 1e-41
    x[4, 0, :] = -2.0 ** -126
    x[5, 0, 7] = -np.inf
    for dt in (torch.bfloat16, torch.float32):
        K = torch.from_numpy(x).to(dt).cuda()
        slots = torch.arange(6, dtype=torch.int32, device="cuda")
        cache = torch.zeros((1, 1, page * (d + d // 16)), dtype=torch.uint8, device="cuda")
        ha.ha_cache4_write(K, K, slots, cache, page)
        for got in ha.ha_cache4_read(cache, slots, page, dtype=dt):
            np.testing.assert_array_equal(host(got), quantised(host(K))[0])
        assert np.isfinite(host(got)[2]).all() and np.isnan(host(got)[0, 0, :32]).all() and (host(got)[0, 0, 32:] == 1).all()


def test_rows_outside_the_cache_are_left_out(ha, torch):
    d, page, Hk = 128, 16, 2
    K = torch.randn(5, Hk, d, device="cuda").bfloat16()
    cache = torch.zeros((2, Hk, page * (d + d // 16)), dtype=torch.uint8, device="cuda")
    slots = torch.tensor([-1, 3, 32, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    ha.ha_cache4_write(K, K, slots, cache, page)
    k, _ = ha.ha_cache4_read(cache, torch.arange(32, dtype=torch.int32, device="cuda"), page)
    want = np.zeros((32, Hk, d))
    want[3] = quantised(host(K))[0][1]
    np.testing.assert_array_equal(host(k), want)
    k, v = ha.ha_cache4_read(cache, slots, page, dtype=torch.float32)
    assert (host(k)[[0, 2, 3, 4]] == 0).all() and (host(v)[[0, 2, 3, 4]] == 0).all() and (host(k)[1] == want[3]).all()


def test_rows_strided_as_slices_of_a_projection(ha, torch):
    rows, Hq, Hk, d, page = 21, 4, 2, 64, 16
    x = torch.randn(rows, Hq + 2 * Hk, d, device="cuda").bfloat16()
    K, V = x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    slots = torch.arange(rows, dtype=torch.int32, device="cuda")
    a, b = (torch.zeros((2, Hk, page * (d + d // 16)), dtype=torch.uint8, device="cuda") for _ in range(2))
    ha.ha_cache4_write(K, V, slots, a, page)
    ha.ha_cache4_write(K.contiguous(), V.contiguous(), slots, b, page)
    assert torch.equal(a, b)
    back = torch.zeros(rows, Hk, 2, d, device="cuda")   # every second row of d
    ha.ha_cache4_read(a, slots, page, K=back[:, :, 0], V=back[:, :, 1])
    np.testing.assert_array_equal(host(back[:, :, 0]), quantised(host(K))[0])
    np.testing.assert_array_equal(host(back[:, :, 1]), quantised(host(V))[0])


# ---------------------------------------------------------------- attention
def filled_cache(ha, torch, rng, lens, Hk, d, page, scale=1.0, spare=2, tokens=0):
    """A cache with random rows of these lengths, a shuffled block table, and the rows' values [len, Hk, d] per sequence."""
    blocks = [-(-n // page) for n in lens]
    n_pages = sum(blocks) + spare
    order = rng.permutation(n_pages).astype(np.int32)
    most = max(1, max(blocks) if blocks else 1, tokens // page)   # tokens: of a wider table
    table = np.full((len(lens), most), -7, np.int32)
    slots, at = [], 0
    for s, (n, b) in enumerate(zip(lens, blocks)):
        table[s, :b] = order[at:at + b]
        at += b
        t = np.arange(n)
        slots.append(table[s, t // page] * page + t % page)
    slots = np.concatenate(slots).astype(np.int32) if slots else np.zeros(0, np.int32)
    T = slots.size
    K = (scale * rng.standard_normal((T, Hk, d)) * d ** -0.25).astype(np.float32)
    V = rng.standard_normal((T, Hk, d)).astype(np.float32)
    # pages start as garbage with NaN scales: what lies behind a sequence must not count
    cache = torch.full((n_pages, Hk, page * (d + d // 16)), 255, dtype=torch.uint8, device="cuda")
    if T:
        ha.ha_cache4_write(torch.from_numpy(K).cuda(), torch.from_numpy(V).cuda(), torch.from_numpy(slots).cuda(), cache, page)
    kq, vq = quantised(K)[0], quantised(V)[0]
    cut = np.cumsum(lens)[:-1]
    return cache, torch.from_numpy(table).cuda(), np.split(kq, cut), np.split(vq, cut)


def attention64(q, ks, vs, q_len):
    """q [n_seq * q_len, Hq, d] -> out, lse, and the bounds' parts absv [rows, Hq, d], weight error [rows, Hq]."""
    rows, Hq, d = q.shape
    out, absv = np.zeros((rows, Hq, d)), np.zeros((rows, Hq, d))
    lse, werr = np.full((Hq, rows), -np.inf), np.zeros((rows, Hq))
    for s, (k, v) in enumerate(zip(ks, vs)):
        n, Hk = len(k), k.shape[1]
        for i in range(q_len):
            see = n - q_len + 1 + i
            if see <= 0:
                continue
            for h in range(Hq):
                kk, vv = k[:see, h * Hk // Hq], v[:see, h * Hk // Hq]
                x = q[s * q_len + i, h]
                S = kk @ x
                m = S.max()
                p = np.exp(S - m)
                L = p.sum()
                p /= L
                r = s * q_len + i
                out[r, h], absv[r, h], lse[h, r] = p @ vv, p @ np.abs(vv), m + np.log(L)
                werr[r, h] = 2 * (d * 2.0 ** -24 * (np.abs(kk) @ np.abs(x)).max() + 2.0 ** -22 * (1 + np.abs(S).max()))
    return out, lse, absv, werr


def check_attention(got, got_lse, ref, lse, absv, werr, dtype, n):
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tol = absv * (half + werr[..., None] + 2.0 ** -24 * min(max(n, 1), 4096)) + half * np.abs(ref)
    err = np.abs(got - ref)
    assert np.isfinite(got).all() and (err <= tol).all(), f"{(err > tol).sum()} of {err.size} off, worst {np.max(err / np.maximum(tol, 1e-300)):.2f} of what is allowed"
    seen = np.isfinite(lse)
    assert np.array_equal(seen, np.isfinite(got_lse)) and (got_lse[~seen] == -np.inf).all()
    le = np.abs(got_lse[seen] - lse[seen])
    assert (le <= werr.T[seen] + 2.0 ** -22 * (1 + np.abs(lse[seen]))).all()


CASES = [
    # lens, q_len, Hq, Hk, d, page
    ([1], 1, 1, 1, 64, 16),
    ([0], 1, 2, 1, 128, 16),
    ([15, 16, 17, 63, 64, 65], 1, 4, 2, 128, 16),
    ([0, 0, 300, 0, 1, 0, 129, 0], 1, 8, 2, 64, 32),
    ([777], 1, 8, 4, 64, 16),
    ([5000], 1, 16, 1, 128, 64),                 # one tile of rows, filled
    ([2, 700, 1, 3], 4, 6, 2, 128, 128),         # rows that see nothing: fewer tokens than queries
    ([400, 33], 7, 15, 3, 64, 256),              # 35 rows of a key head: three tiles
    ([64] * 70 + [0] * 5 + [200] * 3, 2, 2, 2, 64, 64),   # more sequences than lanes
]


@pytest.mark.parametrize("tokens", [0, 4096])   # of the table: small ones have a workgroup per sequence, larger ones share the tokens out
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_over_pages(ha, torch, dtype, case, tokens):
    lens, q_len, Hq, Hk, d, page = CASES[case]
    rng = np.random.default_rng(100 + case)
    cache, table, ks, vs = filled_cache(ha, torch, rng, lens, Hk, d, page, tokens=tokens)
    Q = torch.from_numpy(2 * d ** -0.25 * rng.standard_normal((len(lens) * q_len, Hq, d))).to(dtypes(torch, dtype)).cuda()
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = ha.ha_cache4_attn(Q, cache, table, L, page, q_len=q_len)
    ref, rl, absv, werr = attention64(host(Q), ks, vs, q_len)
    check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, max(lens))
    o2, l2 = ha.ha_cache4_attn(Q, cache, table, L, page, q_len=q_len)
    assert torch.equal(out, o2) and torch.equal(lse, l2)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64)])
def test_attention_of_many_rows_in_few_and_in_many_parts(ha, torch, dtype, d):
    """More rows than workgroups run at once: a row of few parts is joined by some threads of a workgroup, one of many by all of them."""
    lens, q_len, Hq, Hk, page = [9000, 900, 0, 2, 1500, 64, 300, 1, 700, 0, 1100, 90, 65, 500], 5, 32, 8, 64
    rng = np.random.default_rng(31)
    cache, table, ks, vs = filled_cache(ha, torch, rng, lens, Hk, d, page)
    Q = torch.from_numpy(2 * d ** -0.25 * rng.standard_normal((len(lens) * q_len, Hq, d))).to(dtypes(torch, dtype)).cuda()
    out, lse = ha.ha_cache4_attn(Q, cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), page, q_len=q_len)
    ref, rl, absv, werr = attention64(host(Q), ks, vs, q_len)
    check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, max(lens))


@pytest.mark.parametrize("tokens", [0, 4096])
def test_attention_with_large_scores_and_far_references(ha, torch, tokens):
    """Scores of hundreds, whose largest comes late, in either direction."""
    for dtype in ("bf16", "fp32"):
        rng = np.random.default_rng(8)
        lens, Hq, Hk, d, page = [1000, 260], 4, 2, 64, 16
        cache, table, ks, vs = filled_cache(ha, torch, rng, lens, Hk, d, page, scale=8.0, tokens=tokens)
        Q = torch.from_numpy(8 * d ** -0.25 * rng.standard_normal((2, Hq, d))).to(dtypes(torch, dtype)).cuda()
        out, lse = ha.ha_cache4_attn(Q, cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), page)
        ref, rl, absv, werr = attention64(host(Q), ks, vs, 1)
        assert np.abs(rl).max() > 100
        check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, 1000)


@pytest.mark.parametrize("tokens", [0, 4096])
def test_attention_pages_that_are_not_there(ha, torch, tokens):
    """Tokens of page numbers outside the cache count as absent; lens past the table as its capacity; negative ones as none."""
    rng = np.random.default_rng(5)
    lens, Hq, Hk, d, page = [200, 100, 50], 4, 2, 128, 16
    cache, table, ks, vs = filled_cache(ha, torch, rng, lens, Hk, d, page, tokens=tokens)
    table[0, 2], table[0, 5], table[1, :] = -1, cache.shape[0], 2 ** 31 - 1
    keep = np.ones(200, bool)
    keep[2 * page:3 * page] = keep[5 * page:6 * page] = False
    Q = torch.from_numpy(rng.standard_normal((3, Hq, d))).bfloat16().cuda()
    out, lse = ha.ha_cache4_attn(Q, cache, table, torch.tensor([200, 100, -3], dtype=torch.int32, device="cuda"), page)
    none = np.zeros((0, Hk, d))
    ref, rl, absv, werr = attention64(host(Q), [ks[0][keep], none, none], [vs[0][keep], none, none], 1)
    check_attention(host(out), host(lse), ref, rl, absv, werr, "bf16", 200)
    full = table[:1].clamp(0, cache.shape[0] - 1)
    cache.fill_(120)   # (a NaN, as the unwritten tokens have it, equals nothing)
    a = ha.ha_cache4_attn(Q[:1], cache, full, torch.tensor([2 ** 30], dtype=torch.int32, device="cuda"), page)
    b = ha.ha_cache4_attn(Q[:1], cache, full, torch.tensor([full.shape[1] * page], dtype=torch.int32, device="cuda"), page)
    assert torch.equal(a[1], b[1])


@pytest.mark.parametrize("tokens", [0, 4096])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_nan_token_counts_for_the_queries_that_see_it(ha, torch, dtype, tokens):
    """Five queries a sequence, the third of their tokens with a NaN in channels 32 ... 63 of V: NaN there from that query on, nothing elsewhere."""
    for d in (64, 128):
        rng = np.random.default_rng(9)
        lens, Hq, Hk, page, q_len = [77, 130], 4, 2, 16, 5
        cache, table, ks, vs = filled_cache(ha, torch, rng, lens, Hk, d, page, tokens=tokens)
        Q = torch.from_numpy(rng.standard_normal((2 * q_len, Hq, d))).to(dtypes(torch, dtype)).cuda()
        L = torch.tensor(lens, dtype=torch.int32, device="cuda")
        want, wl = ha.ha_cache4_attn(Q, cache, table, L, page, q_len=q_len)
        for s, n in enumerate(lens):
            pos = n - 3
            slot = torch.tensor([int(table[s, pos // page]) * page + pos % page], dtype=torch.int32, device="cuda")
            k, v = ha.ha_cache4_read(cache, slot, page, dtype=torch.float32)
            v[:, 1, 40] = float("nan")   # the second key head
            ha.ha_cache4_write(k, v, slot, cache, page)
        out, lse = ha.ha_cache4_attn(Q, cache, table, L, page, q_len=q_len)
        hit = torch.zeros_like(out, dtype=torch.bool).view(2, q_len, Hq, d)
        hit[:, 2:, Hq // Hk:, 32:64] = True
        hit = hit.view(out.shape)
        assert torch.isnan(out[hit]).all() and torch.equal(lse, wl)
        # (k went through the cache twice: its values stay; other channels of V too)
        assert torch.equal(out[~hit], want[~hit])


def test_attention_strides_streams_and_a_workspace_kept(ha, torch):
    rng = np.random.default_rng(6)
    lens, Hq, Hk, d, page, q_len = [300, 40], 4, 2, 64, 16, 2
    cache, table, _, _ = filled_cache(ha, torch, rng, lens, Hk, d, page)
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    x = torch.randn(4, Hq + 3, d, device="cuda").bfloat16()
    ref, rl = ha.ha_cache4_attn(x[:, :Hq].contiguous(), cache, table, L, page, q_len=q_len)
    ws = torch.empty(ha.ha_cache4_attn_workspace_bytes(cache, page, 2, q_len, Hq, table.shape[1]), dtype=torch.uint8, device="cuda")
    ws.fill_(255)
    wide = torch.zeros(4, 2 * Hq, d, device="cuda", dtype=torch.bfloat16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, lse = ha.ha_cache4_attn(x[:, :Hq], cache, table, L, page, q_len=q_len, out=wide[:, ::2], workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(out, ref) and torch.equal(lse, rl) and (wide[:, 1::2] == 0).all()
    o2, l2 = ha.ha_cache4_attn(x[:, :Hq], cache, table, L, page, q_len=q_len, stream=s)
    s.synchronize()
    assert torch.equal(o2, ref) and torch.equal(l2, rl)


# ---------------------------------------------------------------- the plan
def plan64(lens, add, table, free, count, page, rows):
    """The header's words, one sequence after the other."""
    n, most = table.shape
    N = len(free)
    table, stack = table.copy(), list(free[:max(0, min(count, N))])
    lens = [min(max(int(x), 0), most * page) for x in lens]
    old = table.copy()
    for s in range(n):
        if add[s] < 0:
            stack += list(old[s, :-(-lens[s] // page)])
    stack = stack[:N]
    out, cu, slots, refused = [], [0], np.full(rows, -1, np.int64), False
    asked = 0
    avail = len(stack)
    for s in range(n):
        more = max(int(add[s]), 0)
        cu.append(cu[-1] + more)
        if add[s] < 0:
            out.append(0)
            continue
        have = -(-lens[s] // page)
        fits = lens[s] + more <= most * page and cu[-1] <= rows
        need = -(-(lens[s] + more) // page) - have if fits else 0
        asked += need
        if not fits or (need and asked > avail):
            out.append(lens[s])
            continue
        for j in range(need):
            table[s, have + j] = stack.pop()
        for i in range(more):
            pos = lens[s] + i
            p = table[s, pos // page]
            slots[cu[-2] + i] = p * page + pos % page if 0 <= p < N else -1
        out.append(lens[s] + more)
    return np.array(out), np.minimum(cu, 2 ** 31 - 1), slots, table, stack


PLANS = [
    # n_seq, max_blocks, page, n_pages, max_add, ends, rows, free share
    (1, 4, 16, 8, 1, 0.0, 1, 1.0),
    (7, 6, 16, 60, 40, 0.3, 300, 1.0),
    (64, 20, 32, 2000, 90, 0.2, 5000, 0.3),      # too few pages
    (300, 8, 16, 4000, 1, 0.5, 300, 1.0),
    (1000, 16, 64, 20000, 300, 0.1, 60000, 1.0),  # too few rows and blocks
    (5000, 4, 256, 30000, 3, 0.3, 12000, 1.0),
]


@pytest.mark.parametrize("case", range(len(PLANS)))
def test_plan(ha, torch, case):
    n, most, page, N, max_add, ends, rows, share = PLANS[case]
    rng = np.random.default_rng(case)
    lens = rng.integers(0, most * page // 2 + 1, n)
    lens[rng.random(n) < 0.2] = 0
    add = np.where(rng.random(n) < ends, -1, rng.integers(0, max_add + 1, n))
    order, table, at = rng.permutation(N).astype(np.int32), np.full((n, most), -1, np.int32), 0
    for s in range(n):
        b = -(-lens[s] // page)
        if at + b > N:
            lens[s], b = 0, 0
        table[s, :b] = order[at:at + b]
        at += b
    left = order[at:at + int((N - at) * share)]
    free = np.full(N, -1, np.int32)
    free[:len(left)] = left
    dev = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()  # noqa: E731
    t, f = dev(table), dev(free)
    got = ha.ha_page_plan(dev(lens), dev(add), t, f, dev([len(left)]), page, rows=rows)
    out, cu, slots, table2, stack = plan64(lens, add, table, free, len(left), page, rows)
    for g, w, name in zip(got, (out, cu, slots, [len(stack)]), ("lens", "cu_seqlens", "slots", "free_count")):
        np.testing.assert_array_equal(g.cpu().numpy(), w, err_msg=name)
    np.testing.assert_array_equal(t.cpu().numpy(), table2)
    np.testing.assert_array_equal(f.cpu().numpy()[:len(stack)], stack)


def test_plan_with_senseless_numbers_stays_inside(ha, torch):
    """Lengths, counts and additions that no program should have: clamped or refused, as documented, and tables keep their size."""
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    big = 2 ** 31 - 1
    table = torch.full((5, 3), -9, dtype=torch.int32, device="cuda")
    free = dev([0, 1, 2, 3])
    lens, cu, slots, count = ha.ha_page_plan(dev([-5, big, 3, 0, 20]), dev([2, 1, big, big, -big]), table, free, dev([99]), 16, rows=10)
    assert lens.tolist() == [2, 48, 3, 0, 0] and cu.tolist() == [0, 2, 3, big, big, big]
    assert count.tolist() == [3] and slots.tolist()[:2] == [48, 49] and slots.tolist()[2:] == [-1] * 8


# ---------------------------------------------------------------- together
def test_a_decoding_run(ha, torch):
    """Prompts admitted, their rows written, then steps of one token with sequences that end and others that take their pages: every step's attention
    against 64 bits over the rows that were written."""
    rng = np.random.default_rng(3)
    Hq, Hk, d, page, n, most, N = 4, 2, 64, 16, 6, 12, 40
    cache = ha.alloc_cache4(N, page, Hk, d)
    cache.fill_(255)
    table = torch.full((n, most), -1, dtype=torch.int32, device="cuda")
    free, count = torch.arange(N, dtype=torch.int32, device="cuda"), torch.tensor([N], dtype=torch.int32, device="cuda")
    lens = torch.zeros(n, dtype=torch.int32, device="cuda")
    held = [np.zeros((0, 2, Hk, d)) for _ in range(n)]
    for step in range(8):
        add = rng.integers(1, 90, n) if step == 0 else np.ones(n, int)
        if step in (3, 5):
            add[rng.integers(0, n)] = -1
        if step in (4, 6):
            add = np.where(np.array([len(h) for h in held]) == 0, 50, add)
        rows = int(np.maximum(add, 0).sum()) + 5    # padded
        lens, cu, slots, count = ha.ha_page_plan(lens, torch.from_numpy(add.astype(np.int32)).cuda(), table, free, count, page, rows=rows)
        kv = torch.from_numpy(rng.standard_normal((rows, 2 * Hk, d))).bfloat16().cuda()
        ha.ha_cache4_write(kv[:, :Hk], kv[:, Hk:], slots, cache, page)
        x, c = host(kv).reshape(rows, 2, Hk, d), cu.tolist()
        for s in range(n):
            held[s] = np.zeros((0, 2, Hk, d)) if add[s] < 0 else np.concatenate([held[s], x[c[s]:c[s + 1]]])
        assert lens.tolist() == [len(h) for h in held]
        used = sum(-(-len(h) // page) for h in held)
        assert count.item() == N - used
        Q = torch.from_numpy(rng.standard_normal((n, Hq, d))).bfloat16().cuda()
        out, lse = ha.ha_cache4_attn(Q, cache, table, lens, page)
        ref, rl, absv, werr = attention64(host(Q), [quantised(h[:, 0])[0] for h in held], [quantised(h[:, 1])[0] for h in held], 1)
        check_attention(host(out), host(lse), ref, rl, absv, werr, "bf16", 200)
    pages = torch.cat([table[s, :-(-len(held[s]) // page)] for s in range(n)] + [free[:count.item()]])
    assert sorted(pages.tolist()) == list(range(N))    # no page lost, none given twice


def test_a_captured_step_replays(ha, torch):
    """Plan, write and attention in one graph, replayed with eager work between, against the eager calls."""
    rng = np.random.default_rng(4)
    Hq, Hk, d, page, n, most, N = 4, 1, 128, 16, 3, 8, 24
    lens0 = torch.tensor([20, 0, 33], dtype=torch.int32, device="cuda")
    add = torch.tensor([1, 4, 1], dtype=torch.int32, device="cuda")
    table0 = torch.full((n, most), -1, dtype=torch.int32, device="cuda")
    table0[0, :2], table0[2, :3] = torch.tensor([0, 1]), torch.tensor([2, 3, 4])
    free0 = torch.cat([torch.arange(5, N), torch.full((5,), -1)]).to(torch.int32).cuda()
    count = torch.tensor([N - 5], dtype=torch.int32, device="cuda")
    start = torch.randint(0, 120, (N, Hk, page * (d + d // 16)), dtype=torch.uint8, device="cuda")
    start[:, :, page * d:] = 120
    kv, Q = torch.randn(6, 2 * Hk, d, device="cuda").bfloat16(), torch.randn(n, Hq, d, device="cuda").bfloat16()
    ws = torch.empty(ha.ha_cache4_attn_workspace_bytes(start, page, n, 1, Hq, most), dtype=torch.uint8, device="cuda")

    def step(table, free, cache):
        lens, cu, slots, left = ha.ha_page_plan(lens0, add, table, free, count, page, rows=6)
        ha.ha_cache4_write(kv[:, :Hk], kv[:, Hk:], slots, cache, page)
        return ha.ha_cache4_attn(Q, cache, table, lens, page, workspace=ws) + (slots, left)

    t, f, c = table0.clone(), free0.clone(), start.clone()
    step(t, f, c)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        t.copy_(table0)
        got = step(t, f, c)
    for trial in range(3):
        kv.copy_(torch.randn_like(kv))
        Q.copy_(torch.randn_like(Q))
        want = step(table0.clone(), free0.clone(), start.clone())
        c.copy_(start)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
