"""Eviction from the paged 4-bit cache (ha_cache4_evict) against the header's words, one token after the other, and the calls of a serving program that holds its cache to a
budget, together.  Rows are moved as they lie and weights as they are: everything is compared bit for bit."""
import numpy as np
import pytest

from ha_testutil import have_gpu
from test_gpu_cache4 import check_attention, ha, host, quantised, torch  # noqa: F401  (ha and torch: fixtures)
from test_gpu_cache4_chunk import chunks64, ints

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


def row_bytes(page, d, t):
    """Places of token t's bytes in its page's block of a head (include/hyperattn.h): K codes, V codes, K scales, V scales."""
    G = d // 32
    return np.concatenate([t * (d // 2) + np.arange(d // 2),
                           page * d // 2 + t // 4 * (2 * d) + np.repeat(16 * np.arange(d // 8), 4) + t % 4 * 4 + np.tile(np.arange(4), d // 8),
                           page * d + t * G + np.arange(G), page * (d + G) + t * G + np.arange(G)])


def evict64(cache, weights, table, lens, keep, recent, page, d):
    """(cache, weights, lens, freed pages, places that are defined [n_pages, Hk, page]) afterwards."""
    n_pages, Hk, _ = cache.shape
    old, cache, old_w, weights = cache, cache.copy(), weights, weights.copy()
    at = np.stack([row_bytes(page, d, t) for t in range(page)])
    out, freed, defined = [], [], np.ones((n_pages, Hk, page), bool)
    cap = table.shape[1] * page
    for s, n in enumerate(np.clip(lens, 0, cap)):
        n, k = int(n), int(keep[s])
        if k < 0 or k >= n:
            out.append(n)
            continue
        r = min(recent, k)
        out.append(k)
        freed += list(table[s, -(-k // page):-(-n // page)])

        def place(p):
            pg = int(table[s, p // page])
            return (pg, p % page) if 0 <= pg < n_pages else None

        for p in range(k, n):
            if place(p):
                defined[place(p)[0], :, place(p)[1]] = False
        for h in range(Hk):
            w = [old_w[place(p)[0], h, place(p)[1]] if place(p) else np.nan for p in range(n - r)]
            kept = sorted(range(n - r), key=lambda p: (np.isnan(w[p]), 0.0 if np.isnan(w[p]) else -w[p], p))[:k - r]
            stay = set(p for p in kept if p < k - r)
            moves = list(zip(sorted(p for p in kept if p >= k - r), (p for p in range(k - r) if p not in stay))) + [(n - r + i, k - r + i) for i in range(r)]
            for a, b in moves:
                a, b = place(a), place(b)
                if b and not a:
                    defined[b[0], h, b[1]] = False
                if a and b:
                    cache[b[0], h, at[b[1]]] = old[a[0], h, at[a[1]]]
                    weights[b[0], h, b[1]] = old_w[a[0], h, a[1]]
    return cache, weights, out, freed, defined


def a_pool(torch, rng, lens, Hk, d, page, spare=3, wide=0):
    blocks = [-(-max(0, n) // page) for n in lens]
    n_pages, most = sum(blocks) + spare, max(1, max(blocks), wide // page)
    order = rng.permutation(n_pages).astype(np.int32)
    table, at = np.full((len(lens), most), -7, np.int32), 0
    for s, b in enumerate(blocks):
        table[s, :b] = order[at:at + b]
        at += b
    cache = rng.integers(0, 256, (n_pages, Hk, page * (d + d // 16)), dtype=np.uint8)
    free = np.full(n_pages, -1, np.int32)
    free[:spare] = order[at:]
    return cache, table, free


def some_weights(rng, law, shape):
    w = np.exp(2 * rng.standard_normal(shape)).astype(np.float32)
    if law == "alike":
        w[:] = 0.25
    elif law == "few values":
        w = rng.integers(0, 5, shape).astype(np.float32) / 4
    elif law == "zeros":
        w[rng.random(shape) < 0.9] = 0
        w[rng.random(shape) < 0.3] *= -0.0
    elif law == "near":
        w = (1 + rng.integers(0, 40, shape) * 2.0 ** -23).astype(np.float32)
    elif law == "any":
        w = rng.standard_normal(shape).astype(np.float32) * 2.0 ** rng.integers(-120, 120, shape).astype(np.float32)
        for x in (np.nan, -np.nan, np.inf, -np.inf, 1e-42, -0.0, 0.0):
            w[rng.random(shape) < 0.06] = x
    return w


def run(ha, torch, rng, lens, keep, recent, Hk, d, page, law="heavy", apart=False, cache_table=None, wide=0, spare=3):
    cache, table, free = cache_table or a_pool(torch, rng, lens, Hk, d, page, wide=wide, spare=spare)
    w = some_weights(rng, law, (cache.shape[0], Hk, page))
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    C, W, F, T = dev(cache), dev(w), dev(free), dev(table)
    other = torch.full_like(W, -5.0) if apart else None
    count = int((free >= 0).sum())
    out, left = ha.ha_cache4_evict(C, W, T, ints(torch, lens), ints(torch, keep), F, ints(torch, [count]), page, recent=recent, weights_out=other)
    want_c, want_w, want_lens, freed, defined = evict64(cache, w, table, lens, keep, recent, page, d)
    assert out.tolist() == want_lens
    stack = (list(free[:count]) + freed)[:len(free)]
    assert left.tolist() == [len(stack)] and F.tolist()[:len(stack)] == stack and F.tolist()[len(stack):] == list(free[len(stack):])
    assert torch.equal(T, dev(table))
    got, got_w = C.cpu().numpy(), (other if apart else W).cpu().numpy()
    mine = np.zeros(got.shape, bool)
    at = np.stack([row_bytes(page, d, t) for t in range(page)])
    for p, h, t in zip(*np.nonzero(defined)):
        mine[p, h, at[t]] = True
    np.testing.assert_array_equal(got[mine], want_c[mine])
    if apart:
        np.testing.assert_array_equal(W.cpu().numpy().view(np.uint32), w.view(np.uint32))
        moved = defined & ((want_w.view(np.uint32) != w.view(np.uint32)) | (got_w != -5))
        np.testing.assert_array_equal(got_w[moved].view(np.uint32), want_w[moved].view(np.uint32))
    else:
        np.testing.assert_array_equal(got_w[defined].view(np.uint32), want_w[defined].view(np.uint32))
    return C, T, out, want_lens


CASES = [
    # lens, keep, recent, Hk, d, page
    ([1], [0], 0, 1, 64, 16),
    ([1, 2, 5, 0], [1, 1, 4, 0], 1, 2, 128, 16),
    ([15, 16, 17, 33, 300], [14, 15, 16, 16, 100], 0, 3, 128, 16),
    ([100, 100, 100], [-1, 100, 2 ** 31 - 1], 5, 2, 64, 32),            # nothing is let go
    ([300, 257, 90], [0, 20, 60], 500, 2, 64, 16),                      # the last ones alone
    ([300, 257, 90], [299, 256, 1], 64, 2, 128, 64),                    # one token goes; the last ones overlap their places
    ([1000, 31], [128, 30], 64, 4, 64, 128),
    ([5000], [700], 100, 2, 128, 256),
    ([1200] * 3 + [0, 7], [1199, 600, 17, 3, 3], 599, 1, 128, 16),
    ([40] * 130, [9, 33] * 65, 4, 1, 64, 16),                           # many sequences
]


@pytest.mark.parametrize("law", ["heavy", "alike", "few values", "zeros", "near", "any"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_eviction(ha, torch, case, law):
    lens, keep, recent, Hk, d, page = CASES[case]
    run(ha, torch, np.random.default_rng(case), lens, keep, recent, Hk, d, page, law, apart=case % 2 == 1)


@pytest.mark.parametrize("lens,keep,recent", [([9000, 40000], [4000, 4000], 256), ([33500, 12], [33400, 3], 3000), ([20000], [19999], 15000), ([60000], [10], 0),
                                              ([5000, 3000, 2100], [4990, 2999, 500], 300), ([5000, 4000], [513, 3600], 512)])
def test_long_sequences(ha, torch, lens, keep, recent):
    """More weights than a workgroup's registers hold, and more last rows than it moves at a time."""
    for law in ("heavy", "few values"):
        run(ha, torch, np.random.default_rng(3), lens, keep, recent, 1, 64, 64, law)


def test_small_sequences_in_a_wide_table(ha, torch):
    run(ha, torch, np.random.default_rng(4), [70, 0, 500], [30, 0, 499], 10, 2, 128, 16, wide=20000)


def test_pages_that_are_not_there_senseless_lengths_and_a_full_stack(ha, torch):
    rng = np.random.default_rng(5)
    cache, table, free = a_pool(torch, rng, [200, 150, 90, 48], 2, 64, 16)
    table[0, 1], table[0, 7], table[1, :4], table[2, 5] = -1, cache.shape[0], 2 ** 31 - 1, -2 ** 31   # places that rows go to, and come from
    cap = table.shape[1] * 16
    table[3, 3:] = np.arange(cap // 16 - 3) % cache.shape[0]   # (its length is past the table: its capacity; what it has there is let go)
    run(ha, torch, rng, [200, 150, 90, -4], [60, 100, 20, 10], 20, 2, 64, 16, cache_table=(cache, table, free))
    count = ints(torch, [cache.shape[0] + 9])   # more free pages than there are: a full stack stays full
    F, T = torch.arange(cache.shape[0], dtype=torch.int32, device="cuda"), torch.from_numpy(table).cuda()
    W = torch.rand(cache.shape[0], 2, 16, device="cuda")
    out, left = ha.ha_cache4_evict(torch.from_numpy(cache).cuda(), W, T[2:], ints(torch, [90, 2 ** 31 - 1]), ints(torch, [7, 0]), F, count, 16)
    assert out.tolist() == [7, 0] and left.tolist() == [cache.shape[0]] and F.tolist() == list(range(cache.shape[0]))


def test_no_pages_no_table_no_sequences(ha, torch):
    one = ints(torch, [0])
    cache, W = ha.alloc_cache4(0, 16, 2, 64), ha.alloc_cache4_weights(0, 16, 2)
    out, left = ha.ha_cache4_evict(cache, W, torch.zeros(2, 4, dtype=torch.int32, device="cuda"), ints(torch, [64, 3]), ints(torch, [5, 5]), one[:0], one, 16, recent=2)
    assert out.tolist() == [5, 3] and left.tolist() == [0]
    cache, W, F = ha.alloc_cache4(3, 16, 2, 64), ha.alloc_cache4_weights(3, 16, 2), ints(torch, [2, 0, 0])
    out, left = ha.ha_cache4_evict(cache, W, torch.zeros(2, 0, dtype=torch.int32, device="cuda"), ints(torch, [64, 3]), ints(torch, [5, 5]), F, ints(torch, [1]), 16)
    assert out.tolist() == [0, 0] and left.tolist() == [1]
    out, left = ha.ha_cache4_evict(cache, W, torch.zeros(0, 4, dtype=torch.int32, device="cuda"), one[:0], one[:0], F, ints(torch, [1]), 16)
    assert out.shape == (0,) and left.tolist() == [1] and F.tolist() == [2, 0, 0]


def test_no_sequences_of_a_long_table(ha, torch):
    cache, W, F, none = ha.alloc_cache4(3, 16, 2, 64), ha.alloc_cache4_weights(3, 16, 2), ints(torch, [2, 0, 0]), ints(torch, [])
    out, left = ha.ha_cache4_evict(cache, W, torch.zeros(0, 5000, dtype=torch.int32, device="cuda"), none, none, F, ints(torch, [1]), 16, recent=3)
    assert out.shape == (0,) and left.tolist() == [1] and F.tolist() == [2, 0, 0]


@pytest.mark.parametrize("n,blocks,keep", [(256, 300, 100), (256, 1200, 9000), (40, 1200, 9000)])
def test_pages_that_sequences_share_against_the_rule(ha, torch, n, blocks, keep):
    """Rows may be any, but nothing beside these pages is written, and the lengths and the stack are those of the rule."""
    page, N = 16, blocks + 50
    rng = np.random.default_rng(8)
    table = torch.from_numpy(np.stack([rng.permutation(blocks) for _ in range(n)]).astype(np.int32)).cuda()
    cache = torch.from_numpy(rng.integers(0, 256, (N, 1, page * 68), dtype=np.uint8)).cuda()
    W = torch.rand(N, 1, page, device="cuda")
    before, was = cache.clone(), W.clone()
    need = ha.ha_cache4_evict_workspace_bytes(cache, page, n, blocks)
    ws = torch.full((need + 4096,), 7, dtype=torch.uint8, device="cuda")
    F = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    out, left = ha.ha_cache4_evict(cache, W, table, ints(torch, [blocks * page - 3] * n), ints(torch, [keep] * n), F, ints(torch, [0]), page, recent=30, workspace=ws[:need])
    assert out.tolist() == [keep] * n and left.tolist() == [min(N, n * (blocks - -(-keep // page)))]
    assert torch.equal(cache[blocks:], before[blocks:]) and torch.equal(W[blocks:], was[blocks:]) and bool((ws[need:] == 7).all())


def test_streams_a_workspace_kept_and_a_graph(ha, torch):
    rng = np.random.default_rng(6)
    lens, Hk, d, page = [900, 300, 77], 2, 128, 16
    cache, table, free = a_pool(torch, rng, lens, Hk, d, page)
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    W0, C0, F0, T = dev(some_weights(rng, "heavy", (cache.shape[0], Hk, page))), dev(cache), dev(free), dev(table)
    L, K, count = ints(torch, lens), ints(torch, [200, 299, 20]), ints(torch, [3])
    ws = torch.empty(ha.ha_cache4_evict_workspace_bytes(C0, page, 3, table.shape[1]), dtype=torch.uint8, device="cuda")
    ws.fill_(255)

    def call(stream=None, workspace=None, C=None, W=None, F=None):
        C, W, F = C0.clone() if C is None else C, W0.clone() if W is None else W, F0.clone() if F is None else F
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        return (C, W, F) + ha.ha_cache4_evict(C, W, T, L, K, F, count, page, recent=50, workspace=workspace, stream=stream)

    s = torch.cuda.Stream()
    want, a, b = call(), call(s, ws), call(s)
    s.synchronize()
    for x, y, z in zip(want, a, b):
        assert torch.equal(x, y) and torch.equal(x, z)
    C, W, F = C0.clone(), W0.clone(), F0.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = call(None, ws, C, W, F)
    for now, keep in ((lens, [200, 299, 20]), ([850, 300, 5], [849, 0, 3]), ([900, 11, 77], [-1, 10, 76])):
        L.copy_(ints(torch, now))
        K.copy_(ints(torch, keep))
        W0.copy_(torch.rand_like(W0))
        want = call(None, ws)
        C.copy_(C0), W.copy_(W0), F.copy_(F0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("d", [64, 128])
def test_a_serving_run_within_a_budget(ha, torch, d):
    """Prompts come in pieces beside sequences that decode; after every step's attention the weight that tokens got is added up, and sequences past their budget are cut.  Against
    a model of the cache that holds rows and weights by place: attention and weights in 64 bits, evictions exactly (from the weights that the device found)."""
    rng = np.random.default_rng(7)
    Hq, Hk, page, n, most, N, budget, recent = 6, 2, 16, 5, 20, 60, 70, 24
    cache, weights = ha.alloc_cache4(N, page, Hk, d), ha.alloc_cache4_weights(N, page, Hk)
    cache.fill_(255)
    weights.fill_(float("nan"))
    table = torch.full((n, most), -1, dtype=torch.int32, device="cuda")
    free, count = torch.arange(N, dtype=torch.int32, device="cuda"), ints(torch, [N])
    lens, keep = ints(torch, [0] * n), ints(torch, [budget] * (n - 1) + [-1])
    held = [np.zeros((0, 2, Hk, d)) for _ in range(n)]
    prompts = [150, 1, 64, 0, 90]
    for step in range(9):
        add = [min(40, p) if p > 0 else 1 for p in prompts]
        if step == 6:
            add[2] = -1
        if step == 7:
            prompts[2], add[2] = 33, 33
        prompts = [max(0, p - 40) for p in prompts]
        rows = sum(max(a, 0) for a in add) + 3
        lens, cu, slots, count = ha.ha_page_plan(lens, ints(torch, add), table, free, count, page, rows=rows)
        qkv = torch.from_numpy(rng.standard_normal((rows, Hq + 2 * Hk, d)) * d ** -0.25).bfloat16().cuda()
        Q, K, V = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
        ha.ha_cache4_write(K, V, slots, cache, page)
        x, c = host(qkv[:, Hq:]).reshape(rows, 2, Hk, d), cu.tolist()
        for s in range(n):
            held[s] = held[s][:0] if add[s] < 0 else np.concatenate([held[s], quantised(x[c[s]:c[s + 1]].astype(np.float32))[0]])
        assert lens.tolist() == [len(h) for h in held]
        new = [max(a, 0) for a in add]
        out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, lens, page)
        ref, rl, absv, werr = chunks64(host(Q)[:c[-1]], [h[:, 0] for h in held], [h[:, 1] for h in held], new)
        check_attention(host(out)[:c[-1]], host(lse)[:, :c[-1]], ref, rl, absv, werr, "bf16", 300)
        ha.ha_cache4_weights(Q, cache, cu, table, lens, lse, weights, page)
        w, t = weights.cpu().numpy(), table.cpu().numpy()
        after, count = ha.ha_cache4_evict(cache, weights, table, lens, keep, free, count, page, recent=recent)
        for s in range(n):
            have, k = len(held[s]), len(held[s]) if s == n - 1 else min(budget, len(held[s]))
            if k < have:
                r = min(recent, k)
                moved = held[s][:k].copy()
                p = np.arange(have)
                for h in range(Hk):
                    mine = w[t[s, p // page], h, p % page]
                    assert np.isfinite(mine).all() and (mine >= 0).all()
                    kept = sorted(range(have - r), key=lambda i: (-mine[i], i))[:k - r]
                    gaps = [i for i in range(k - r) if i not in kept]
                    for a, b in list(zip(sorted(i for i in kept if i >= k - r), gaps)) + [(have - r + i, k - r + i) for i in range(r)]:
                        moved[b, :, h] = held[s][a, :, h]
                held[s] = moved
        lens = after
        assert lens.tolist() == [len(h) for h in held]
        assert count.item() == N - sum(-(-len(h) // page) for h in held)
        k, v = zip(*(ha.ha_cache4_read(cache, table[s, torch.arange(len(h), device="cuda") // page] * page + torch.arange(len(h), dtype=torch.int32, device="cuda") % page,
                                       page, dtype=torch.float32) for s, h in enumerate(held)))
        for s, h in enumerate(held):
            np.testing.assert_array_equal(host(k[s]), h[:, 0])
            np.testing.assert_array_equal(host(v[s]), h[:, 1])
    pages = torch.cat([table[s, :-(-len(held[s]) // page)] for s in range(n)] + [free[:count.item()]])
    assert sorted(pages.tolist()) == list(range(N))    # no page lost, none given twice


def test_layers_that_share_a_table(ha, torch):
    """Each cut from the same lengths and the same stack: every layer keeps its own heaviest tokens, and no page lies on the stack twice."""
    rng = np.random.default_rng(9)
    lens, keep, recent, Hk, d, page = [500, 90, 33, 0, 257], [200, 90, 7, 3, 31], 16, 2, 64, 16
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    _, table, free = a_pool(torch, rng, lens, Hk, d, page)
    n_pages, spare = len(free), int((free >= 0).sum())
    T, L, K, F, count = dev(table), ints(torch, lens), ints(torch, keep), dev(free), ints(torch, [spare])
    results = []
    for layer in range(3):
        cache = rng.integers(0, 256, (n_pages, Hk, page * (d + d // 16)), dtype=np.uint8)
        w = some_weights(rng, "heavy", (n_pages, Hk, page))
        C, W = dev(cache), dev(w)
        results.append(ha.ha_cache4_evict(C, W, T, L, K, F, count, page, recent=recent))
        want_c, want_w, want_lens, freed, defined = evict64(cache, w, table, lens, keep, recent, page, d)
        got, got_w, at = C.cpu().numpy(), W.cpu().numpy(), np.stack([row_bytes(page, d, t) for t in range(page)])
        for p, h, t in zip(*np.nonzero(defined)):
            np.testing.assert_array_equal(got[p, h, at[t]], want_c[p, h, at[t]])
        np.testing.assert_array_equal(got_w[defined], want_w[defined])
        assert results[-1][0].tolist() == want_lens and L.tolist() == lens and count.tolist() == [spare]
    after, left = results[-1]
    held = [int(p) for s, n in enumerate(after.tolist()) for p in table[s, :-(-n // page)]]
    assert left.tolist() == [spare + len(freed)] and sorted(held + F[:left.item()].tolist()) == list(range(n_pages))
    # the next step's pages are nobody else's
    add = ints(torch, [40, 5, 1, 60, 16])
    lens2, *_ = ha.ha_page_plan(after, add, T, F, left, page, rows=122)
    t = T.tolist()
    pages = [p for s, n in enumerate(lens2.tolist()) for p in t[s][:-(-n // page)]]
    assert len(set(pages)) == len(pages) and set(pages) <= set(range(n_pages))
