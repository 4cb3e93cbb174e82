"""Chunks over the cache, the weight that tokens get, and eviction at the far ends of what include/hyperattn.h allows: offsets past 32 bits, the most heads and sequences.
References and tolerances are those of test_gpu_cache4_chunk.py, test_gpu_cache4_weights.py and test_gpu_cache4_evict.py."""
import numpy as np
import pytest

import test_gpu_cache4_evict as evicted
import test_gpu_cache4_weights as weighed
from ha_testutil import have_gpu
from test_gpu_cache4 import check_attention, dtypes, ha, host, quantised, torch  # noqa: F401  (ha and torch: fixtures)
from test_gpu_cache4_chunk import DTYPES, WIDE, a_case, chunks64, ints, starts

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page,d", [(16, 64), (256, 128)])
def test_a_cache_of_more_than_4_gib(ha, torch, page, d, dtype):
    """Sequences in the last pages and the first: attention, weights, eviction."""
    Hk, Hq, dt = 4, 8, dtypes(torch, dtype)
    N = (1 << 32) // (Hk * page * (d + d // 16)) + 40
    cache = ha.alloc_cache4(N, page, Hk, d)
    cache.fill_(255)
    rng = np.random.default_rng(1)
    lens, new = [5 * page + 3, 1, 3 * page], [page + 5, 1, 2]
    pages = [[N - 1, 0, N - 2, 1, N - 3, N // 2], [N - 4], [2, N - 5, N // 2 + 1]]
    table = np.full((3, 6), -1, np.int32)
    for s, p in enumerate(pages):
        table[s, :len(p)] = p
    slots = np.concatenate([[table[s, t // page] * page + t % page for t in range(n)] for s, n in enumerate(lens)]).astype(np.int32)
    K, V = (torch.from_numpy(rng.standard_normal((len(slots), Hk, d))).to(dt).cuda() for _ in range(2))
    ha.ha_cache4_write(K, V, torch.from_numpy(slots).cuda(), cache, page)
    cut = np.cumsum(lens)[:-1]
    ks, vs = (np.split(quantised(host(x))[0], cut) for x in (K, V))
    T, L, cu = torch.from_numpy(table).cuda(), ints(torch, lens), starts(torch, new)
    Q = torch.from_numpy(d ** -0.25 * rng.standard_normal((sum(new), Hq, d))).to(dt).cuda()
    out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, T, L, page)
    ref, rl, absv, werr = chunks64(host(Q), ks, vs, new)
    check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, max(lens))
    w = ha.alloc_cache4_weights(N, page, Hk)
    ha.ha_cache4_weights(Q, cache, cu, T, L, lse, w, page)
    sums, bounds = weighed.weights64(host(Q), host(lse), ks, new)
    for s, n in enumerate(lens):
        got = host(w[T[s, torch.arange(n, device="cuda") // page].long(), :, torch.arange(n, device="cuda") % page])
        assert (np.abs(got - sums[s]) <= bounds[s] + 2.0 ** -24 * sums[s]).all()
    assert int((w != 0).sum()) <= sum(lens) * Hk
    keep, recent = [page + 9, 0, 2 * page], 7
    small = np.unique(np.concatenate(pages))   # the pages in use, as a pool of their own for the reference
    where = {p: i for i, p in enumerate(small)}
    own = np.vectorize(lambda p: where.get(p, -1))(table)
    at = torch.from_numpy(small.astype(np.int64)).cuda()
    want_c, want_w, want_lens, freed, defined = evicted.evict64(cache[at].cpu().numpy(), w[at].cpu().numpy(), own, lens, keep, recent, page, d)
    free = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    after, count = ha.ha_cache4_evict(cache, w, T, L, ints(torch, keep), free, ints(torch, [0]), page, recent=recent)
    assert after.tolist() == want_lens and free[:count.item()].tolist() == [int(small[p]) for p in freed]
    got, got_w, rows = cache[at].cpu().numpy(), w[at].cpu().numpy(), np.stack([evicted.row_bytes(page, d, t) for t in range(page)])
    mine = np.zeros(got.shape, bool)
    for p, h, t in zip(*np.nonzero(defined)):
        mine[p, h, rows[t]] = True
    np.testing.assert_array_equal(got[mine], want_c[mine])
    np.testing.assert_array_equal(got_w[defined], want_w[defined])
    untouched = torch.ones(N, dtype=torch.bool, device="cuda")
    untouched[at] = False
    step = 1 << 12
    assert all(bool((cache[i:i + step][untouched[i:i + step]] == 255).all()) for i in range(0, N, step)) and not bool(w[untouched].any())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("both,Hq,Hk,d", [([(3, 60), (0, 5), (1, 30), (20, 1)], 1024, 1, 64), ([(2, 70), (5, 0)], 1024, 1024, 64), ([(30, 300)], 512, 2, 128)])
@pytest.mark.parametrize("tokens", [0, WIDE])
def test_the_most_heads(ha, torch, both, Hq, Hk, d, dtype, tokens):
    """1024 query heads on one key head (tiles of one token's run of heads) and on as many."""
    page = 16
    Q, cache, cu, table, L, ks, vs, new, lens = a_case(ha, torch, both, Hq, Hk, d, page, dtype, tokens, seed=2)
    out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    ref, rl, absv, werr = chunks64(host(Q), ks, vs, new)
    check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, max(lens))
    before = torch.rand(cache.shape[0], Hk, page, device="cuda")
    w = before.clone()
    ha.ha_cache4_weights(Q, cache, cu, table, L, lse, w, page)
    weighed.check(torch, w, before, Q, lse, ks, new, table, page, False)


@pytest.mark.parametrize("blocks", [1, 70])   # of the table: a workgroup per tile, work shared out
def test_the_most_sequences(ha, torch, blocks):
    """2^16 sequences of up to 16 tokens, some without rows."""
    n, Hq, Hk, d, page = 1 << 16, 2, 1, 64, 16
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 17, n)
    new = np.minimum(rng.integers(0, 3, n), lens)
    new[::1000] = np.minimum(lens[::1000], 12)
    x = torch.from_numpy(rng.standard_normal((n * page, 2, d)).astype(np.float32)).cuda()
    cache = ha.alloc_cache4(n, page, Hk, d)
    order = torch.from_numpy(rng.permutation(n).astype(np.int32)).cuda()
    slots = (order[:, None] * page + torch.arange(page, dtype=torch.int32, device="cuda")).reshape(-1)
    ha.ha_cache4_write(x[:, :1], x[:, 1:], slots, cache, page)
    table = torch.full((n, blocks), -1, dtype=torch.int32, device="cuda")
    table[:, 0] = order
    L, cu = ints(torch, lens), starts(torch, new)
    Q = torch.randn(int(new.sum()), Hq, d, device="cuda").bfloat16()
    out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    w = ha.ha_cache4_weights(Q, cache, cu, table, L, lse, torch.full((n, Hk, page), 9.0, device="cuda"), page, fresh=True)
    at, held = cu.tolist(), x.view(n, page, 2, d)
    for a, b in ((0, 300), (n // 2, n // 2 + 300), (n - 300, n)):
        rows = held[a:b].cpu().numpy()
        ks, vs = (quantised(rows[:, :, i:i + 1])[0] for i in range(2))
        ks, vs = [k[:m] for k, m in zip(ks, lens[a:b])], [v[:m] for v, m in zip(vs, lens[a:b])]
        mine = slice(at[a], at[b])
        ref, rl, absv, werr = chunks64(host(Q[mine]), ks, vs, new[a:b])
        check_attention(host(out[mine]), host(lse[:, mine]), ref, rl, absv, werr, "bf16", 16)
        sums, bounds = weighed.weights64(host(Q[mine]), host(lse[:, mine]), ks, new[a:b])
        got = host(w[order[a:b].long()])[:, 0]
        for s in range(b - a):
            m = lens[a + s]
            assert (np.abs(got[s, :m] - sums[s][:, 0]) <= bounds[s][:, 0] + 2.0 ** -24 * sums[s][:, 0]).all() and (got[s, m:] == 9).all()


def test_evictions_of_many_sequences(ha, torch):
    """8192 sequences, of two key heads."""
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 40, 8192)
    keep = np.where(rng.random(8192) < 0.5, rng.integers(-1, 40, 8192), 20)
    evicted.run(ha, torch, rng, [int(x) for x in lens], [int(x) for x in keep], 5, 2, 64, 16, "few values")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [16, 32])
@pytest.mark.parametrize("new", [2, 20, 32])   # 12 rows of the key head (the form for few rows), 120 (weights: the form for few rows), 192
def test_the_longest_sequence(ha, torch, page, new, dtype):
    """A table of the most tokens that a call may hold, nearly all of them in pages that are not there, and a length past it: held tokens and what a tile's start counts
    for on the line of work are more than 2^31 together."""
    Hq, Hk, d = 6, 1, 64
    blocks = (2 ** 31 - 257) // page
    n = blocks * page
    assert n - new + 320 >= 2 ** 31   # (320: what a tile's start counts for)
    rng = np.random.default_rng(5)
    held = [0, 1, blocks // 2, blocks - 4, blocks - 3, blocks - 2, blocks - 1]
    cache = ha.alloc_cache4(len(held), page, Hk, d)
    dt = dtypes(torch, dtype)
    K, V = (torch.from_numpy(rng.standard_normal((len(held) * page, Hk, d))).to(dt).cuda() for _ in range(2))
    ha.ha_cache4_write(K, V, torch.arange(len(held) * page, dtype=torch.int32, device="cuda"), cache, page)
    table = torch.full((1, blocks), -1, dtype=torch.int32, device="cuda")
    table[0, torch.tensor(held, device="cuda")] = torch.arange(len(held), dtype=torch.int32, device="cuda")
    Q = torch.from_numpy(d ** -0.25 * rng.standard_normal((new, Hq, d))).to(dt).cuda()
    L = ints(torch, [2 ** 31 - 1])
    cu = starts(torch, [new])
    out, lse = ha.ha_cache4_attn_chunk(Q, cache, cu, table, L, page)
    ks, vs = (quantised(host(x))[0] for x in (K, V))
    # the pages that are there, one behind the other: the new tokens are the last ones of them too
    ref, rl, absv, werr = chunks64(host(Q), [ks], [vs], [new])
    check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, len(ks))
    w = ha.ha_cache4_weights(Q, cache, cu, table, L, lse, torch.full((len(held), Hk, page), 9.0, device="cuda"), page, fresh=True)
    sums, bounds = weighed.weights64(host(Q), host(lse), [ks], [new])
    got = host(w).transpose(0, 2, 1).reshape(-1, Hk)
    assert (np.abs(got - sums[0]) <= bounds[0] + 2.0 ** -24 * sums[0]).all()
