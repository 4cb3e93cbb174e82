"""Attention over pages where test_gpu_cache4.py does not go: scale bytes that only other writers give, and every form of the launch.  Reference
and tolerances are that file's."""
import numpy as np
import pytest

from ha_testutil import have_gpu
from test_gpu_cache4 import STEPS, attention64, check_attention, dtypes, filled_cache, ha, host, torch  # noqa: F401  (ha and torch: fixtures)

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


def v_places(d):
    """Of channel c of a V row: its word among the row's d / 8, and its nibble there (include/hyperattn.h)."""
    c = np.arange(d)
    g, m, e = c // 32, c % 32 // 2, c % 2
    return (m, 2 * g + e) if d == 128 else (m // 2, 2 * (2 * g + m % 2) + e)


def put_v(block, page, t, codes, scales):
    """Token t of a page's block of a head (bytes, changed in place): V as these codes and scale bytes."""
    d = len(codes)
    words = block[page * d // 2:page * d].view(np.uint32).reshape(page // 4, d // 8, 4)
    row = np.zeros(d // 8, np.uint64)
    for w, nib, code in zip(*v_places(d), codes):
        row[w] |= np.uint64(int(code) << (4 * int(nib)))
    words[t // 4, :, t % 4] = row.astype(np.uint32)
    block[page * (d + d // 32):].reshape(page, d // 32)[t] = scales


@pytest.mark.parametrize("tokens", [0, 4096])
@pytest.mark.parametrize("byte", [252, 253, 254])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_scales_count_for_the_queries_that_see_them(ha, torch, d, dtype, byte, tokens):
    """Five queries a sequence, the third of their tokens with channels 32 ... 63 of V at a scale of 2^125 ... 2^127, where code times scale can be past the
    largest number: values times weights from that query on, nothing before it.  (The token's K is 0, its score no larger than the largest: a weight of
    at most 1, so that what is finite stays finite.)"""
    rng = np.random.default_rng(19)
    lens, Hq, Hk, page, q_len = [77, 130], 4, 2, 16, 5
    cache, table, ks, vs = filled_cache(ha, torch, rng, lens, Hk, d, page, tokens=tokens)
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    Q = torch.from_numpy(rng.standard_normal((2 * q_len, Hq, d))).to(dtypes(torch, dtype)).cuda()
    for s, n in enumerate(lens):   # K of the token: zeros; its V as it is
        pos = n - 3
        slot = torch.tensor([int(table[s, pos // page]) * page + pos % page], dtype=torch.int32, device="cuda")
        k, v = ha.ha_cache4_read(cache, slot, page, dtype=torch.float32)
        ha.ha_cache4_write(torch.zeros_like(k), v, slot, cache, page)
        ks[s][pos] = 0
    want, wl = ha.ha_cache4_attn(Q, cache, table, L, page, q_len=q_len)
    codes = np.arange(d) % 16
    bytes_ = cache.cpu().numpy()
    values = STEPS[codes] * 2.0 ** (byte - 127)
    with np.errstate(over="ignore"):
        values = values.astype(np.float32).astype(np.float64)   # past the largest number: infinite
    for s, n in enumerate(lens):
        pos, group = n - 3, vs[s][n - 3, 1]
        scales = np.full(d // 32, 127, np.uint8)
        scales[1] = byte
        put_v(bytes_[int(table[s, pos // page]), 1], page, pos % page, np.where(np.arange(d) // 32 == 1, codes, 2), scales)
        group[:] = 1.0
        group[32:64] = np.where(np.isfinite(values[32:64]), values[32:64], 0.0)
    cache.copy_(torch.from_numpy(bytes_))
    out, lse = ha.ha_cache4_attn(Q, cache, table, L, page, q_len=q_len)
    assert torch.equal(lse, wl)
    got = host(out).reshape(2, q_len, Hq, d)
    sees = np.zeros((2, q_len, Hq), bool)
    sees[:, 2:, Hq // Hk:] = True
    np.testing.assert_array_equal(got[~sees], host(want).reshape(got.shape)[~sees])
    ref, _, absv, werr = attention64(host(Q), ks, vs, q_len)
    infinite = np.zeros(got.shape, bool)
    infinite[sees] = np.arange(d) // 32 == 1
    infinite &= ~np.isfinite(values)
    sign = np.broadcast_to(np.sign(np.where(np.isfinite(values), 0, values)), got.shape)
    np.testing.assert_array_equal(got[infinite], np.inf * sign[infinite])
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tol = (absv * (half + werr[..., None] + 2.0 ** -24 * max(lens)) + half * np.abs(ref)).reshape(got.shape)
    err = np.abs(np.where(infinite, 0, got - ref.reshape(got.shape)))
    assert (err[~infinite] <= tol[~infinite]).all(), np.max(err[~infinite] / tol[~infinite])


# name: (waves of a workgroup that takes a whole sequence, codes past the caches), lens, key heads, page, tokens of the table at least
RAGGED = [0, 1, 300, 64, 65, 129, 0, 1000, 17, 2, 511]
FORMS = {
    "whole, eight waves": ((8, False), RAGGED, 2, 16, 0),
    "whole, four waves": ((4, False), RAGGED * 12, 2, 16, 0),
    "shared": ((0, False), [0, 5000, 1, 777, 130, 6], 2, 64, 6000),
    "shared, past the caches": ((0, True), [0, 5000, 1, 777, 130, 6], 4, 256, 0),
}


def a_call(ha, torch, form, d, dtype, q_len, group=3):
    want, lens, Hk, page, tokens = FORMS[form]
    if want[1]:   # a table with room for more than 256 MiB, nearly all of it unused
        tokens = ((256 << 20) // (Hk * page * (d + d // 16) * len(lens)) + 1) * page
    rng = np.random.default_rng(40 + d + q_len)
    cache, table, ks, vs = filled_cache(ha, torch, rng, lens, Hk, d, page, tokens=tokens)
    Hq, dt = group * Hk, dtypes(torch, dtype)
    assert ha.ha_cache4_attn_form(cache.shape[0], page, Hk, d, len(lens), q_len, Hq, table.shape[1], dt) == want   # by the rule of the dispatch itself
    Q = torch.from_numpy(2 * d ** -0.25 * rng.standard_normal((len(lens) * q_len, Hq, d))).to(dt).cuda()
    return cache, table, ks, vs, Q, torch.tensor(lens, dtype=torch.int32, device="cuda"), page, lens


@pytest.mark.parametrize("q_len", [1, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_every_form(ha, torch, form, d, dtype, q_len):
    cache, table, ks, vs, Q, L, page, lens = a_call(ha, torch, form, d, dtype, q_len)
    out, lse = ha.ha_cache4_attn(Q, cache, table, L, page, q_len=q_len)
    ref, rl, absv, werr = attention64(host(Q), ks, vs, q_len)
    check_attention(host(out), host(lse), ref, rl, absv, werr, dtype, max(lens))
    again = ha.ha_cache4_attn(Q, cache, table, L, page, q_len=q_len)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    if q_len == 1:
        return
    # NaN in channels 32 ... 63 of the last tokens' V: for the last query of every sequence, and it alone
    of = [s for s, n in enumerate(lens) if n > 0]
    slots = torch.tensor([int(table[s, (lens[s] - 1) // page]) * page + (lens[s] - 1) % page for s in of], dtype=torch.int32, device="cuda")
    k, v = ha.ha_cache4_read(cache, slots, page, dtype=torch.float32)
    v[:, :, 40] = float("nan")
    ha.ha_cache4_write(k, v, slots, cache, page)
    got, got_lse = ha.ha_cache4_attn(Q, cache, table, L, page, q_len=q_len)
    hit = torch.zeros((len(lens), q_len, out.shape[1], d), dtype=torch.bool, device="cuda")
    hit[of, q_len - 1, :, 32:64] = True
    hit = hit.view(out.shape)
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], out[~hit]) and torch.equal(got_lse, lse)


@pytest.mark.parametrize("form", FORMS)
def test_large_values_stay_finite(ha, torch, form):
    """The largest |V| times the tokens just below 2^120, in both types (a scale changes no result but by itself: compared after it is taken out again)."""
    for dtype in ("bf16", "fp32"):
        cache, table, ks, vs, Q, L, page, lens = a_call(ha, torch, form, 64, dtype, 1)
        G, at = 2, page * 66   # V's scale bytes lie last in a block
        top = max(np.abs(v).max() for v in vs if len(v))
        up = 119 - int(np.ceil(np.log2(top * max(lens))))
        scales = cache[:, :, at:]
        assert scales.shape[2] == page * G
        scales[scales != 255] += up
        out, lse = ha.ha_cache4_attn(Q, cache, table, L, page)
        ref, rl, absv, werr = attention64(host(Q), ks, vs, 1)
        check_attention(host(out) * 2.0 ** -up, host(lse), ref, rl, absv, werr, dtype, max(lens))
