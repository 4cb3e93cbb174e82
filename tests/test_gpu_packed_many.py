"""Exact attention over more packed sequences than one lane-and-register table of them holds (256): their tiles are found by bisection of cu_seqlens.
Reference and tolerances are test_gpu_packed.py's."""
import numpy as np
import pytest

from ha_testutil import have_gpu
from test_gpu_packed import attention64, check, ha, host, inputs, run_all, torch  # noqa: F401  (ha and torch: fixtures)

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]

CASES = [
    # sequences, first row, query heads, key heads, d, rows behind the last
    (256, 0, 2, 1, 64, 0),      # the last number of the one way, the first of the other
    (257, 0, 2, 1, 64, 0),
    (256, 7, 4, 2, 128, 3),
    (257, 7, 4, 2, 128, 3),
    (300, 130, 8, 8, 64, 0),    # heads in eights
    (4097, 1, 1, 1, 64, 40),    # a third step of the bisection
    (6000, 5, 2, 1, 128, 0),
]


def lengths(rng, n):
    """Empty ones, runs of single rows, tiles exactly filled and overfilled, and some of several tiles."""
    kind = rng.random(n)
    lens = np.where(kind < 0.2, 0, np.where(kind < 0.5, 1, rng.integers(2, 12, n)))
    lens[n // 3:n // 3 + 20] = 1
    lens[n // 2:n // 2 + 6] = [31, 32, 33, 127, 128, 129]
    lens[rng.integers(0, n, 4)] = [300, 200, 64, 65]
    lens[n - 3:] = [0, 260, 0]
    return lens


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_many_sequences(ha, torch, case, dtype, causal):
    n, first, Hq, Hk, d, pad = CASES[case]
    rng = np.random.default_rng(70 + case)
    cu = first + np.concatenate([[0], np.cumsum(lengths(rng, n))])
    Q, K, V, dO = inputs(torch, rng, int(cu[-1]) + pad, Hq, Hk, d, dtype, fused=case % 2 == 0, scale=1.5)
    c = torch.from_numpy(cu.astype(np.int32)).cuda()
    got = run_all(ha, torch, Q, K, V, dO, c, causal, dtype)
    ref, mag = attention64(*(host(t) for t in (Q, K, V, dO)), cu, causal)
    for name, roundings in (("out", 1), ("lse", 0), ("dV", 1), ("dQ", 2), ("dK", 2)):
        check(host(got[name]), ref[name], mag[name], dtype, name, roundings)   # (rows of no sequence: zeros, as they were)
    plain = ha.exact_attn_packed_forward(Q, K, V, c, causal=causal)   # the forward alone
    seen = slice(int(cu[0]), int(cu[-1]))
    check(host(plain[0][seen]), ref["out"][seen], mag["out"][seen], dtype, "out", 1)
    check(host(plain[1][:, seen]), ref["lse"][:, seen], mag["lse"][:, seen], dtype, "lse", 0)


def test_the_longest_number_of_sequences(ha, torch):
    """n_seq * Hq = 2^22, nearly all of them empty: a row each for some, in front, in the middle and at the end."""
    n = 1 << 22
    rng = np.random.default_rng(90)
    lens = np.zeros(n, np.int64)
    lens[[0, 1, 63, 64, 65, 4095, 4096, 1 << 18, n // 2, n - 2]] = [3, 1, 2, 140, 1, 1, 5, 33, 1, 2]
    cu = np.concatenate([[0], np.cumsum(lens)])
    Q, K, V, dO = inputs(torch, rng, int(cu[-1]), 1, 1, 64, "bf16", True)
    got = run_all(ha, torch, Q, K, V, dO, torch.from_numpy(cu.astype(np.int32)).cuda(), True, "bf16")
    ref, mag = attention64(*(host(t) for t in (Q, K, V, dO)), np.unique(cu), True)
    for name, roundings in (("out", 1), ("lse", 0), ("dV", 1), ("dQ", 2), ("dK", 2)):
        check(host(got[name]), ref[name], mag[name], "bf16", name, roundings)
