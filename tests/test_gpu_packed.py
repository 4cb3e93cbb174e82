"""Exact attention over packed sequences with grouped heads, forward and backward, against a plain implementation in 64 bits.

Tolerances per element, derived from the arithmetic (eps: half a step of the tensors' type, relative: bf16 2^-8, fp32 2^-24).
A magnitude sum is the formula with every term's absolute value and differences turned into sums:
  |out| = sum_j p_j |v_j|,  |dV_j| = sum_i P_ij |dO_i|,  |delta_i| = sum_j P_ij <|dO_i|, |v_j|>,
  |dQ_i| = sum_j P_ij (<|dO_i|, |v_j|> + |delta_i|) |k_j|,  |dK_j| likewise with |q_i|.
bf16: weights enter a product rounded (eps of its magnitude sum), so do the dS; delta carries the forward's rounding of its weights (another eps of
  |dQ|, |dK|), and where it is formed from the rounded output, that rounding too (one more); every result is rounded once (eps of itself).
Both types: what is summed in fp32.  A score is a sum of d products, its error enters the weight as a factor, and results are sums over up to 2^10
  rows of magnitude: (d + 2^10) 2^-24 < 2^-13 of the magnitude sum.  That is all there is to fp32 tensors, whose products are within 2^-23.2.
  The matrix cores take operands below 2^-126 as zeros: times at most 2^10 terms of 2^16 that is less than 2^-100 of any result.
lse: a score's error, d 2^-24 sum_c |q_c k_c|, the exponential's 2^-22 (1 + |lse|), and a rounding."""
import numpy as np
import pytest

from ha_testutil import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]

EPS = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
SUMS = 2.0 ** -13


@pytest.fixture(scope="module")
def ha():
    import paper_2310_05869_amd as mod
    mod.lib()
    return mod


@pytest.fixture(scope="module")
def torch():
    import torch as t
    return t


def host(t):
    return t.detach().double().cpu().numpy()


def attention64(Q, K, V, dO, cu, causal):
    """out, lse, dQ, dK, dV in 64 bits and the magnitude sums of all but lse; rows of no sequence: zeros."""
    (T, Hq, d), Hk = Q.shape, K.shape[1]
    r = {k: np.zeros(s) for k, s in (("out", Q.shape), ("dQ", Q.shape), ("dK", K.shape), ("dV", V.shape), ("lse", (Hq, T)))}
    m = {k: np.zeros_like(v) for k, v in r.items()}
    for a, b in zip(cu[:-1], cu[1:]):
        if a == b:
            continue
        hidden = np.triu(np.ones((b - a, b - a), bool), 1) if causal else None
        for h in range(Hq):
            g = h * Hk // Hq
            q, k, v, do = Q[a:b, h], K[a:b, g], V[a:b, g], dO[a:b, h]
            S = q @ k.T
            if causal:
                S[hidden] = -np.inf
            top = S.max(1, keepdims=True)
            P = np.exp(S - top)
            L = P.sum(1, keepdims=True)
            P /= L
            o = P @ v
            r["out"][a:b, h], r["lse"][h, a:b] = o, (top + np.log(L))[:, 0]
            dP = do @ v.T
            delta = (do * o).sum(1, keepdims=True)
            dS = P * (dP - delta)
            r["dQ"][a:b, h] = dS @ k
            r["dK"][a:b, g] += dS.T @ q
            r["dV"][a:b, g] += P.T @ do
            adP = np.abs(do) @ np.abs(v).T
            adS = P * (adP + (P * adP).sum(1, keepdims=True))
            m["out"][a:b, h] = P @ np.abs(v)
            m["dQ"][a:b, h] = adS @ np.abs(k)
            m["dK"][a:b, g] += adS.T @ np.abs(q)
            m["dV"][a:b, g] += P.T @ np.abs(do)
            m["lse"][h, a:b] = d * 2.0 ** -24 * (np.abs(q) @ np.abs(k).T).max(1) + 2.0 ** -22 * (1 + np.abs(r["lse"][h, a:b]))
    return r, m


def check(got, ref, mag, dtype, name, roundings):
    eps = EPS[dtype]
    tol = mag + 2.0 ** -24 * np.abs(ref) if name == "lse" else (roundings * (eps if dtype == "bf16" else 0) + SUMS) * mag + eps * np.abs(ref) + 2.0 ** -100
    err = np.abs(got - ref)
    assert np.isfinite(got).all() and (err <= tol).all(), \
        f"{name}: {(err > tol).sum()} of {err.size} off, at worst {np.max(err / np.maximum(tol, 1e-300)):.2f} of what is allowed"


def inputs(torch, rng, T, Hq, Hk, d, dtype, fused, scale=1.0):
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    x = rng.standard_normal((T, Hq + 2 * Hk, d))
    x[:, :Hq + Hk] *= scale * d ** -0.25
    x = torch.from_numpy(x).to(dt).cuda()
    parts = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    dO = torch.from_numpy(rng.standard_normal((T, Hq, d))).to(dt).cuda()
    return (parts if fused else tuple(p.contiguous() for p in parts)) + (dO,)


def run_all(ha, torch, Q, K, V, dO, cu, causal, dtype, keep_f32=True, **kw):
    T, Hq, d = Q.shape
    f32 = torch.zeros(T, Hq, d, device="cuda") if dtype == "bf16" and keep_f32 else None
    out = torch.zeros(T, Hq, d, dtype=Q.dtype, device="cuda")
    lse = torch.zeros(Hq, T, device="cuda")
    ha.exact_attn_packed_forward(Q, K, V, cu, causal=causal, out=out, lse=lse, out_f32=f32)
    dQ, dK, dV = ha.exact_attn_packed_backward(Q, K, V, cu, out, lse, dO, causal=causal, out_f32=f32, **kw)
    return dict(out=out, lse=lse, dQ=dQ, dK=dK, dV=dV)


CASES = [
    # lens, Hq, Hk, d, pad
    ([1], 1, 1, 64, 0),
    ([1, 1, 1, 2], 2, 1, 128, 3),
    ([0, 5, 0, 0, 31, 32, 33], 4, 2, 64, 0),
    ([127, 128, 129], 3, 3, 128, 1),
    ([63, 64, 65, 0, 200], 8, 2, 128, 70),
    ([513], 6, 1, 64, 0),
    ([700, 3, 260], 5, 5, 64, 0),
    ([1500], 8, 8, 64, 5),           # heads in eights: a head's tiles on one XCD
    ([300] * 9 + [0] * 70 + [17], 8, 1, 64, 0),   # more sequences than lanes
    ([2100, 40], 4, 2, 128, 0),
    # the gradients' passes one behind the other: long rows at d = 128, and many workgroups of either type
    ([2300], 4, 2, 128, 0),
    ([400] * 6 + [90], 16, 4, 128, 2),
    ([300] * 12, 32, 8, 128, 0),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_packed_forward_and_backward(ha, torch, case, dtype, causal):
    lens, Hq, Hk, d, pad = CASES[case]
    rng = np.random.default_rng(case)
    cu = np.concatenate([[0], np.cumsum(lens)])
    T = int(cu[-1]) + pad
    Q, K, V, dO = inputs(torch, rng, T, Hq, Hk, d, dtype, fused=case % 2 == 0, scale=1.5)
    c = torch.from_numpy(cu.astype(np.int32)).cuda()
    got = run_all(ha, torch, Q, K, V, dO, c, causal, dtype)
    ref, mag = attention64(*(host(t) for t in (Q, K, V, dO)), cu, causal)
    for name, n in (("out", 1), ("lse", 0), ("dV", 1), ("dQ", 2), ("dK", 2)):
        check(host(got[name]), ref[name], mag[name], dtype, name, n)
    again = run_all(ha, torch, Q, K, V, dO, c, causal, dtype)
    for name in got:
        assert torch.equal(got[name], again[name]), name


@pytest.mark.parametrize("lens,Hq,Hk,split", [([900, 1300, 1100, 128, 600, 777] * 2, 16, 8, True), ([1024] * 7 + [700], 32, 16, False)])
def test_many_workgroups(ha, torch, lens, Hq, Hk, split):
    """Key heads in eights, and enough tiles that one bf16 workgroup takes a key head's query heads together."""
    rng = np.random.default_rng(50)
    d = 64
    cu = np.concatenate([[0], np.cumsum(lens)])
    assert (ha.exact_attn_packed_backward_workspace_bytes(int(cu[-1]), len(lens), Hq, Hk, d) > int(cu[-1]) * Hq * 4 + 512) == split
    c = torch.from_numpy(cu.astype(np.int32)).cuda()
    for dtype in ("bf16", "fp32"):
        Q, K, V, dO = inputs(torch, rng, int(cu[-1]), Hq, Hk, d, dtype, True)
        got = run_all(ha, torch, Q, K, V, dO, c, True, dtype)
        ref, mag = attention64(*(host(t) for t in (Q, K, V, dO)), cu, True)
        for name, n in (("out", 1), ("lse", 0), ("dV", 1), ("dQ", 2), ("dK", 2)):
            check(host(got[name]), ref[name], mag[name], dtype, name, n)


def test_backward_from_the_rounded_output(ha, torch):
    rng = np.random.default_rng(51)
    lens, Hq, Hk, d = [300, 90], 4, 2, 128
    cu = np.concatenate([[0], np.cumsum(lens)])
    Q, K, V, dO = inputs(torch, rng, 390, Hq, Hk, d, "bf16", True)
    got = run_all(ha, torch, Q, K, V, dO, torch.from_numpy(cu.astype(np.int32)).cuda(), True, "bf16", keep_f32=False)
    ref, mag = attention64(*(host(t) for t in (Q, K, V, dO)), cu, True)
    for name, n in (("dV", 1), ("dQ", 3), ("dK", 3)):
        check(host(got[name]), ref[name], mag[name], "bf16", name, n)


def test_gradients_against_differences(ha, torch):
    """<dO, out> along random directions: its difference quotient in 64 bits, of step 1e-5 (error of the order of 1e-10 and 1e-16 / 1e-5), against the
    gradients' products with the direction: 2^-13 of their magnitude sums, as above, and that."""
    rng = np.random.default_rng(52)
    lens, Hq, Hk, d = [40, 1, 100], 4, 2, 64
    cu = np.concatenate([[0], np.cumsum(lens)])
    x = inputs(torch, rng, 141, Hq, Hk, d, "fp32", False)
    got = run_all(ha, torch, *x, torch.from_numpy(cu.astype(np.int32)).cuda(), True, "fp32")
    Q, K, V, dO = (host(t) for t in x)
    _, mag = attention64(Q, K, V, dO, cu, True)
    for i, name in enumerate(("dQ", "dK", "dV")):
        way = rng.standard_normal((Q, K, V)[i].shape)
        ends = []
        for sign in (1, -1):
            args = [Q, K, V]
            args[i] = args[i] + sign * 1e-5 * way
            ends.append((attention64(*args, dO, cu, True)[0]["out"] * dO).sum())
        quotient = (ends[0] - ends[1]) / 2e-5
        assert abs(quotient - (host(got[name]) * way).sum()) <= SUMS * (mag[name] * np.abs(way)).sum() + 1e-6 * max(1, abs(quotient))


def test_rows_of_no_sequence_and_of_others_do_not_matter(ha, torch):
    """NaN and infinities in padding rows and in another sequence reach no other sequence; rows of no sequence are left as they were."""
    rng = np.random.default_rng(53)
    for dtype in ("bf16", "fp32"):
        for d in (64, 128):
            Q, K, V, dO = inputs(torch, rng, 300, 4, 2, d, dtype, True)
            cu = torch.tensor([10, 110, 205, 270], dtype=torch.int32, device="cuda")
            want = run_all(ha, torch, Q, K, V, dO, cu, True, dtype)
            for t in (Q, K, V, dO):
                t[:10] = float("nan")
                t[270:] = float("inf")
                t[110:205] = float("nan")
            grads = tuple(torch.full_like(t, 7) for t in (Q.contiguous(), K.contiguous(), V.contiguous()))
            got = run_all(ha, torch, Q, K, V, dO, cu, True, dtype, grads=grads)
            for name in want:
                a, b = (x[name].transpose(0, 1) if name == "lse" else x[name] for x in (got, want))
                for rows in (slice(10, 110), slice(205, 270)):
                    assert torch.equal(a[rows], b[rows]), name
                for rows in (slice(0, 10), slice(270, 300)):
                    assert (a[rows] == (7 if name[0] == "d" else 0)).all(), name


def test_one_sequence_is_exact_attention(ha, torch):
    """The same rows as one head-major batch through exact_attn_forward: one operand rounding apart."""
    torch.manual_seed(1)
    T, H, d = 777, 4, 128
    q, k, v = (torch.randn(1, H, T, d, device="cuda").mul_(d ** -0.25).bfloat16() for _ in range(3))
    out, lse = ha.exact_attn_forward(q, k, v, causal=True)
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    o2, l2 = ha.exact_attn_packed_forward(*(t[0].transpose(0, 1) for t in (q, k, v)), cu, causal=True)   # strided as it lies
    tol = 2 * 2.0 ** -8 * 4 * d ** -0.25   # |v| below 4 standard deviations but for a few: weights' and results' rounding, twice
    assert (out[0].transpose(0, 1).float() - o2.float()).abs().max() <= tol and (lse[0] - l2).abs().max() <= 1e-5


def test_far_references_and_large_scores(ha, torch):
    rng = np.random.default_rng(54)
    lens = [400, 130]
    cu = np.concatenate([[0], np.cumsum(lens)])
    for dtype in ("bf16", "fp32"):
        Q, K, V, dO = inputs(torch, rng, 530, 2, 1, 64, dtype, True, scale=6.0)
        got = run_all(ha, torch, Q, K, V, dO, torch.from_numpy(cu.astype(np.int32)).cuda(), True, dtype)
        ref, mag = attention64(*(host(t) for t in (Q, K, V, dO)), cu, True)
        assert ref["lse"].max() > 80
        # scores of hundreds: a weight's relative error is a score's absolute one, bounded by the lse's
        score = mag["lse"].max()
        for name, n in (("out", 1), ("dV", 1), ("dQ", 2), ("dK", 2)):
            check(host(got[name]), ref[name], mag[name] * (1 + 2 * score / SUMS), dtype, name, n)


def test_senseless_bounds_stay_inside(ha, torch):
    """cu_seqlens past the rows, negative, decreasing: clamped; a guard around every tensor stays whole and no access leaves them."""
    T, Hq, Hk, d = 100, 2, 1, 64
    for cu in ([0, 2 ** 31 - 1], [-5, 50, 2 ** 30], [90, 20, 60], [200, 300, 400], [0, 100, 0, 100]):
        big = torch.zeros(3 * T, Hq, d, device="cuda", dtype=torch.bfloat16)
        Q, K, V = (torch.randn(T, h, d, device="cuda").bfloat16() for h in (Hq, Hk, Hk))
        lse = torch.zeros(Hq, T, device="cuda")
        c = torch.tensor(cu, dtype=torch.int32, device="cuda")
        ha.exact_attn_packed_forward(Q, K, V, c, causal=True, out=big[T:2 * T], lse=lse)
        assert (big[:T] == 0).all() and (big[2 * T:] == 0).all()
        dbig = tuple(torch.zeros(3 * T, h, d, device="cuda", dtype=torch.bfloat16) for h in (Hq, Hk, Hk))
        ha.exact_attn_packed_backward(Q, K, V, c, big[T:2 * T], lse, Q, causal=True, grads=tuple(t[T:2 * T] for t in dbig))
        for t in dbig:
            assert (t[:T] == 0).all() and (t[2 * T:] == 0).all()
    whole = ha.exact_attn_packed_forward(Q, K, V, torch.tensor([0, T], dtype=torch.int32, device="cuda"), causal=True)
    over = ha.exact_attn_packed_forward(Q, K, V, torch.tensor([-3, T + 1000], dtype=torch.int32, device="cuda"), causal=True)
    assert torch.equal(whole[0], over[0]) and torch.equal(whole[1], over[1])


def test_streams_workspaces_and_outputs_as_slices(ha, torch):
    rng = np.random.default_rng(55)
    T, Hq, Hk, d = 260, 4, 2, 64
    Q, K, V, dO = inputs(torch, rng, T, Hq, Hk, d, "bf16", True)
    cu = torch.tensor([0, 60, 260], dtype=torch.int32, device="cuda")
    want = run_all(ha, torch, Q, K, V, dO, cu, False, "bf16", keep_f32=False)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, lse = ha.exact_attn_packed_forward(Q, K, V, cu, stream=s)
    all_grads = torch.zeros(T, Hq + 2 * Hk, d, dtype=torch.bfloat16, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    grads = all_grads[:, :Hq], all_grads[:, Hq:Hq + Hk], all_grads[:, Hq + Hk:]
    ws = torch.full((ha.exact_attn_packed_backward_workspace_bytes(T, 2, Hq, Hk, d),), 255, dtype=torch.uint8, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    ha.exact_attn_packed_backward(Q, K, V, cu, out, lse, dO, stream=s, grads=grads, workspace=ws)
    free = ha.exact_attn_packed_backward(Q, K, V, cu, out, lse, dO, stream=s)
    s.synchronize()
    assert torch.equal(out, want["out"]) and torch.equal(lse, want["lse"])
    for name, a, b in zip(("dQ", "dK", "dV"), grads, free):
        assert torch.equal(a, want[name]) and torch.equal(b, want[name])


def test_a_captured_training_step_replays(ha, torch):
    rng = np.random.default_rng(56)
    T, Hq, Hk, d = 300, 6, 2, 64
    cu = torch.tensor([0, 100, 100, 290], dtype=torch.int32, device="cuda")
    for dtype in ("bf16", "fp32"):
        x = inputs(torch, rng, T, Hq, Hk, d, dtype, True)
        ws = torch.empty(ha.exact_attn_packed_backward_workspace_bytes(T, 3, Hq, Hk, d, x[0].dtype), dtype=torch.uint8, device="cuda")
        bufs = {k: torch.zeros_like(v) for k, v in run_all(ha, torch, *x, cu, True, dtype).items()}

        def step():
            ha.exact_attn_packed_forward(*x[:3], cu, causal=True, out=bufs["out"], lse=bufs["lse"])
            ha.exact_attn_packed_backward(*x[:3], cu, bufs["out"], bufs["lse"], x[3], causal=True, workspace=ws, grads=(bufs["dQ"], bufs["dK"], bufs["dV"]))

        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for trial in range(3):
            for t in x:
                t.copy_(torch.randn_like(t) * 0.5)
            want = run_all(ha, torch, *x, cu, True, dtype, keep_f32=False)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for name in want:
                assert torch.equal(bufs[name], want[name]), (dtype, name)
