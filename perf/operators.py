"""Packed attention and the 4-bit paged cache: what their speed and results are measured on.

A case is one call, or the calls that belong together, on tensors that stay on the GPU:
  packed_fwd    exact_attn_packed_forward: exact attention over sequences of different lengths in one batch of rows, grouped heads
  packed_train  the same with the unrounded output (bf16) and exact_attn_packed_backward
  plan          ha_page_plan: pages given to sequences and taken back, block tables and slots of the step's rows
  rows          ha_cache4_write of new rows of K and V into pages, then ha_cache4_read of the same slots, as for a prefix used again
  attend        ha_cache4_attn: queries of every sequence's last tokens over the sequence's pages

Scores carry no 1/sqrt(d): Q and K come scaled by d^(-1/4) each.  The cache holds E2M1 values, 32 channels to a power of two (OCP MX FP4).
The plain forms are computed in 32 bits and rounded once.
"""
import math
import random

import torch

own = False

CACHE_GROUP = 32   # channels that share a scale
LEAST_BYTE, LARGEST_BYTE = 2, 252   # scales that a writer gives: 2^-125 ... 2^125


# ---------------------------------------------------------------- cases
def _packed(name, kind, n_seq, max_len, Hq, Hk, d, dtype="bf16", causal=True, fused=False, pad=0, law="ragged", lens_seed=1):
    return dict(name=name, kind=kind, n_seq=n_seq, max_len=max_len, Hq=Hq, Hk=Hk, d=d, dtype=dtype, causal=causal, fused=fused, pad=pad,
                law=law, lens_seed=lens_seed)


def listed():
    return [
        # a few short prompts together: a call is its latency
        _packed("packed_fwd_short_prompts", "packed_fwd", 7, 300, 8, 2, 64, pad=5),
        # a serving step's prompts, up to 8192 tokens, as slices of one projection's output
        _packed("packed_fwd_prompts_8k", "packed_fwd", 24, 8192, 32, 8, 128, fused=True, lens_seed=3),
        # texts to encode: no mask, fp32
        _packed("packed_fwd_encode_fp32", "packed_fwd", 9, 700, 6, 3, 64, dtype="fp32", causal=False),
        # a training step's attention over packed documents
        _packed("packed_train_documents", "packed_train", 16, 4096, 12, 4, 128, fused=True, lens_seed=4),
        # the same in fp32, small
        _packed("packed_train_fp32", "packed_train", 5, 900, 4, 2, 64, dtype="fp32", pad=3),
        # a decoding step: every sequence one token further, a few end
        dict(name="plan_decode_256", kind="plan", n_seq=256, page=64, max_blocks=256, n_pages=40000, max_add=1, slots=256, ends=0.02, lens_seed=2),
        # prompts admitted while others end: long runs of slots, many pages
        dict(name="plan_prompts_1k", kind="plan", n_seq=1000, page=16, max_blocks=1024, n_pages=500000, max_add=2000, slots=500000, ends=0.2, lens_seed=5),
        # one decoding step's rows of a small fp32 layer
        dict(name="rows_decode_fp32", kind="rows", rows=48, Hk=4, d=64, page=16, n_pages=512, dtype="fp32"),
        # the rows of a batch of prompts
        dict(name="rows_prompts_16k", kind="rows", rows=16411, Hk=8, d=128, page=64, n_pages=1024, dtype="bf16"),
        # one short sequence: a call is its latency
        dict(name="attend_one_short", kind="attend", n_seq=1, q_len=1, max_len=777, Hq=8, Hk=4, d=64, page=16, dtype="bf16", law="even", lens_seed=1),
        # a batch in full flight: lengths from nothing to 16384, three tokens a sequence (drafted ones are verified together)
        dict(name="attend_batch_64", kind="attend", n_seq=64, q_len=3, max_len=16384, Hq=32, Hk=8, d=128, page=64, dtype="bf16", law="ragged", lens_seed=6),
        # long contexts, one token each: the largest
        dict(name="attend_4_long", kind="attend", n_seq=4, q_len=1, max_len=131072, Hq=32, Hk=8, d=128, page=128, dtype="bf16", law="even", lens_seed=7),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / (1e15 if case.get("dtype") != "fp32" else 1e14))


def draw(rng):
    """One more case: every kind, both types and head sizes, one to 64 query heads, sequences from none to 16384 tokens packed, to 131072 cached."""
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["packed_fwd", "packed_fwd", "packed_train", "packed_train", "plan", "rows", "attend", "attend", "attend"])
        d, dtype = rng.choice([64, 128]), rng.choice(["bf16", "bf16", "fp32"])
        Hk = _log_int(rng, 1, 16)
        Hq = Hk * rng.choice([1, 2, 3, 4, 4, 5, 8])
        c = dict(kind=kind, lens_seed=rng.randrange(1 << 20))
        if kind in ("packed_fwd", "packed_train"):
            c.update(n_seq=_log_int(rng, 1, 200), max_len=_log_int(rng, 16, 16384 if dtype == "bf16" else 3000), Hq=Hq, Hk=Hk, d=d, dtype=dtype,
                     causal=rng.random() < 0.75, fused=rng.random() < 0.4, pad=rng.choice([0, 0, rng.randrange(200)]), law=rng.choice(["ragged", "ragged", "even"]))
            if sum(_lens(c)) > 70000 or sum(_lens(c)) == 0 or c["n_seq"] * c["max_len"] > 400000:
                continue
        elif kind == "plan":
            c.update(n_seq=_log_int(rng, 1, 4000), page=rng.choice([16, 32, 64, 128, 256]), max_blocks=_log_int(rng, 4, 2000), n_pages=_log_int(rng, 64, 400000),
                     max_add=rng.choice([1, 1, _log_int(rng, 2, 4000)]), ends=rng.choice([0.0, 0.1, 0.5]))
            c["slots"] = max(1, int(c["n_seq"] * c["max_add"] * rng.choice([1.0, 1.0, 0.4])))
            if c["n_seq"] * c["max_blocks"] > 4e6 or c["slots"] > 2e6:
                continue
        elif kind == "rows":
            c.update(rows=_log_int(rng, 1, 30000), Hk=Hk, d=d, page=rng.choice([16, 32, 64, 128, 256]), dtype=dtype)
            c["n_pages"] = 1 + int(c["rows"] * rng.choice([1.0, 2.0, 5.0])) // c["page"]
        else:
            if Hq > 64:
                continue
            c.update(n_seq=_log_int(rng, 1, 256), q_len=rng.choice([1, 1, 1, 2, 4, 7]), max_len=_log_int(rng, 1, 131072), Hq=Hq, Hk=Hk, d=d,
                     page=rng.choice([16, 32, 64, 128, 256]), dtype=dtype, law=rng.choice(["ragged", "ragged", "even"]))
            if c["n_seq"] * c["max_len"] * Hk * d > 1 << 30:
                continue
        if _cost(c) <= most and (Hq + 2 * Hk) * d != 3 << 10:
            return c


def _lens(c):
    """Tokens of every sequence; ragged: from none to max_len, over their logarithm, one of them the longest."""
    rng = random.Random(c["lens_seed"])
    if c["law"] == "even":
        return [c["max_len"] - (i % 3 if c["max_len"] > 8 else 0) for i in range(c["n_seq"])]
    lens = [0 if rng.random() < 0.05 else _log_int(rng, 1, c["max_len"]) for _ in range(c["n_seq"])]
    lens[rng.randrange(len(lens))] = c["max_len"]
    return lens


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _plan_numbers(c):
    """(tokens held, tokens to add or -1 for an end) of every sequence."""
    rng = random.Random(c["lens_seed"])
    cap = c["max_blocks"] * c["page"]
    held = [rng.randrange(0, max(1, min(cap, c["n_pages"] * c["page"] // c["n_seq"]) // 2 + 1)) for _ in range(c["n_seq"])]
    add = [-1 if rng.random() < c["ends"] else 1 if c["max_add"] == 1 else rng.randrange(0, c["max_add"] + 1) for _ in range(c["n_seq"])]
    return held, add


def _cached_pages(n, page):
    return (n + page - 1) // page


# ---------------------------------------------------------------- inputs
def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _token_bytes(d):
    return d + d // 16


def _quantised(x):
    """E2M1 codes (sign bit 3) and scale bytes of x [..., d] in fp32: 32 channels share the smallest power of two s with max |x| <= 6 s, of 2^-125 ... 2^125."""
    g = x.reshape(*x.shape[:-1], -1, CACHE_GROUP)
    most = g.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(most)
    f, k = torch.frexp(torch.where(fine, most, torch.ones_like(most)))
    e = (k - torch.where(f <= 0.75, 3, 2)).clamp(LEAST_BYTE - 127, LARGEST_BYTE - 127)
    y = torch.ldexp(torch.where(fine, g, torch.zeros_like(g)), -e)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=x.device)   # half way: to the even code
    a = y.abs()
    code = (a > edges[0]).int() + (a >= edges[1]).int() + (a > edges[2]).int() + (a >= edges[3]).int() + (a > edges[4]).int() + \
        (a >= edges[5]).int() + (a > edges[6]).int()
    code = code + 8 * ((y < 0) & (code > 0)).int()
    byte = torch.where(fine, e + 127, torch.full_like(e, 255))
    return code.reshape(x.shape), byte.reshape(*x.shape[:-1], -1).to(torch.uint8)


def _values(code, byte, dtype):
    """What codes [..., d] and scale bytes [..., d / 32] stand for."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], dtype=dtype, device=code.device)
    s = torch.where(byte == 255, torch.full((), float("nan"), dtype=dtype, device=code.device),
                    torch.ldexp(torch.ones((), dtype=dtype, device=code.device), byte.int() - 127))
    return (table[code.long()].reshape(*byte.shape, CACHE_GROUP) * s[..., None]).reshape(code.shape)


def _v_places(d, device):
    """Of channel c of a V row: its word among the row's d / 8, and its nibble there."""
    c = torch.arange(d, device=device)
    g, m, e = c // 32, (c % 32) // 2, c % 2
    return (m, 2 * g + e) if d == 128 else (m // 2, 2 * (2 * g + m % 2) + e)


def _k_places(d, device):
    c = torch.arange(d, device=device)
    return (c % 32) // 8 * (d // 32) + c // 32, c % 8


def _page_bytes(kc, ks, vc, vs):
    """Pages of the cache from codes [n, Hk, page, d] and scale bytes [n, Hk, page, d / 32]."""
    n, Hk, page, d = kc.shape

    def words(codes, places):
        w, nib = places
        out = torch.zeros(n, Hk, page, d // 8, dtype=torch.int64, device=codes.device)
        out.index_add_(3, w, codes.long() << (4 * nib))
        return out

    kw = words(kc, _k_places(d, kc.device))
    vw = words(vc, _v_places(d, vc.device)).reshape(n, Hk, page // 4, 4, d // 8).transpose(3, 4)
    as_bytes = lambda w: torch.stack([(w >> s) & 255 for s in (0, 8, 16, 24)], -1).to(torch.uint8).reshape(n, Hk, -1)  # noqa: E731
    return torch.cat([as_bytes(kw), as_bytes(vw), ks.reshape(n, Hk, -1), vs.reshape(n, Hk, -1)], -1)


def _page_values(pages, page, d, dtype):
    """K and V [n, Hk, page, d] of pages [n, Hk, bytes]."""
    n, Hk, _ = pages.shape
    half = page * d // 2
    place = lambda w, nib: (w * 4 + nib // 2, 4 * (nib % 2))  # noqa: E731
    kb, ksh = place(*_k_places(d, pages.device))
    kc = (pages[..., :half].reshape(n, Hk, page, d // 2)[..., kb] >> ksh.to(torch.uint8)) & 15
    vb = pages[..., half:2 * half].reshape(n, Hk, page // 4, d // 8, 4, 4).transpose(3, 4).reshape(n, Hk, page, d // 2)
    at, vsh = place(*_v_places(d, pages.device))
    vc = (vb[..., at] >> vsh.to(torch.uint8)) & 15
    G = d // CACHE_GROUP
    ks = pages[..., 2 * half:2 * half + page * G].reshape(n, Hk, page, G)
    vs = pages[..., 2 * half + page * G:].reshape(n, Hk, page, G)
    return _values(kc, ks, dtype), _values(vc, vs, dtype)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = None if c["kind"] == "plan" else _type(c)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    s = {"c": c}
    if c["kind"] in ("packed_fwd", "packed_train"):
        lens, Hq, Hk, d = _lens(c), c["Hq"], c["Hk"], c["d"]
        T = sum(lens) + c["pad"]
        s["lens"] = lens
        s["cu"] = torch.tensor(_starts(lens), dtype=torch.int32, device="cuda")
        if c["fused"]:
            all_heads = torch.cat([2 * d ** -0.25 * randn(T, Hq, d), d ** -0.25 * randn(T, Hk, d), randn(T, Hk, d)], 1).to(dt)
            s["Q"], s["K"], s["V"] = all_heads[:, :Hq], all_heads[:, Hq:Hq + Hk], all_heads[:, Hq + Hk:]
        else:
            s["Q"], s["K"], s["V"] = ((2 * d ** -0.25 * randn(T, Hq, d)).to(dt), (d ** -0.25 * randn(T, Hk, d)).to(dt), randn(T, Hk, d).to(dt))
        s["out"] = torch.zeros(T, Hq, d, dtype=dt, device="cuda")   # rows behind the last sequence stay as they are
        s["lse"] = torch.zeros(Hq, T, dtype=torch.float32, device="cuda")
        if c["kind"] == "packed_train":
            s["d_out"] = randn(T, Hq, d).to(dt)
            s["out_f32"] = torch.zeros(T, Hq, d, dtype=torch.float32, device="cuda") if c["dtype"] == "bf16" else None
            s["grads"] = tuple(torch.zeros(T, H, d, dtype=dt, device="cuda") for H in (Hq, Hk, Hk))
            # fp32 rows of the key heads' partial sums and one float per query row, at most
            s["workspace"] = torch.empty(256 * 4 + 4 * T * Hq * (1 + 2 * d), dtype=torch.uint8, device="cuda")
    elif c["kind"] == "plan":
        held, add = _plan_numbers(c)
        page, most, n = c["page"], c["max_blocks"], c["n_seq"]
        order = torch.randperm(c["n_pages"], generator=g, device="cuda").to(torch.int32)
        used = [min(_cached_pages(h, page), most) for h in held]
        table = torch.full((n, most), -1, dtype=torch.int32, device="cuda")
        first = torch.tensor(_starts(used)[:-1], device="cuda")
        j = torch.arange(most, device="cuda")
        inside = j[None, :] < torch.tensor(used, device="cuda")[:, None]
        table[inside] = order[(first[:, None] + j[None, :])[inside]]
        left = order[sum(used):].contiguous()
        free = torch.full((c["n_pages"],), -1, dtype=torch.int32, device="cuda")
        free[:left.numel()] = left
        s.update(lens=torch.tensor(held, dtype=torch.int32, device="cuda"), add=torch.tensor(add, dtype=torch.int32, device="cuda"), table=table, free=free,
                 free_count=torch.tensor([left.numel()], dtype=torch.int32, device="cuda"),
                 lens_out=torch.empty(n, dtype=torch.int32, device="cuda"), cu=torch.empty(n + 1, dtype=torch.int32, device="cuda"),
                 slots=torch.empty(c["slots"], dtype=torch.int32, device="cuda"), free_count_out=torch.empty(1, dtype=torch.int32, device="cuda"))
    elif c["kind"] == "rows":
        N, Hk, d = c["rows"], c["Hk"], c["d"]
        scale = 2.0 ** torch.randint(-3, 4, (1, Hk, d), generator=g, device="cuda")   # channels of unlike size, as keys have them
        s["K"], s["V"] = (scale * randn(N, Hk, d)).to(dt), randn(N, Hk, d).to(dt)
        s["slots"] = torch.randperm(c["n_pages"] * c["page"], generator=g, device="cuda")[:N].to(torch.int32)
        s["cache"] = torch.zeros(c["n_pages"], Hk, c["page"] * _token_bytes(d), dtype=torch.uint8, device="cuda")
        s["K_back"], s["V_back"] = torch.empty_like(s["K"]), torch.empty_like(s["V"])
    else:
        lens, Hq, Hk, d, page = _lens(c), c["Hq"], c["Hk"], c["d"], c["page"]
        blocks = [_cached_pages(n, page) for n in lens]
        most, total = max(1, max(blocks)), sum(blocks)
        pool = min(total + 1, 1 << 22 >> int(math.log2(Hk * page * d)) if Hk * page * d < 1 << 22 else 1)
        pool = max(pool, min(total + 1, 8))
        pages = _page_bytes(*_quantised(d ** -0.25 * randn(pool, Hk, page, d)), *_quantised(randn(pool, Hk, page, d)))
        s["cache"] = pages[torch.randint(0, pool, (total + 1,), generator=g, device="cuda")]
        order = torch.randperm(total + 1, generator=g, device="cuda").to(torch.int32)
        table = torch.full((c["n_seq"], most), -1, dtype=torch.int32, device="cuda")
        first = torch.tensor(_starts(blocks)[:-1], device="cuda")
        j = torch.arange(most, device="cuda")
        inside = j[None, :] < torch.tensor(blocks, device="cuda")[:, None]
        table[inside] = order[(first[:, None] + j[None, :])[inside]]
        s["table"], s["lens"], s["host_lens"] = table, torch.tensor(lens, dtype=torch.int32, device="cuda"), lens
        s["Q"] = (2 * d ** -0.25 * randn(c["n_seq"] * c["q_len"], Hq, d)).to(dt)
        s["out"], s["lse"] = torch.empty_like(s["Q"]), torch.empty(Hq, c["n_seq"] * c["q_len"], dtype=torch.float32, device="cuda")
        s["workspace"] = torch.empty(_attend_workspace(c), dtype=torch.uint8, device="cuda")
    return s


def _attend_workspace(c):
    """Bytes that serve any split of the call's keys: 2048 parts and one more per sequence, of 16 query rows per key head and tile of rows, in fp32."""
    tiles = (c["q_len"] * c["Hq"] // c["Hk"] + 15) // 16
    return 4096 + 4 * c["n_seq"] + (2048 + c["n_seq"] * c["Hk"] * tiles) * 16 * (c["d"] + 4) * 4


# ---------------------------------------------------------------- plain forms
def _groups(lens, per_pair, most=1 << 28):
    """Runs of sequences whose padded scores fit together."""
    out, first = [], 0
    for i in range(1, len(lens) + 1):
        if i == len(lens) or (i + 1 - first) * max(lens[first:i + 1]) ** 2 * per_pair > most:
            out.append((first, i))
            first = i
    return [(a, b) for a, b in out if max(lens[a:b]) > 0]


def _packed_plain(s):
    c, lens = s["c"], s["lens"]
    Hq, Hk, d = c["Hq"], c["Hk"], c["d"]
    G, dev = Hq // Hk, s["Q"].device
    train = c["kind"] == "packed_train"
    out, lse = s["out"].clone(), s["lse"].clone()
    grads = [x.clone() for x in s["grads"]] if train else None
    for a, b in _groups(lens, Hq):
        L = max(lens[a:b])
        n = s["cu"][a + 1:b + 1] - s["cu"][a:b]
        pos = torch.arange(L, device=dev)
        live = pos[None, :] < n[:, None]                                  # [c, L]
        rows = torch.where(live, s["cu"][a:b, None] + pos[None, :], 0)

        def head_first(x, H):
            x = torch.where(live[..., None, None], x[rows].float(), 0.0)   # [c, L, H, d]
            return x.permute(0, 2, 1, 3).reshape(b - a, Hk, (H // Hk) * L, d)

        q, k, v = head_first(s["Q"], Hq), head_first(s["K"], Hk), head_first(s["V"], Hk)
        allowed = live[:, None, :] & live[:, :, None]
        if c["causal"]:
            allowed = allowed & (pos[None, :] <= pos[:, None])
        allowed = allowed[:, None, None]                                  # [c, 1, 1, L, L]
        S = torch.matmul(q, k.transpose(-1, -2)).view(b - a, Hk, G, L, L).masked_fill(~allowed, float("-inf"))
        top = S.amax(-1, keepdim=True)
        top = torch.where(top == float("-inf"), 0.0, top)
        P = torch.exp(S - top)
        del S
        total = P.sum(-1, keepdim=True)
        P = P / torch.where(total > 0, total, 1.0)
        P2 = P.view(b - a, Hk, G * L, L)
        O = torch.matmul(P2, v)
        back = lambda x, H: x.reshape(b - a, H, L, d).permute(0, 2, 1, 3)[live]  # noqa: E731
        at = rows[live]
        out[at] = back(O, Hq).to(out.dtype)
        lse[:, at] = (top + torch.log(total)).view(b - a, Hq, L).transpose(0, 1)[:, live]
        if train:
            g = head_first(s["d_out"], Hq)
            grads[2][at] = back(torch.matmul(P2.transpose(-1, -2), g), Hk).to(out.dtype)
            dS = torch.matmul(g, v.transpose(-1, -2)).sub_((g * O).sum(-1, keepdim=True)).mul_(P2)
            grads[0][at] = back(torch.matmul(dS, k), Hq).to(out.dtype)
            grads[1][at] = back(torch.matmul(dS.transpose(-1, -2), q), Hk).to(out.dtype)
    r = {"out": out, "lse": lse}
    if train:
        r.update(dQ=grads[0], dK=grads[1], dV=grads[2])
    return r


def _plan_plain(s):
    c = s["c"]
    page, most, N, cap_rows = c["page"], c["max_blocks"], c["n_pages"], c["slots"]
    held = s["lens"].long().clamp(0, most * page)
    add = s["add"].long()
    ends = add < 0
    rows = add.clamp(min=0)
    have, to = (held + page - 1) // page, held + rows
    cu_end = rows.cumsum(0)
    fits = ~ends & (to <= most * page) & (cu_end <= cap_rows)
    need = torch.where(fits, (to + page - 1) // page - have, 0)
    upto = need.cumsum(0)
    freed = torch.where(ends, have, 0)
    count = s["free_count"].long().clamp(0, N)
    avail = (count + freed.sum()).clamp(max=N)
    served = fits & ((need == 0) | (upto <= avail))
    need = torch.where(served, need, 0)
    j = torch.arange(most, device=held.device)
    table = s["table"].clone()
    # pages of sequences that end, in order, on top of the free ones
    stack = torch.cat([s["free"].long(), torch.zeros(1, dtype=torch.long, device=held.device)])
    given = ends[:, None] & (j[None, :] < have[:, None])
    at = count + (freed.cumsum(0) - freed)[:, None] + j[None, :]
    stack[torch.where(given, at.clamp(max=N), N)[given]] = table.long()[given]
    taken = (j[None, :] >= have[:, None]) & (j[None, :] < (have + need)[:, None])
    kth = (upto - need)[:, None] + j[None, :] - have[:, None]
    table = torch.where(taken, stack[(avail - 1 - kth).clamp(0, N)].to(torch.int32), table)
    left = avail - need.sum()
    free = torch.where(torch.arange(N, device=held.device) < left, stack[:N].to(torch.int32), s["free"])
    row = torch.arange(cap_rows, device=held.device)
    seq = torch.searchsorted(cu_end, row, right=True).clamp(max=c["n_seq"] - 1)
    pos = held[seq] + row - (cu_end - rows)[seq]
    live = served[seq] & (row < cu_end[-1])
    pg = table[seq, (pos // page).clamp(0, most - 1)].long()
    live = live & (pg >= 0) & (pg < N)
    slots = torch.where(live, pg * page + pos % page, -1).to(torch.int32)
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=held.device), cu_end]).to(torch.int32)
    after = torch.where(served, to, torch.where(ends, 0, held)).to(torch.int32)
    return {"lens": after, "cu": cu, "slots": slots, "table": table, "free": free, "free_count": left.to(torch.int32).reshape(1)}


def _attend_plain(s, dtype=torch.float32):
    c, lens = s["c"], s["host_lens"]
    n, q_len, Hq, Hk, d, page = c["n_seq"], c["q_len"], c["Hq"], c["Hk"], c["d"], c["page"]
    G = Hq // Hk
    dev = s["Q"].device
    out = torch.zeros(n, q_len, Hq, d, dtype=dtype, device=dev)
    lse = torch.full((Hq, n, q_len), float("-inf"), dtype=dtype, device=dev)
    first = 0
    while first < n:   # sequences whose padded keys fit together
        last = first + 1
        while last < n and (last + 1 - first) * max(lens[first:last + 1]) * Hk * d <= 1 << 29:
            last += 1
        nb = _cached_pages(max(lens[first:last]), page)
        if nb:
            m, L = last - first, nb * page
            table = s["table"][first:last, :nb].long().clamp(min=0)
            k, v = _page_values(s["cache"][table.reshape(-1)], page, d, dtype)
            k, v = (x.view(m, nb, Hk, page, d).transpose(1, 2).reshape(m, Hk, L, d) for x in (k, v))
            limit = s["lens"][first:last, None] - q_len + 1 + torch.arange(q_len, device=dev)[None, :]      # keys that a query sees
            pos = torch.arange(L, device=dev)
            v = torch.where((pos[None, :] < s["lens"][first:last, None])[:, None, :, None], v, 0.0)
            q = s["Q"].view(n, q_len, Hk, G, d)[first:last].to(dtype).permute(0, 2, 1, 3, 4).reshape(m, Hk, q_len * G, d)
            seen = (pos[None, None, :] < limit[:, :, None])[:, None, :, None, :].expand(m, 1, q_len, G, L).reshape(m, 1, q_len * G, L)
            S = torch.matmul(q, k.transpose(-1, -2)).masked_fill(~seen, float("-inf"))
            top = S.amax(-1, keepdim=True)
            top = torch.where(top == float("-inf"), 0.0, top)
            P = torch.exp(S - top)
            total = P.sum(-1, keepdim=True)
            O = torch.matmul(P, v) / torch.where(total > 0, total, 1.0)
            out[first:last] = O.view(m, Hk, q_len, G, d).permute(0, 2, 1, 3, 4).reshape(m, q_len, Hq, d)
            lse[:, first:last] = (top + torch.log(total)).view(m, Hk, q_len, G).permute(1, 3, 0, 2).reshape(Hq, m, q_len)
        first = last
    return out.view(n * q_len, Hq, d), lse.view(Hq, n * q_len)


def run(s):
    c = s["c"]
    if own:
        return _run_own(s)
    if c["kind"] in ("packed_fwd", "packed_train"):
        return _packed_plain(s)
    if c["kind"] == "plan":
        return _plan_plain(s)
    if c["kind"] == "rows":
        return {"K": _values(*_quantised(s["K"].float()), torch.float32).to(s["K"].dtype), "V": _values(*_quantised(s["V"].float()), torch.float32).to(s["V"].dtype)}
    out, lse = _attend_plain(s)
    return {"out": out.to(s["Q"].dtype), "lse": lse}


# ---------------------------------------------------------------- the framework's calls
def _run_own(s):
    import paper_2310_05869_amd as ha
    c = s["c"]
    if c["kind"] in ("packed_fwd", "packed_train"):
        ha.exact_attn_packed_forward(s["Q"], s["K"], s["V"], s["cu"], causal=c["causal"], out=s["out"], lse=s["lse"], out_f32=s.get("out_f32"))
        if c["kind"] == "packed_fwd":
            return {"out": s["out"], "lse": s["lse"]}
        dQ, dK, dV = ha.exact_attn_packed_backward(s["Q"], s["K"], s["V"], s["cu"], s["out"], s["lse"], s["d_out"], causal=c["causal"],
                                                   workspace=s["workspace"], grads=s["grads"], out_f32=s["out_f32"])
        return {"out": s["out"], "lse": s["lse"], "dQ": dQ, "dK": dK, "dV": dV}
    if c["kind"] == "plan":
        ha.ha_page_plan(s["lens"], s["add"], s["table"], s["free"], s["free_count"], c["page"], lens_out=s["lens_out"], cu_seqlens=s["cu"],
                        slots=s["slots"], free_count_out=s["free_count_out"])
        return {"lens": s["lens_out"], "cu": s["cu"], "slots": s["slots"], "table": s["table"], "free": s["free"], "free_count": s["free_count_out"]}
    if c["kind"] == "rows":
        ha.ha_cache4_write(s["K"], s["V"], s["slots"], s["cache"], c["page"])
        ha.ha_cache4_read(s["cache"], s["slots"], c["page"], K=s["K_back"], V=s["V_back"])
        return {"K": s["K_back"], "V": s["V_back"]}
    ha.ha_cache4_attn(s["Q"], s["cache"], s["table"], s["lens"], c["page"], q_len=c["q_len"], out=s["out"], lse=s["lse"], workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Packed: every tensor's live rows once, two products (4 d flop) per allowed pair and query head, seven (14 d) in training.  Plan: the numbers read and
    written.  Rows: rows in, pages out and in, rows out.  Attend: the sequences' pages once, queries and outputs."""
    c = case
    if c["kind"] in ("packed_fwd", "packed_train"):
        lens, d, esz = _lens(c), c["d"], 2 if c["dtype"] == "bf16" else 4
        pairs = sum(n * (n + 1) // 2 if c["causal"] else n * n for n in lens) * c["Hq"]
        T, train = sum(lens), c["kind"] == "packed_train"
        rows = T * d * esz * ((4 * c["Hq"] + 4 * c["Hk"]) if train else (2 * c["Hq"] + 2 * c["Hk"]))
        return {"bytes": rows + 4 * T * c["Hq"], "flops": pairs * d * (14 if train else 4)}
    if c["kind"] == "plan":
        held, add = _plan_numbers(c)
        moved = sum(_cached_pages(h, c["page"]) if a < 0 else _cached_pages(h + a, c["page"]) - _cached_pages(h, c["page"]) for h, a in zip(held, add))
        return {"bytes": 4 * (4 * c["n_seq"] + c["slots"] + 2 * moved + 3), "flops": 0}
    if c["kind"] == "rows":
        values = 2 * c["rows"] * c["Hk"] * c["d"]
        return {"bytes": values * 2 * (2 if c["dtype"] == "bf16" else 4) + 2 * values * 17 // 32 + 8 * c["rows"], "flops": 0}
    lens, d = _lens(c), c["d"]
    rows = c["n_seq"] * c["q_len"]
    pairs = sum(lens) * c["q_len"] * c["Hq"]
    return {"bytes": sum(lens) * c["Hk"] * _token_bytes(d) + rows * c["Hq"] * (2 * d * (2 if c["dtype"] == "bf16" else 4) + 4) + 4 * c["n_seq"],
            "flops": pairs * 4 * d}


# ---------------------------------------------------------------- 64 bits
def _exact_row_values(x):
    """What the cache holds of x [N, H, d], by distances to the sixteen values in 64 bits."""
    g = x.double().reshape(*x.shape[:-1], -1, CACHE_GROUP)
    most = g.abs().amax(-1, keepdim=True)
    s = 2.0 ** torch.ceil(torch.log2(most.clamp(min=1e-300) / 6))
    s = torch.where(most <= 3 * s, s / 2, torch.where(most > 6 * s, s * 2, s)).clamp(2.0 ** -125, 2.0 ** 125)   # log2's rounding
    steps = torch.tensor([0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0], dtype=torch.float64, device=x.device)   # even codes first: the nearest, ties to them
    which = ((g.abs() / s)[..., None] - steps).abs().argmin(-1)
    return (torch.sign(g) * steps[which] * s).reshape(x.shape)


def exact(case, seed):
    c = dict(case)
    if c["kind"] == "plan":
        return None
    s = prepare(c, seed)
    if c["kind"] == "rows":
        return {"K": _exact_row_values(s["K"]), "V": _exact_row_values(s["V"])}
    if c["kind"] == "attend":
        Hq, Hk, d, page, q_len = c["Hq"], c["Hk"], c["d"], c["page"], c["q_len"]
        out = torch.zeros(c["n_seq"] * q_len, Hq, d, dtype=torch.float64, device="cuda")
        lse = torch.full((Hq, c["n_seq"] * q_len), float("-inf"), dtype=torch.float64, device="cuda")
        for i, n in enumerate(s["host_lens"]):
            if n == 0:
                continue
            k, v = _page_values(s["cache"][s["table"][i, :_cached_pages(n, page)].long()], page, d, torch.float64)   # [blocks, Hk, page, d]
            for h in range(Hk):
                kh, vh = k[:, h].reshape(-1, d)[:n], v[:, h].reshape(-1, d)[:n]
                for j in range(max(0, q_len - n), q_len):
                    see = n - q_len + 1 + j
                    mine = slice(h * (Hq // Hk), (h + 1) * (Hq // Hk))
                    S = s["Q"][i * q_len + j, mine].double() @ kh[:see].T
                    lse[mine, i * q_len + j] = torch.logsumexp(S, -1)
                    out[i * q_len + j, mine] = torch.softmax(S, -1) @ vh[:see]
        return {"out": out, "lse": lse}
    Hq, Hk = c["Hq"], c["Hk"]
    out, lse = s["out"].double(), s["lse"].double()
    grads = [x.double() for x in s["grads"]] if c["kind"] == "packed_train" else None
    at = _starts(s["lens"])
    for a, b in zip(at[:-1], at[1:]):
        if a == b:
            continue
        hidden = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1) if c["causal"] else None
        for h in range(Hq):
            q, k, v = s["Q"][a:b, h].double(), s["K"][a:b, h * Hk // Hq].double(), s["V"][a:b, h * Hk // Hq].double()
            S = q @ k.T
            if hidden is not None:
                S.masked_fill_(hidden, float("-inf"))
            lse[h, a:b] = torch.logsumexp(S, -1)
            P = torch.softmax(S, -1)
            out[a:b, h] = P @ v
            if grads:
                g = s["d_out"][a:b, h].double()
                dP = g @ v.T
                dS = P * (dP - (P * dP).sum(-1, keepdim=True))
                grads[0][a:b, h] = dS @ k
                grads[1][a:b, h * Hk // Hq] += dS.T @ q
                grads[2][a:b, h * Hk // Hq] += P.T @ g
    r = {"out": out, "lse": lse}
    if grads:
        r.update(dQ=grads[0], dK=grads[1], dV=grads[2])
    return r
