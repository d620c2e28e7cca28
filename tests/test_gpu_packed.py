"""Attention over packed prompts, and over a paged cache of 8-bit codes with its planning and writing, against plain loops in
64 bits (packed_ref.py).

Tolerances, from arithmetic.  A score is a sum of d products in fp32, exact for bf16 and E4M3 operands: its error is at most
(d + 4) 2^-24 S, S = scale * sum |q||k| (the 4: scaling, and the exponent's argument); a weight's relative error is twice that
(weight and sum), plus 2^-20 for the exponential and the sum's roundings per 16 steps, here `delta`.  bf16: weights are rounded
to bf16 (2^-8 relative at most) for the product with the values, and the output is rounded to bf16 (2^-8 of it).  So
|o - o_ref| <= 2^-8 |o_ref| + (2^-8 + delta + n 2^-24) * 1.02 * sum w|v|;  fp32: the same without the 2^-8, 2^-24 |o_ref| for
the rounding.  Weights below 2^-126 of the row's largest are zero in the bf16 kernels (the exponential instruction has no subnormal
results), so that each of n keys may lack 2^-126 of its value: n 2^-126 max|v| more (peaked rows over codes reach that: an output
whose other values are zero was 2^-120).  lse: the largest score error, 2^-20 and 2^-22 of itself (logarithm, rounding).
Codes, scales, tables and slots are exact.
"""
import math

import numpy as np
import pytest
import torch

import packed_ref as ref
import paper_2602_01801_amd as fa

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prefix(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int64)


def check(O, lse, want, n, d, bf16, what=""):
    Or, lr, A, S, vmax = want
    o, l = f64(O), None if lse is None else f64(lse)
    delta = 2 * (d + 4) * 2.0 ** -24 * S[..., None] + 2.0 ** -20
    unit = 2.0 ** -8 if bf16 else 2.0 ** -24
    tol = unit * np.abs(Or) + ((2.0 ** -8 if bf16 else 0.0) + delta + n * 2.0 ** -24) * 1.02 * A + n * 2.0 ** -126 * vmax
    assert np.isfinite(o).all() == np.isfinite(Or).all(), what
    bad = ~(np.abs(o - Or) <= tol) & ~(np.isnan(o) & np.isnan(Or))
    assert not bad.any(), (what, np.argwhere(bad)[:4], o[bad][:4], Or[bad][:4], tol[bad][:4])
    if l is not None:
        with np.errstate(invalid="ignore"):
            tl = (d + 4) * 2.0 ** -24 * S + 2.0 ** -20 + n * 2.0 ** -24 + 2.0 ** -22 * np.abs(lr)
            ok = (np.abs(l - lr) <= tl) | (l == lr) | (np.isnan(l) & np.isnan(lr))
        assert ok.all(), (what, np.argwhere(~ok)[:4], l[~ok][:4], lr[~ok][:4])


def view(g, H, n, d, dtype, layout, mul=1.0):
    """[H, n, d] view of random values: head-major, token-major, or part of a fused projection's output."""
    x = torch.randn((n, H, d) if layout != "heads" else (H, n, d), generator=g) * mul
    if layout == "heads":
        return x.to(dtype).cuda()
    if layout == "tokens":
        return x.to(dtype).cuda().transpose(0, 1)
    buf = torch.full((n, H + 3, d), math.nan, dtype=dtype)
    buf[:, 1:H + 1] = x.to(dtype)
    return buf.cuda()[:, 1:H + 1].transpose(0, 1)


PROMPTS = [   # queries, keys (None: the same)
    ([1], None), ([2, 0, 31, 33], None), ([64, 65], None), ([127, 1, 129], None), ([300, 77, 200], None), ([515], None),
    ([5, 70, 3, 0], [9, 40, 0, 50]), ([257], [64]), ([130], [700]), ([1, 1, 1], [1, 129, 400]), ([0], [5]),
]


@pytest.mark.parametrize("q,k", PROMPTS, ids=lambda x: "-".join(map(str, x)) if x else "same")
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d,Hq,Hkv,layout", [("bf16", 128, 4, 2, "tokens"), ("bf16", 64, 3, 1, "fused"), ("bf16", 128, 5, 5, "heads"),
                                                   ("bf16", 64, 8, 8, "tokens"), ("f32", 128, 6, 2, "fused"), ("f32", 64, 2, 2, "heads")])
def test_prompt_attention(q, k, causal, dtype, d, Hq, Hkv, layout):
    g = torch.Generator().manual_seed(sum(q) * 31 + d + Hq)
    kk = q if k is None else k
    pad_q, pad_k = 3, 3 if k is None else 2   # rows in front of the first sequence and behind the last
    nq, nk = sum(q) + 2 * pad_q, sum(kk) + 2 * pad_k
    Q = view(g, Hq, nq, d, DT[dtype], layout, 1.5)
    K = view(g, Hkv, nk, d, DT[dtype], layout)
    V = view(g, Hkv, nk, d, DT[dtype], layout)
    for t, n, p in ((K, nk, pad_k), (V, nk, pad_k), (Q, nq, pad_q)):   # rows of nobody
        t[:, :p] = math.nan
        t[:, n - p:] = math.inf
    cq, ck = prefix(q) + pad_q, prefix(kk) + pad_k
    O = view(g, Hq, nq, d, DT[dtype], layout)
    O[:] = 7.0
    lse = torch.full((Hq, nq), 7.0, device="cuda")
    fa.prompt_attn_fwd(Q, K, V, i32(cq), None if k is None else i32(ck), causal=causal, out=(O, lse))
    for b in range(len(q)):
        i, j = slice(cq[b], cq[b + 1]), slice(ck[b], ck[b + 1])
        want = ref.attend(f64(Q[:, i]), f64(K[:, j]), f64(V[:, j]), causal, d ** -0.5)
        check(O[:, i], lse[:, i], want, kk[b], d, dtype == "bf16", f"sequence {b}")
    for t in (O, lse):
        assert (t[:, :cq[0]] == 7.0).all() and (t[:, cq[-1]:] == 7.0).all()


@pytest.mark.parametrize("dtype,d,Hq,Hkv,n", [("bf16", 128, 3, 1, 2200), ("bf16", 64, 2, 1, 1777), ("f32", 128, 2, 1, 900), ("bf16", 128, 8, 1, 1025)])
def test_prompt_attention_over_long_prompts(dtype, d, Hq, Hkv, n):
    g = torch.Generator().manual_seed(n)
    Q, K, V = (view(g, h, n, d, DT[dtype], "tokens", m) for h, m in ((Hq, 2.0), (Hkv, 1.0), (Hkv, 1.0)))
    K[:, n // 3: n // 3 + 40] *= 4     # maxima that climb in the middle
    O, lse = fa.prompt_attn_fwd(Q, K, V, i32([0, n]))
    check(O, lse, ref.attend(f64(Q), f64(K), f64(V), True, d ** -0.5), n, d, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
def test_what_a_query_does_not_see_does_not_reach_it(dtype, causal):
    """Keys and values of later tokens and of other sequences that are not finite."""
    g = torch.Generator().manual_seed(9)
    q = [150, 90, 70]
    n, d = sum(q), 128
    Q, K, V = (view(g, h, n, d, DT[dtype], "tokens") for h in (4, 2, 2))
    cu = prefix(q)
    bad = [cu[0] + 100, cu[2] + 69, cu[2] + 5]   # within a sequence; the last one's last and an early one
    for x, t in zip((math.nan, math.inf, -math.inf), bad):
        K[:, t], V[:, t] = x, x
    O, lse = fa.prompt_attn_fwd(Q, K, V, i32(cu), causal=causal)
    for b in range(3):
        i = slice(cu[b], cu[b + 1])
        with np.errstate(invalid="ignore", over="ignore"):
            want = ref.attend(f64(Q[:, i]), f64(K[:, i]), f64(V[:, i]), causal, d ** -0.5)
        a = q[b] if b == 1 else (100 if b == 0 else 5) if causal else 0   # queries that see nothing of it
        check(O[:, i][:, :a], lse[:, i][:, :a], [w[:, :a] for w in want[:4]] + [want[4]], q[b], d, dtype == "bf16", f"sequence {b}")
        if a < q[b]:
            assert not torch.isfinite(O[:, i][:, a:]).all(-1).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_a_query_does_not_see_does_not_reach_it_in_launches_that_fill_the_chip(dtype):
    g = torch.Generator().manual_seed(10)
    Hkv, Hq, n, d = 40, 80, 900, 128
    Q, K, V = (view(g, h, n, d, DT[dtype], "tokens") for h in (Hq, Hkv, Hkv))
    for h, t, x in ((0, 850, math.nan), (16, 500, math.inf), (39, 899, -math.inf)):
        K[h, t], V[h, t] = x, x
    O, lse = fa.prompt_attn_fwd(Q, K, V, i32([0, n]))
    for hq, t in ((1, 850), (32, 500), (79, 899), (10, 900)):
        k, v = f64(K[hq // 2:hq // 2 + 1]), f64(V[hq // 2:hq // 2 + 1])
        want = ref.attend(f64(Q[hq:hq + 1, :t]), k[:, :t], v[:, :t], True, d ** -0.5)
        check(O[hq:hq + 1, :t], lse[hq:hq + 1, :t], want, n, d, dtype == "bf16", f"head {hq}")
        assert not torch.isfinite(O[hq, t:]).all(-1).any()


def test_prompt_attention_with_shared_rows_and_extreme_scales():
    g = torch.Generator().manual_seed(11)
    n, d = 200, 128
    Q, K = view(g, 4, n, d, torch.bfloat16, "tokens"), view(g, 1, n, d, torch.bfloat16, "tokens")
    V = K[:, :1].expand(1, n, d)    # one value row for all keys: stride 0
    for scale in (2.0 ** -140, 1e-20, 3.0, 40.0):
        O, lse = fa.prompt_attn_fwd(Q, K, V, i32([0, n]), scale=scale)
        want = ref.attend(f64(Q), f64(K), f64(V), True, float(np.float32(scale)))
        check(O, lse, want, n, d, True, str(scale))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [256, 257, 300, 1100])
def test_prompt_attention_of_many_sequences(B, dtype):
    """More sequences than one look at the offsets takes, empty ones among them; without lse."""
    rng = np.random.default_rng(B)
    q = rng.integers(0, 4, size=B)
    q[rng.integers(0, B, size=3)] = (0, 37, 300)
    q[-1] = 5
    g = torch.Generator().manual_seed(B)
    n, d = int(q.sum()), 64
    Q, K, V = (view(g, h, n, d, DT[dtype], "tokens") for h in (3, 1, 1))
    cu = prefix(q)
    O, none = fa.prompt_attn_fwd(Q, K, V, i32(cu), want_lse=False)
    assert none is None
    Qh, Kh, Vh = f64(Q), f64(K), f64(V)
    for b in range(B):
        i = slice(cu[b], cu[b + 1])
        want = ref.attend(Qh[:, i], Kh[:, i], Vh[:, i], True, d ** -0.5)
        check(O[:, i], None, want, int(q[b]), d, dtype == "bf16", f"sequence {b}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,causal", [(900, True), (700, False), (2049, True)])
def test_prompt_attention_in_launches_that_fill_the_chip(n, causal, dtype):
    """As many heads as it takes for workgroups that are not split; a few rows checked."""
    g = torch.Generator().manual_seed(n)
    Hkv, Hq, d, elt = 40, 80, 128, DT[dtype]
    Q, K, V = (view(g, h, n, d, elt, "tokens", m) for h, m in ((Hq, 1.5), (Hkv, 1.0), (Hkv, 1.0)))
    O, lse = fa.prompt_attn_fwd(Q, K, V, i32([0, n]), causal=causal)
    for h in (0, 33, 79):
        k, v = f64(K[h // 2:h // 2 + 1]), f64(V[h // 2:h // 2 + 1])
        want = ref.attend(f64(Q[h:h + 1]), k, v, causal, d ** -0.5)
        check(O[h:h + 1], lse[h:h + 1], want, n, d, dtype == "bf16", f"head {h}")


def test_prompt_attention_of_rows_beyond_32_bit_offsets():
    n, pitch, d = 70000, 1 << 15, 128          # 4.6 GB of rows 64 KB apart
    big = torch.empty((n, pitch), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    big[:, :256] = torch.randn((n, 256), generator=g, device="cuda").bfloat16()
    K, V = big[:, :128].unsqueeze(0), big[:, 128:256].unsqueeze(0)
    Q = view(torch.Generator().manual_seed(4), 2, 3, d, torch.bfloat16, "tokens", 2.0)
    O, lse = fa.prompt_attn_fwd(Q, K, V, i32([0, 3]), i32([0, n]))
    check(O, lse, ref.attend(f64(Q), f64(K), f64(V), True, d ** -0.5), n, d, True)


# ------------------------------------------------------------------------------------------------ the paged cache


def random_pages(rng, n_pages, Hkv, P, d, nan_from=None):
    """Codes of every finite kind and scales of several powers of two, as numpy and on the device."""
    K = rng.integers(0, 256, size=(n_pages, Hkv, P // 16, d // 16, 16, 16)).astype(np.uint8)
    V = rng.integers(0, 256, size=K.shape).astype(np.uint8)
    for c in (K, V):   # mostly values around one
        c[...] = np.where(rng.random(c.shape) < 0.9, (c & 0x8F) | 0x30, c)
        c[(c & 127) == 127] = 0x30
    ks = 2.0 ** rng.integers(-2, 2, size=(n_pages, Hkv))
    vs = 2.0 ** rng.integers(-6, 7, size=(n_pages, Hkv))
    dev = fa.Pages(*(torch.from_numpy(x.astype(np.float32) if x.dtype == np.float64 else x).cuda() for x in (K, ks, V, vs)))
    return K, ks, V, vs, dev


def gather(code, scale, ids, n, tr):
    """[Hkv, n, d] float64 of a sequence; zeros for pages that do not exist."""
    n_pages = code.shape[0]
    rows = ref.VALUES[ref.rows_of_cells(code, tr)] * scale[:, :, None, None]
    out = np.stack([rows[p] if 0 <= p < n_pages else np.zeros_like(rows[0]) for p in ids], 1) if len(ids) else rows[:0].swapaxes(0, 1).reshape(code.shape[1], 0, 16, rows.shape[3])
    return out.reshape(code.shape[1], -1, rows.shape[3])[:, :n]


def paged_case(q, k, Hq, Hkv, P, d, causal, seed, bad=(), layout="tokens", poison=False):
    rng = np.random.default_rng(seed)
    per = [-(-x // P) for x in k]
    n_pages = sum(per) + 2
    K, ks, V, vs, dev = random_pages(rng, n_pages, Hkv, P, d)
    order = rng.permutation(n_pages)
    mp = max(max(per, default=1), 1) + 1
    table = rng.integers(-5, n_pages + 5, size=(len(q), mp)).astype(np.int32)   # beyond the length: anything
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    for b, j, x in bad:
        table[b, j] = x
    if poison:   # what lies behind a sequence on its last page is not a number
        for b, n in enumerate(k):
            if n % P:
                p = table[b, n // P]
                for code, tr in ((K, False), (V, True)):
                    rows = ref.rows_of_cells(code[p:p + 1], tr).copy()
                    rows[0, :, n % P:] = 0x7F
                    code[p:p + 1] = ref.cells_of_rows(rows, tr)
        dev = fa.Pages(*(torch.from_numpy(x.astype(np.float32) if x.dtype == np.float64 else x).cuda() for x in (K, ks, V, vs)))
    g = torch.Generator().manual_seed(seed)
    nq = sum(q) + 2
    Q = view(g, Hq, nq, d, torch.bfloat16, layout)
    cu = prefix(q) + 1
    O = view(g, Hq, nq, d, torch.bfloat16, layout)
    O[:] = 7.0
    lse = torch.full((Hq, nq), 7.0, device="cuda")
    ws = torch.full((fa.workspace_bytes(fa.OP_PAGED_ATTN, Hq, nq, 0),), 0xFF, dtype=torch.uint8, device="cuda")
    fa.paged_attn_fwd(Q, i32(cu), i32(k), i32(table), dev, causal=causal, out=(O, lse), ws=ws)
    for b in range(len(q)):
        i = slice(cu[b], cu[b + 1])
        ids = table[b, :per[b]]
        live = np.repeat([0 <= p < n_pages for p in ids], P)[:k[b]] if len(ids) else np.zeros(0, bool)
        want = ref.attend(f64(Q[:, i]), gather(K, ks, ids, k[b], False), gather(V, vs, ids, k[b], True), causal, d ** -0.5, live)
        check(O[:, i], lse[:, i], want, k[b], d, True, f"sequence {b}")
    for t in (O, lse):
        assert (t[:, :cu[0]] == 7.0).all() and (t[:, cu[-1]:] == 7.0).all()


TOKENS = [([1], [1]), ([1], [2]), ([1] * 4, [15, 16, 17, 64]), ([1] * 5, [63, 65, 0, 130, 1000]), ([1, 0, 1], [300, 40, 77]),
          ([2, 1, 7], [2, 500, 129]), ([3], [1]), ([17, 1], [40, 333]), ([70, 1, 140], [70, 900, 517]), ([300], [1300])]


@pytest.mark.parametrize("q,k", TOKENS, ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Hq,Hkv,P,d", [(4, 4, 16, 128), (10, 2, 64, 128), (6, 2, 32, 64), (16, 1, 64, 64), (24, 1, 16, 128)])
def test_paged_attention(q, k, causal, Hq, Hkv, P, d):
    paged_case(q, k, Hq, Hkv, P, d, causal, seed=sum(q) + 3 * sum(k) + P + d, poison=True)


@pytest.mark.parametrize("Hq,Hkv,P,d,q,k", [(2, 1, 64, 128, [1, 1], [20000, 3]), (5, 1, 16, 64, [1], [9001]), (2, 2, 32, 128, [4, 9], [7000, 4097]),
                                            (40, 8, 64, 128, [1] * 9, [1, 700, 64, 65, 2000, 3, 1999, 128, 5]), (4, 1, 64, 128, [130], [5000])])
def test_paged_attention_over_long_caches_in_pieces(Hq, Hkv, P, d, q, k):
    paged_case(q, k, Hq, Hkv, P, d, True, seed=sum(k), layout="heads")


@pytest.mark.parametrize("Hq,Hkv,P,d,q,k", [(8, 1, 16, 128, 1, 1500), (12, 12, 64, 128, 1, 700), (4, 1, 32, 64, 2, 333), (5, 1, 64, 128, 1, 9000),
                                            (6, 3, 16, 64, 4, 5000)])
def test_weights_of_few_rows_have_sixteen_bits(Hq, Hkv, P, d, q, k):
    """At most eight rows of a key head: what rounding to bf16 takes from a weight is rounded to bf16 again and multiplied too, so that
    2^-16 of it is missing instead of 2^-8 (or 2^-126 of the largest, where the rest is too small a number)."""
    rng = np.random.default_rng(k)
    per = -(-k // P)
    K, ks, V, vs, dev = random_pages(rng, per, Hkv, P, d)
    table = rng.permutation(per).astype(np.int32)[None]
    Q = view(torch.Generator().manual_seed(k), Hq, q, d, torch.bfloat16, "tokens")
    O, lse = fa.paged_attn_fwd(Q, i32([0, q]), i32([k]), i32(table), dev)
    Or, _, A, S, vmax = ref.attend(f64(Q), gather(K, ks, table[0], k, False), gather(V, vs, table[0], k, True), True, d ** -0.5)
    delta = 2 * (d + 4) * 2.0 ** -24 * S[..., None] + 2.0 ** -20
    tol = 2.0 ** -8 * np.abs(Or) + (2.0 ** -16 + delta + k * 2.0 ** -24) * 1.02 * A + 2 * k * 2.0 ** -126 * vmax
    assert (np.abs(f64(O) - Or) <= tol).all()


@pytest.mark.parametrize("P", [16, 32, 64])
def test_keys_on_pages_that_do_not_exist_are_left_out(P):
    n = 5 * P + 3
    paged_case([1, 3, 60], [n, n, n], 4, 2, P, 128, True, seed=P, bad=[(0, 1, -1), (0, 2, 2 ** 30), (1, 0, -2 ** 31), (1, 5, 10 ** 6), (2, 3, -7)])
    paged_case([1, 40], [2 * P, 2 * P], 4, 2, P, 64, True, seed=P + 1, bad=[(b, j, -1) for b in (0, 1) for j in (0, 1)])


@pytest.mark.parametrize("a,n,few,d", [(50, 100, 20, 128), (6, 90, 4, 128), (150, 2500, 100, 128), (7, 2600, 3, 128), (12, 2200, 11, 64), (90, 130, 45, 64)])
def test_paged_attention_of_codes_that_are_no_numbers_among_later_tokens(a, n, few, d):
    """Causal chunk: tokens `few` and on of the chunk hold NaN; the queries before do not see them.  Few rows and chunks, in one piece
    and in several."""
    rng = np.random.default_rng(4)
    P = 32
    per = -(-n // P)
    K, ks, V, vs, _ = random_pages(rng, per, 1, P, d)
    table = rng.permutation(per).astype(np.int32)[None]
    first = n - a + few
    for code, tr in ((K, False), (V, True)):
        rows = ref.rows_of_cells(code, tr).copy()
        for j in range(first, n):
            rows[table[0, j // P], :, j % P] = 0x7F
        code[...] = ref.cells_of_rows(rows, tr)
    dev = fa.Pages(*(torch.from_numpy(x.astype(np.float32) if x.dtype == np.float64 else x).cuda() for x in (K, ks, V, vs)))
    Q = view(torch.Generator().manual_seed(1), 2, a, d, torch.bfloat16, "tokens")
    O, lse = fa.paged_attn_fwd(Q, i32([0, a]), i32([n]), i32(table), dev)
    want = ref.attend(f64(Q), gather(K, ks, table[0], n, False), gather(V, vs, table[0], n, True), True, d ** -0.5)
    check(O[:, :few], lse[:, :few], [w[:, :few] for w in want[:4]] + [want[4]], n, d, True)
    assert torch.isnan(O[:, few:]).all()


def test_lengths_beyond_the_table_are_cut():
    rng = np.random.default_rng(6)
    K, ks, V, vs, dev = random_pages(rng, 3, 2, 16, 64)
    Q = view(torch.Generator().manual_seed(2), 2, 2, 64, torch.bfloat16, "heads")
    O, lse = fa.paged_attn_fwd(Q, i32([0, 1, 2]), i32([2 ** 31 - 1, -5]), i32([[1, 2], [0, 0]]), dev)
    want = ref.attend(f64(Q[:, :1]), gather(K, ks, [1, 2], 32, False), gather(V, vs, [1, 2], 32, True), True, 64 ** -0.5)
    check(O[:, :1], lse[:, :1], want, 32, 64, True)
    assert (O[:, 1] == 0).all() and torch.isneginf(lse[:, 1]).all()


@pytest.mark.parametrize("B,q,k", [(257, 1, 70), (300, 2, 2100), (1025, 1, 33), (260, 40, 300), (300, 13, 2300)])
def test_paged_attention_of_many_sequences(B, q, k):
    """More sequences than one look at the lengths takes; few rows and chunks, one launch and two."""
    rng = np.random.default_rng(B + k)
    qs, ks = rng.integers(0, q + 1, size=B), rng.integers(0, 60, size=B)
    qs[B // 2], ks[B // 2], qs[-1], ks[-1], qs[0] = q, k, q, k // 2, q
    if q > 8:
        qs[:] = np.maximum(qs, q - 3)    # rows on average decide on the kernel
    paged_case([int(x) for x in qs], [int(x) for x in ks], 4, 1, 16, 64, True, seed=B)


def test_paged_attention_and_writing_beyond_32_bit_offsets():
    """Pages whose codes lie beyond 4 GB, against the same ones in a small cache."""
    Hkv, P, d, n = 8, 64, 128, 700
    n_pages = 66000 + 11     # 65536 bytes of K each
    big = fa.Pages(*(torch.empty((n_pages, Hkv) + s, dtype=t, device="cuda") for s, t in (((4, 8, 16, 16), torch.uint8), ((), torch.float32)) * 2))
    small = fa.Pages.empty(11, Hkv, P, d)
    K, V = (view(torch.Generator().manual_seed(i), Hkv, n, d, torch.bfloat16, "tokens") for i in range(2))
    slot = torch.arange(n, dtype=torch.int32, device="cuda")
    fa.kv_pages_write(big, slot + 66000 * P, K, V)
    fa.kv_pages_write(small, slot, K, V)
    last = n // P * P   # the rest of the last page means nothing
    assert torch.equal(big.K8[66000:66010], small.K8[:10]) and torch.equal(big.V8[66000:66010], small.V8[:10]) and last == 640
    assert torch.equal(big.kscale[66000:], small.kscale) and torch.equal(big.vscale[66000:], small.vscale)
    for a in (1, 200):   # single tokens and chunks
        Q = view(torch.Generator().manual_seed(9), 16, a, d, torch.bfloat16, "tokens")
        table = torch.arange(11, dtype=torch.int32, device="cuda")[None]
        want = fa.paged_attn_fwd(Q, i32([0, a]), i32([n]), table, small)
        got = fa.paged_attn_fwd(Q, i32([0, a]), i32([n]), table + 66000, big)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ------------------------------------------------------------------------------------------------ planning


def run_plan(n_new, length, table, pool, free, P, n_tok, in_place):
    t, p = i32(table).reshape(len(n_new), -1) if n_new else torch.zeros((0, 3), dtype=torch.int32, device="cuda"), i32(pool)
    L, F = i32(length), i32([free])
    slot = torch.full((n_tok,), -9, dtype=torch.int32, device="cuda")
    z = lambda n: torch.full((n,), -9, dtype=torch.int32, device="cuda")
    out = (L if in_place else z(len(n_new)), F if in_place else z(1), z(len(n_new) + 1), slot, z(len(n_new)))
    fa.kv_pages_plan(i32(n_new), L, t, p, F, P, n_tok, out=out)
    want_t, want_p = [list(r) for r in table], list(pool)
    after, top, cu, slots, status = ref.plan(n_new, length, want_t, want_p, free, P, n_tok)
    assert out[0].tolist() == after and out[1].tolist() == [top] and out[2].tolist() == cu and out[4].tolist() == status
    assert t.tolist() == want_t and p.tolist() == want_p
    got = slot.tolist()
    assert got == [slots.get(i, -9) for i in range(n_tok)]


@pytest.mark.parametrize("B", [0, 1, 2, 64, 65, 1000, 1025, 2500])
@pytest.mark.parametrize("P", [16, 32, 64])
def test_plan(B, P):
    rng = np.random.default_rng(B + P)
    mp = 9
    length = [int(x) for x in rng.integers(0, 6 * P, size=B)]
    n_new = [int(x) for x in rng.choice([-1, 0, 1, 2, P, 3 * P + 1, 20 * P], size=B, p=[0.1, 0.1, 0.5, 0.1, 0.1, 0.07, 0.03])]
    held = [-(-x // P) for x in length]
    n_pages = sum(held) + max(3, B // 3)
    order = [int(x) for x in rng.permutation(n_pages)]
    table, at = [[-3] * mp for _ in range(B)], 0
    for b in range(B):
        table[b][:held[b]] = order[at:at + held[b]]
        at += held[b]
    pool = order[at:] + [-1] * at
    total = sum(max(x, 0) for x in n_new)
    for n_tok in (total, total + 7, max(total * 2 // 3, 1), 5000 + total):
        run_plan(n_new, length, table, pool, n_pages - at, P, n_tok, in_place=bool(n_tok & 1))


@pytest.mark.parametrize("in_place", [True, False])
def test_plan_of_many_tokens(in_place):
    """More slots than one workgroup writes, in place and not; some requests are refused, some end."""
    rng = np.random.default_rng(5)
    P, B, mp = 16, 70, 60
    length = [int(x) for x in rng.integers(0, 300, size=B)]
    n_new = [int(x) for x in rng.choice([-1, 0, 1, 200, 600], size=B)]
    held = [-(-x // P) for x in length]
    n_pages = sum(held) + 700
    order = [int(x) for x in rng.permutation(n_pages)]
    table, at = [[-3] * mp for _ in range(B)], 0
    for b in range(B):
        table[b][:held[b]] = order[at:at + held[b]]
        at += held[b]
    total = sum(max(x, 0) for x in n_new)
    assert total > 9000
    run_plan(n_new, length, table, order[at:] + [-1] * at, n_pages - at, P, total, in_place)


def test_plan_of_lengths_and_pools_that_make_no_sense():
    """Counts are cut to what the arrays hold; pages that do not exist give no slot."""
    run_plan([5, 2 ** 31 - 1, -7, 3], [-10, 5, 2 ** 31 - 1, 10], [[0, 1], [1, 2], [50, -4], [2 ** 30, 3]], [3, 1, 2, 0, 9, 9], 99, 16, 40, False)
    run_plan([4, 4], [0, 20], [[7, 7], [0, 1]], [5, 6, 7], -2, 16, 8, True)
    run_plan([1, 1], [15, 16], [[3, 3], [4, 4]], [-1, 77], 2, 16, 2, True)


# ------------------------------------------------------------------------------------------------ writing


def run_write(rng, runs, Hkv, P, d, dtype, layout, mag, spoil=None):
    """runs: (page, offset, rows) in the order of the array; None: a row without a slot."""
    n_pages = 1 + max(r[0] for r in runs if r)
    K, ks, V, vs, dev = random_pages(rng, n_pages, Hkv, P, d)
    slot = []
    for r in runs:
        slot += [rng.choice([-1, -2 ** 31, n_pages * P, 2 ** 31 - 1])] if r is None else [r[0] * P + r[1] + i for i in range(r[2])]
    n = len(slot)
    g = torch.Generator().manual_seed(int(rng.integers(1 << 30)))
    Kn, Vn = view(g, Hkv, n, d, DT[dtype], layout), view(g, Hkv, n, d, DT[dtype], layout)
    m = torch.from_numpy(2.0 ** rng.integers(-mag, mag + 1, size=(n,))).to(DT[dtype]).cuda()
    Kn *= m[None, :, None]
    Vn *= m.flip(0)[None, :, None]
    if spoil:
        spoil(Kn, Vn)
    for x, code, scale, tr in ((Kn, K, ks, False), (Vn, V, vs, True)):
        ref.write(code, scale, tr, f64(x), [int(s) for s in slot], P)
    fa.kv_pages_write(dev, i32([int(s) for s in slot]), Kn, Vn)
    for got, want in ((dev.K8, K), (dev.V8, V)):
        a, b = got.cpu().numpy(), want
        nan = (a & 127) == 127
        off = np.argwhere(np.where(nan, (b & 127) != 127, a != b))
        assert len(off) == 0, (len(off), off[:4], [(a[tuple(i)], b[tuple(i)]) for i in off[:4]])
    for got, want in ((dev.kscale, ks), (dev.vscale, vs)):
        assert np.array_equal(got.cpu().numpy().astype(np.float64), want)


@pytest.mark.parametrize("dtype,d,Hkv,layout", [("bf16", 128, 2, "tokens"), ("bf16", 64, 3, "fused"), ("f32", 128, 1, "heads"), ("f32", 64, 5, "tokens")])
@pytest.mark.parametrize("P", [16, 32, 64])
@pytest.mark.parametrize("mag", [0, 12, 40])
def test_write(P, dtype, d, Hkv, layout, mag):
    rng = np.random.default_rng(P + d + Hkv + mag)
    run_write(rng, [(0, 0, 1)], Hkv, P, d, dtype, layout, mag)
    run_write(rng, [(2, 0, P), (0, 0, P), (1, 0, P - 1)], Hkv, P, d, dtype, layout, mag)
    run_write(rng, [(3, P - 1, 1), (1, 5, 7), None, (0, 1, P - 1), (2, 0, 3), None, None, (5, P - 3, 3), (4, 9, 1)], Hkv, P, d, dtype, layout, mag)
    run_write(rng, [(p, int(rng.integers(0, P)), 1) for p in rng.permutation(70)], Hkv, P, d, dtype, layout, mag)
    # pages whose numbers follow one another are runs of their own
    run_write(rng, [(0, 3, P - 3), (1, 0, P), (2, 0, 5)], Hkv, P, d, dtype, layout, mag)


def test_write_of_values_at_the_ends_of_the_range():
    rng = np.random.default_rng(8)

    def spoil(K, V):
        K[:, 0], V[:, 1] = 0.0, 0.0
        K[:, 2, :3], V[:, 2, 4] = torch.tensor([math.inf, -math.inf, math.nan]).to(K), math.nan
        K[:, 3], V[:, 3] = 3.38e38, -3.38e38
        K[:, 4], V[:, 4] = 1e-39, 2.0 ** -110
        V[:, 5] = math.inf
        K[:, 6, 0], K[:, 6, 1:] = 448.0, 2.0 ** -10      # a tie with zero, and just above
        K[:, 7, 0], K[:, 7, 1:] = 448.0, 1.5 * 2.0 ** -10
        K[:, 8, 0], K[:, 8, 1:], V[:, 8] = 464.0, 232.0, 449.0
    for dtype in ("bf16", "f32"):
        run_write(rng, [(p, 0, 1) for p in range(9)], 2, 16, 64, dtype, "tokens", 0, spoil)
        run_write(rng, [(p, 7, 1) for p in range(9)], 2, 16, 128, dtype, "tokens", 0, spoil)
        run_write(rng, [(0, 0, 9)], 2, 16, 64, dtype, "tokens", 0, spoil)


# ------------------------------------------------------------------------------------------------ together


def serve(steps, graph=False):
    """Requests come, grow by chunks and single tokens, and end; the attention over the pages against the one over the values that
    the codes stand for, and prompts in one piece against both."""
    rng = np.random.default_rng(77)
    Hq, Hkv, d, P, B, mp = 6, 2, 128, 16, 5, 40
    n_pages = 60
    pages = fa.Pages.empty(n_pages, Hkv, P, d)
    table = torch.full((B, mp), -1, dtype=torch.int32, device="cuda")
    pool = torch.from_numpy(rng.permutation(n_pages).astype(np.int32)).cuda()
    length, pool_n = i32([0] * B), i32([n_pages])
    hold = [([], []) for _ in range(B)]     # what was written, per request
    refused = 0
    for step in range(steps):
        n_new = [int(rng.choice([33, 100, 257])) if not hold[b][0] else int(rng.choice([1, 1, 1, 1, 9, -1])) for b in range(B)]
        n_tok = sum(max(x, 0) for x in n_new)
        before = length.tolist()
        _, _, cu, slot, status = fa.kv_pages_plan(i32(n_new), length, table, pool, pool_n, P, n_tok,
                                                  out=(length, pool_n, i32([0] * (B + 1)), i32([0] * n_tok), i32([0] * B)))
        g = torch.Generator().manual_seed(step)
        qkv = (torch.randn((n_tok, Hq + 2 * Hkv, d), generator=g) * 1.2).bfloat16().cuda()
        Q, K, V = (x.transpose(0, 1) for x in qkv.split([Hq, Hkv, Hkv], 1))
        fa.kv_pages_write(pages, slot, K, V)
        O, lse = fa.paged_attn_fwd(Q, cu, length, table, pages)
        c, st = cu.tolist(), status.tolist()
        codes = [x.cpu().numpy() for x in (pages.K8, pages.kscale, pages.V8, pages.vscale)]
        for b in range(B):
            if n_new[b] < 0:
                hold[b] = ([], [])
                assert length[b] == 0
                continue
            if st[b]:
                refused += 1
                assert length[b] == before[b]
                continue
            i = slice(c[b], c[b + 1])
            hold[b][0].append(f64(K[:, i]))
            hold[b][1].append(f64(V[:, i]))
            n = int(length[b])
            kb, vb = np.concatenate(hold[b][0], 1), np.concatenate(hold[b][1], 1)
            assert n == kb.shape[1] == before[b] + n_new[b]
            ids = table[b, : -(-n // P)].tolist()
            k8, v8 = gather(codes[0], codes[1].astype(np.float64), ids, n, False), gather(codes[2], codes[3].astype(np.float64), ids, n, True)
            # a code is off by 2^-4 of the value, or half the least step (2^-10) of the page's scale, twice if it was carried over
            for x8, x, s in ((k8, kb, codes[1]), (v8, vb, codes[3])):
                assert (np.abs(x8 - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -9 * s.max()).all()
            check(O[:, i], lse[:, i], ref.attend(f64(Q[:, i]), k8, v8, True, d ** -0.5), n, d, True, f"step {step} request {b}")
            if before[b] == 0:
                Op, lp = fa.prompt_attn_fwd(Q[:, i], K[:, i], V[:, i], i32([0, n]))
                check(Op, lp, ref.attend(f64(Q[:, i]), kb, vb, True, d ** -0.5), n, d, True, f"prompt, step {step} request {b}")
    assert refused > 0


def test_requests_are_served():
    serve(14)


@pytest.mark.parametrize("Hq,Hkv,k", [(4, 2, [40, 3, 17]), (2, 1, [5000, 64, 900])])
def test_a_step_is_captured_and_replayed(Hq, Hkv, k):
    """Plan, write and attend in one graph; replays with eager work between them, each against the same calls made eagerly."""
    rng = np.random.default_rng(12)
    P, d, B = 16, 128, 3
    per = [-(-(x + 8) // P) + 1 for x in k]
    n_pages, mp = sum(per) + 4, max(per) + 2
    _, _, _, _, pages = random_pages(rng, n_pages, Hkv, P, d)
    order, table, at = rng.permutation(n_pages).astype(np.int32), np.full((B, mp), -1, np.int32), 0
    for b in range(B):
        n = -(-k[b] // P)
        table[b, :n] = order[at:at + n]
        at += n
    state = dict(table=i32(table), pool=i32(np.concatenate([order[at:], order[:at]])), length=i32(k), pool_n=i32([n_pages - at]),
                 n_new=i32([1] * B), pages=pages)
    Q, K, V = (view(torch.Generator().manual_seed(i), h, B, d, torch.bfloat16, "tokens") for i, h in enumerate((Hq, Hkv, Hkv)))
    ws = torch.empty(fa.workspace_bytes(fa.OP_PAGED_ATTN, Hq, B, 0), dtype=torch.uint8, device="cuda")
    O, lse = torch.empty_like(Q), torch.empty((Hq, B), device="cuda")
    plan_out = (state["length"], state["pool_n"], i32([0] * (B + 1)), i32([0] * B), i32([0] * B))

    def step(s, O, lse, out, ws):
        fa.kv_pages_plan(s["n_new"], s["length"], s["table"], s["pool"], s["pool_n"], P, B, out=out)
        fa.kv_pages_write(s["pages"], out[3], K, V)
        fa.paged_attn_fwd(Q, out[2], s["length"], s["table"], s["pages"], out=(O, lse), ws=ws)
        fa.prompt_attn_fwd(Q, K, V, out[2], out=(O2, lse2))

    O2, lse2 = torch.empty_like(Q), torch.empty_like(lse)
    clone = lambda s: {a: fa.Pages(*(x.clone() for x in (v.K8, v.kscale, v.V8, v.vscale))) if a == "pages" else v.clone() for a, v in s.items()}
    eager = clone(state)
    fa.init()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(state, O, lse, plan_out, ws)
    torch.cuda.synchronize()
    assert state["length"].tolist() == k   # captured, not run
    for i in range(5):
        for x in (Q, K, V):
            x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(100 + i)).bfloat16())
        graph.replay()
        got = [x.clone() for x in (O, lse, O2, lse2, state["length"], state["pages"].K8, state["pages"].V8, state["table"])]
        O_e, lse_e = torch.empty_like(O), torch.empty_like(lse)
        step(eager, O_e, lse_e, (eager["length"], eager["pool_n"], i32([0] * (B + 1)), i32([0] * B), i32([0] * B)), torch.empty_like(ws))
        torch.cuda.synchronize()
        for a, b in zip(got, (O_e, lse_e, O2, lse2, eager["length"], eager["pages"].K8, eager["pages"].V8, eager["table"])):
            assert torch.equal(a, b)


def test_calls_on_other_streams_with_a_workspace_each():
    rng = np.random.default_rng(3)
    _, _, _, _, dev = random_pages(rng, 300, 2, 64, 128)
    table = i32(rng.permutation(300).reshape(2, 150))
    Q = view(torch.Generator().manual_seed(1), 4, 2, 128, torch.bfloat16, "tokens")
    args = (i32([0, 1, 2]), i32([9600, 7000]), table, dev)
    want = fa.paged_attn_fwd(Q, *args)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            for _ in range(5):
                got.append(fa.paged_attn_fwd(Q, *args, ws=torch.empty(fa.workspace_bytes(fa.OP_PAGED_ATTN, 4, 2, 0), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for O, lse in got:
        assert torch.equal(O, want[0]) and torch.equal(lse, want[1])


def test_the_binding_refuses_what_does_not_fit():
    Q = torch.zeros((4, 8, 128), dtype=torch.bfloat16, device="cuda")
    K = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device="cuda")
    cu = i32([0, 8])
    with pytest.raises(ValueError):
        fa.prompt_attn_fwd(Q[:3], K, K, cu)
    with pytest.raises(ValueError):
        fa.prompt_attn_fwd(Q, K, K[:, :7], cu)
    with pytest.raises(ValueError):
        fa.prompt_attn_fwd(Q, K.transpose(1, 2).contiguous().transpose(1, 2), K, cu)
    with pytest.raises(TypeError):
        fa.prompt_attn_fwd(Q, K.float(), K, cu)
    with pytest.raises(TypeError):
        fa.prompt_attn_fwd(Q.half(), K.half(), K.half(), cu)
    with pytest.raises(TypeError):
        fa.prompt_attn_fwd(Q, K, K, cu.long())
    with pytest.raises(ValueError):
        fa.prompt_attn_fwd(Q, K, K, cu, i32([0, 4, 8]))
    with pytest.raises(ValueError):
        fa.prompt_attn_fwd(Q, K, K, cu, out=(Q[:, :4], None))
    with pytest.raises(fa.FastarError):
        fa.prompt_attn_fwd(Q, K, K, cu, scale=0.0)
    with pytest.raises(fa.FastarError):
        fa.prompt_attn_fwd(Q[..., :96], K[..., :96], K[..., :96], cu)
    pages = fa.Pages.empty(4, 2, 16, 128)
    with pytest.raises(ValueError):
        fa.paged_attn_fwd(Q[:3], cu, i32([8]), i32([[0]]), pages)
    with pytest.raises(ValueError):
        fa.paged_attn_fwd(Q, cu, i32([8, 8]), i32([[0]]), pages)
    with pytest.raises(fa.FastarError):
        fa.paged_attn_fwd(Q.float(), cu, i32([8]), i32([[0]]), pages)
    with pytest.raises(fa.FastarError):
        fa.paged_attn_fwd(Q, cu, i32([8]), i32([[0]]), pages, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        fa.kv_pages_write(pages, i32([0] * 7), K, K)
    with pytest.raises(ValueError):
        fa.Pages(pages.K8, pages.kscale[:2], pages.V8, pages.vscale)
    with pytest.raises(TypeError):
        fa.Pages(pages.K8, pages.kscale, pages.V8.view(torch.int8), pages.vscale)
    with pytest.raises(ValueError):
        fa.kv_pages_plan(i32([1]), i32([0, 0]), i32([[0]]), i32([0]), i32([1]), 16, 1)


def test_workspaces_that_do_not_fit_are_refused():
    """Nothing is launched."""
    Q, cu, length, table = torch.zeros((4, 8, 128), dtype=torch.bfloat16, device="cuda"), i32([0, 8]), i32([8]), i32([[0]])
    pages = fa.Pages.empty(4, 2, 16, 128)
    n = fa.workspace_bytes(fa.OP_PAGED_ATTN, 4, 8, 0)
    for ws in (torch.empty(n, dtype=torch.uint8), torch.empty((n, 2), dtype=torch.uint8, device="cuda")[:, 0]):
        with pytest.raises(ValueError):
            fa.paged_attn_fwd(Q, cu, length, table, pages, ws=ws)
    q = torch.zeros((1, 128, 32), dtype=torch.int8, device="cuda")
    with pytest.raises(ValueError):
        fa.ann_select_self(q, q, i32([128]), 128, 4, 64, 1, ws=torch.empty(1 << 20, dtype=torch.uint8))


# ------------------------------------------------------------------------------------------------ the ends of the range


def check_kinds(O, lse, want, n, d, bf16, what=""):
    """Infinities, NaN and finite numbers where the definition has them; the finite ones as everywhere."""
    Or, lr, A, S, vmax = want
    o = f64(O)
    for kind in (np.isnan, np.isposinf, np.isneginf):
        assert (kind(o) == kind(Or)).all(), (what, kind.__name__, np.argwhere(kind(o) != kind(Or))[:4], o[kind(o) != kind(Or)][:4])
    fin = np.isfinite(Or)
    assert (np.isfinite(S) | ~fin.any(-1)).all()   # a row without a bound has no finite output
    S = np.where(np.isfinite(S), S, 0.0)
    check(torch.from_numpy(np.where(fin, o, 0.0)), lse, (np.where(fin, Or, 0.0), lr, np.where(fin, A, 0.0), S, vmax), n, d, bf16, what)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,q", [(2, 5), (40, 420)])   # few workgroups, and launches that fill the chip
@pytest.mark.parametrize("n", [1, 17, 64, 70, 130])
def test_infinite_values_of_the_first_key(n, Hkv, q, dtype):
    """Tiles are filled up with the first key, at weight 0: infinite values of it made the sums no numbers, by the length modulo
    the tile."""
    g = torch.Generator().manual_seed(n)
    d, Hq = 128, 2 * Hkv
    Q, K, V = (view(g, h, m, d, DT[dtype], "tokens") for h, m in ((Hq, q), (Hkv, n), (Hkv, n)))
    V[:, 0, 3], V[:, 0, 70], V[:, 0, 127] = math.inf, -math.inf, math.nan
    V[:, n // 2, 5] = -math.inf
    O, lse = fa.prompt_attn_fwd(Q, K, V, i32([0, q]), i32([0, n]), causal=False)
    for h in {0, 1, Hq - 1}:
        with np.errstate(invalid="ignore"):
            want = ref.attend(f64(Q[h:h + 1]), f64(K[h // 2:h // 2 + 1]), f64(V[h // 2:h // 2 + 1]), False, d ** -0.5)
        check_kinds(O[h:h + 1], lse[h:h + 1], want, n, d, dtype == "bf16", f"head {h}")


def climbing(Hq, Hkv, q, n, d, at, octaves=7.5):
    """Scores of 0, and key `at` of so many octaves: Q, K and the scale."""
    Q, K = torch.zeros((Hq, q, d)), torch.zeros((Hkv, n, d))
    Q[:, :, 0], K[:, at, 0] = 8.0, octaves
    return Q, K, math.log(2.0) / 8


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Hkv,q", [(2, 5), (40, 420)])
def test_prompt_attention_of_large_values_under_climbing_scores(Hkv, q, causal, dtype):
    """A value of 2^121 under a key whose score is 7.5 octaves above those before it: its weight against the first tile's maximum
    is 181, and their product beyond the range."""
    n, d = 470, 128
    Q, K, scale = climbing(2 * Hkv, Hkv, q, n, d, at=40 if causal and q == 420 else 100)
    V = torch.randn((Hkv, n, d), generator=torch.Generator().manual_seed(1))
    V[:, 40 if causal and q == 420 else 100] = 2.0 ** 121
    Q, K, V = (x.to(DT[dtype]).cuda() for x in (Q, K, V))
    O, lse = fa.prompt_attn_fwd(Q, K, V, i32([0, q]), i32([0, n]), causal=causal, scale=scale)
    for h in {0, 2 * Hkv - 1}:
        want = ref.attend(f64(Q[h:h + 1]), f64(K[h // 2:h // 2 + 1]), f64(V[h // 2:h // 2 + 1]), causal, float(np.float32(scale)))
        assert np.isfinite(want[0]).all()
        check_kinds(O[h:h + 1], lse[h:h + 1], want, n, d, dtype == "bf16", f"head {h}")


def flat_pages(n, Hkv, P, d, seed, kexp=(-8, -6), vexp=(-8, -6)):
    """Pages of a sequence of n tokens in any order, with two that belong to nobody: codes from 1 to 448 of either sign, so that scores of ordinary queries
    spread by about one and the values by their sign; and the table."""
    rng = np.random.default_rng(seed)
    per = max(-(-n // P), 1)
    code = lambda: (rng.integers(0x38, 0x7F, size=(per + 2, Hkv, P // 16, d // 16, 16, 16)) | 128 * rng.integers(0, 2, size=(per + 2, Hkv, P // 16, d // 16, 16, 16))).astype(np.uint8)
    scale = lambda lo, hi: 2.0 ** rng.integers(lo, hi + 1, size=(per + 2, Hkv))
    return code(), scale(*kexp), code(), scale(*vexp), rng.permutation(per + 2)[:per].astype(np.int32)[None]


def on_device(K, ks, V, vs):
    return fa.Pages(*(torch.from_numpy(x.astype(np.float32) if x.dtype == np.float64 else x).cuda() for x in (K, ks, V, vs)))


PAGED_ENDS = [(40, 1, 16, 128, 1, 470), (40, 1, 64, 64, 1, 5000), (4, 2, 32, 128, 50, 470), (4, 1, 64, 128, 130, 9000)]   # chunks: rows > 32 each


@pytest.mark.parametrize("Hq,Hkv,P,d,q,n", PAGED_ENDS)
@pytest.mark.parametrize("causal", [False, True])
def test_paged_attention_of_large_values_under_climbing_scores(Hq, Hkv, P, d, q, n, causal):
    """As for prompts, over pages: a value of 2^121 from a code of 2 and a scale of 2^120."""
    K, ks, V, vs, table = flat_pages(n, Hkv, P, d, n)
    Q, _, scale = climbing(Hq, Hkv, q, n, d, 100)
    p, off = table[0, 100 // P], 100 % P
    rows = np.zeros((K.shape[0], Hkv, P, d), np.uint8)
    rows[p, :, off, 0] = ref.code_of(7.5)
    K, ks = ref.cells_of_rows(rows, False), np.ones_like(ks)
    rows = ref.rows_of_cells(V, True).copy()
    rows[p] = 0
    rows[p, :, off] = ref.code_of(2.0)
    V, vs[p] = ref.cells_of_rows(rows, True), 2.0 ** 120
    Q = Q.bfloat16().cuda()
    O, lse = fa.paged_attn_fwd(Q, i32([0, q]), i32([n]), i32(table), on_device(K, ks, V, vs), causal=causal, scale=scale)
    want = ref.attend(f64(Q), gather(K, ks, table[0], n, False), gather(V, vs, table[0], n, True), causal, float(np.float32(scale)))
    assert np.isfinite(want[0]).all()
    check_kinds(O, lse, want, n, d, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Hkv,q,n", [(2, 5, 3), (2, 5, 200), (1, 130, 1300), (40, 420, 470)])
def test_prompt_attention_of_values_whose_sums_leave_the_range(Hkv, q, n, causal, dtype):
    """Means of values between 2^126 and 2^128."""
    g = torch.Generator().manual_seed(n)
    d, Hq = 64, 2 * Hkv
    Q, K = view(g, Hq, q, d, DT[dtype], "tokens"), view(g, Hkv, n, d, DT[dtype], "tokens")
    V = ((torch.rand((Hkv, n, d), generator=g) + 1.0) * 2.0 ** 126 * 1.9).to(DT[dtype]).cuda()
    V[:, :, 7] *= -1
    O, lse = fa.prompt_attn_fwd(Q, K, V, i32([0, q]), i32([0, n]), causal=causal)
    for h in {0, Hq - 1}:
        want = ref.attend(f64(Q[h:h + 1]), f64(K[h // 2:h // 2 + 1]), f64(V[h // 2:h // 2 + 1]), causal, d ** -0.5)
        check_kinds(O[h:h + 1], lse[h:h + 1], want, n, d, dtype == "bf16", f"head {h}")


@pytest.mark.parametrize("Hq,Hkv,P,d,q,n", PAGED_ENDS + [(8, 2, 16, 128, 1, 300), (8, 1, 64, 64, 1, 20000), (6, 2, 32, 128, 7, 900), (12, 1, 16, 128, 2, 5000),
                                                         (40, 2, 64, 128, 1, 3)])
@pytest.mark.parametrize("causal", [False, True])
def test_paged_attention_of_values_whose_sums_leave_the_range(Hq, Hkv, P, d, q, n, causal):
    """Codes from 128 to 448 at a scale of 2^119; sums over fragments leave the range where those in a fragment do not, too."""
    K, ks, V, vs, table = flat_pages(n, Hkv, P, d, n)
    V = ((V & 0x07) | 0x70).astype(np.uint8)
    V[V == 0x77] = 0x7E
    vs[:] = 2.0 ** 119
    Q = view(torch.Generator().manual_seed(n), Hq, q, d, torch.bfloat16, "tokens")
    O, lse = fa.paged_attn_fwd(Q, i32([0, q]), i32([n]), i32(table), on_device(K, ks, V, vs), causal=causal)
    want = ref.attend(f64(Q), gather(K, ks, table[0], n, False), gather(V, vs, table[0], n, True), causal, d ** -0.5)
    assert np.isfinite(want[0]).all()
    check_kinds(O, lse, want, n, d, True)


def whole_scores(Hq, Hkv, q, n, d, top, sign):
    """Scores that are whole numbers: 0 to 3 (or -1 to -4), that of key `top` one more than all others."""
    rng = np.random.default_rng(n)
    s = rng.integers(0, 4, size=n)
    s[top] = 4
    if sign < 0:
        s -= 5
    Q, K = torch.zeros((Hq, q, d)), torch.zeros((Hkv, n, d))
    Q[:, :, 1], K[:, :, 1] = 1.0, torch.from_numpy(s).float()
    return Q, K, s


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("scale", [2.0 ** 36, 2.0 ** 90, 2.0 ** 125, 2.3e38])
@pytest.mark.parametrize("Hkv,q,n", [(2, 5, 200), (1, 3, 1), (40, 420, 470)])
def test_prompt_attention_with_scales_that_leave_one_key(Hkv, q, n, scale, sign, dtype):
    """Scales as large as they may be: scaled scores beyond the range, whose differences decide all the same."""
    d, top = 64, n - n // 3 - 1
    Q, K, s = whole_scores(2 * Hkv, Hkv, q, n, d, top, sign)
    V = torch.randn((Hkv, n, d), generator=torch.Generator().manual_seed(2))
    Q, K, V = (x.to(DT[dtype]).cuda() for x in (Q, K, V))
    O, lse = fa.prompt_attn_fwd(Q, K, V, i32([0, q]), i32([0, n]), causal=False, scale=scale)
    assert torch.equal(O, V[:, top].repeat_interleave(2, 0)[:, None].expand_as(O))
    want = float(s[top]) * float(np.float32(scale))
    got = f64(lse)
    assert (got == np.copysign(math.inf, want)).all() if abs(want) > 3.4028235e38 else (np.abs(got - want) <= 2.0 ** -22 * abs(want)).all()


@pytest.mark.parametrize("Hq,Hkv,P,d,q,n", PAGED_ENDS + [(8, 2, 16, 128, 1, 300), (8, 1, 64, 64, 1, 20000), (6, 2, 32, 128, 7, 900), (12, 1, 16, 128, 2, 5000)])
@pytest.mark.parametrize("sign,scale", [(1, 2.0 ** 36), (-1, 2.0 ** 36), (1, 2.0 ** 90), (-1, 2.0 ** 125), (1, 2.3e38), (-1, 2.3e38)])
def test_paged_attention_with_scales_that_leave_one_key(Hq, Hkv, P, d, q, n, sign, scale):
    top = n - n // 3 - 1
    Q, Kf, s = whole_scores(Hq, Hkv, q, n, d, top, sign)
    K, ks, V, vs, table = flat_pages(n, Hkv, P, d, n)
    rows = np.zeros((K.shape[0], Hkv, P, d), np.uint8)
    for j in range(n):
        rows[table[0, j // P], :, j % P] = ref.code_of(Kf[:, j].numpy().astype(np.float64))
    K, ks = ref.cells_of_rows(rows, False), np.ones_like(ks)
    O, lse = fa.paged_attn_fwd(Q.bfloat16().cuda(), i32([0, q]), i32([n]), i32(table), on_device(K, ks, V, vs), causal=False, scale=scale)
    v = gather(V, vs, table[0], n, True)[:, top]
    assert (f64(O) == np.repeat(v, Hq // Hkv, 0)[:, None]).all()
    want = float(s[top]) * float(np.float32(scale))
    got = f64(lse)
    assert (got == np.copysign(math.inf, want)).all() if abs(want) > 3.4028235e38 else (np.abs(got - want) <= 2.0 ** -22 * abs(want)).all()


@pytest.mark.parametrize("Hq,Hkv,P,d,q,n", PAGED_ENDS + [(8, 2, 16, 128, 1, 300), (8, 1, 64, 64, 1, 20000), (6, 2, 32, 128, 7, 900), (40, 2, 64, 128, 1, 200)])
@pytest.mark.parametrize("x", [math.nan, math.inf])
def test_the_scales_of_page_0_do_not_stand_in_for_those_of_pages_that_do_not_exist(Hq, Hkv, P, d, q, n, x):
    """Page 0 belongs to nobody and holds no numbers; two pages of the sequence do not exist."""
    K, ks, V, vs, table = flat_pages(n, Hkv, P, d, n)
    table[table == 0] = np.setdiff1d(np.arange(1, K.shape[0]), table)[0]
    table[0, 1], table[0, -1] = -1, 2 ** 30
    ks[0], vs[0], K[0], V[0] = x, x, 0x7F, 0x7F
    Q = view(torch.Generator().manual_seed(n), Hq, q, d, torch.bfloat16, "tokens")
    O, lse = fa.paged_attn_fwd(Q, i32([0, q]), i32([n]), i32(table), on_device(K, ks, V, vs))
    live = np.repeat([0 <= p < K.shape[0] for p in table[0]], P)[:n]
    want = ref.attend(f64(Q), gather(K, ks, table[0], n, False), gather(V, vs, table[0], n, True), True, d ** -0.5, live)
    check_kinds(O, lse, want, n, d, True)


@pytest.mark.parametrize("q", [1, 60])
def test_paged_attention_of_a_million_sequences_most_of_them_without_queries(q):
    """As many items as a launch cannot have workgroups for, had each its own."""
    B, Hkv, P, d = (1 << 20) + 3, 8, 16, 64
    rng = np.random.default_rng(q)
    K, ks, V, vs, dev = random_pages(rng, 5, Hkv, P, d)
    who = [0, 700001, B - 1]
    cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    length, table = torch.full((B,), 9, dtype=torch.int32, device="cuda"), torch.zeros((B, 1), dtype=torch.int32, device="cuda")
    for i, b in enumerate(who):
        cu[b + 1:] += q
        length[b], table[b] = 16 - i, 4 - i
    if q == 1:
        Q = view(torch.Generator().manual_seed(1), Hkv, len(who), d, torch.bfloat16, "tokens")
    else:   # rows of nobody, as many as it takes for the kernel of many rows; one query for all
        Q = view(torch.Generator().manual_seed(2), Hkv, 1, d, torch.bfloat16, "heads").expand(Hkv, 33 * B, d)
    O = torch.empty((Q.shape[1], Hkv, d), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    lse = torch.empty((Hkv, Q.shape[1]), device="cuda")
    fa.paged_attn_fwd(Q, cu, length, table, dev, causal=False, out=(O, lse))
    for i, b in enumerate(who):
        j = slice(i * q, (i + 1) * q)
        want = ref.attend(f64(Q[:, j]), gather(K, ks, [4 - i], 16 - i, False), gather(V, vs, [4 - i], 16 - i, True), False, d ** -0.5)
        check(O[:, j], lse[:, j], want, 16 - i, d, True, f"sequence {b}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_of_dimensions_of_one_mean_nothing(dtype):
    """What slicing a single row or head out of an odd buffer leaves behind."""
    g = torch.Generator().manual_seed(5)
    d, P, dt = 64, 16, DT[dtype]
    odd = lambda x, dim: x.as_strided(x.shape, [3 if i == dim else s for i, s in enumerate(x.stride())])
    Q, K, V = (torch.randn((h, 1, d), generator=g).to(dt).cuda() for h in (4, 2, 2))
    want = fa.prompt_attn_fwd(Q, K, V, i32([0, 1]))
    O = odd(torch.empty_like(Q), 1)
    fa.prompt_attn_fwd(odd(Q, 1), odd(K, 1), odd(V, 1), i32([0, 1]), out=(O, None))
    assert torch.equal(O, want[0])
    Q, K, V = (torch.randn((1, 40, d), generator=g).to(dt).cuda() for _ in range(3))
    want = fa.prompt_attn_fwd(Q, K, V, i32([0, 40]))
    got = fa.prompt_attn_fwd(odd(Q, 0), odd(K, 0), odd(V, 0), i32([0, 40]))
    assert torch.equal(got[0], want[0])
    pages = [fa.Pages.empty(3, 1, P, d) for _ in range(2)]
    slot = torch.arange(40, dtype=torch.int32, device="cuda")
    for pg, f in zip(pages, (lambda x, dim: x, odd)):
        fa.kv_pages_write(pg, slot, f(K, 0), f(V, 0))
        fa.kv_pages_write(pg, i32([40]), f(K[:, 3:4], 1), f(V[:, 3:4], 1))
    assert all(torch.equal(getattr(pages[0], x), getattr(pages[1], x)) for x in ("K8", "V8", "kscale", "vscale"))
    if dtype == "bf16":
        table = i32([[0, 1, 2]])
        want = fa.paged_attn_fwd(Q, i32([0, 40]), i32([41]), table, pages[0])
        assert torch.equal(fa.paged_attn_fwd(odd(Q, 0), i32([0, 40]), i32([41]), table, pages[0])[0], want[0])
        one = fa.paged_attn_fwd(Q[:, :1], i32([0, 1]), i32([41]), table, pages[0])
        assert torch.equal(fa.paged_attn_fwd(odd(Q[:, :1], 1), i32([0, 1]), i32([41]), table, pages[0])[0], one[0])


# ------------------------------------------------------------------------------------------------ data that shows a lost tile


SPREAD = [   # Hq, Hkv, P, d, queries, keys; at most 16 and 32 rows per key head, and more; whole and in pieces
    (2, 1, 64, 128, [1, 1], [9000, 3]), (5, 1, 16, 64, [1], [2100]), (10, 2, 32, 128, [1] * 4, [100, 1560, 64, 700]), (24, 1, 64, 128, [1, 1], [4097, 700]),
    (6, 2, 16, 128, [7, 5], [900, 2000]), (4, 1, 64, 64, [6, 8], [7000, 2200]), (4, 2, 32, 128, [60, 90], [300, 1200]), (4, 1, 64, 128, [130], [8200]),
    (3, 1, 16, 64, [100], [400])]


def spread_case(Hq, Hkv, P, d, q, k, seed):
    """Per sequence its pages and table, numbered on from those of the sequences before; queries [Hq, n, d]."""
    rng = np.random.default_rng(seed)
    parts, first = [], 0
    for n in k:
        K, ks, V, vs, table = ref.spread_pages(rng, n, Hkv, P, d=d)
        parts.append((K, ks, V, vs, table + first))
        first += K.shape[0]
    K, ks, V, vs = (np.concatenate([p[i] for p in parts]) for i in range(4))
    mp = max(len(p[4]) for p in parts) + 1
    table = np.full((len(k), mp), -1, np.int32)
    for b, p in enumerate(parts):
        table[b, :len(p[4])] = p[4]
    Q = torch.randn((sum(q), Hq, d), generator=torch.Generator().manual_seed(seed)).bfloat16().transpose(0, 1)
    return K, ks, V, vs, table, Q


@pytest.mark.parametrize("Hq,Hkv,P,d,q,k", SPREAD)
@pytest.mark.parametrize("causal", [True, False])
def test_paged_attention_of_rows_that_need_every_tile(Hq, Hkv, P, d, q, k, causal):
    """test_packed_host.py shows that losing or exchanging any tile of these would be seen."""
    K, ks, V, vs, table, Q = spread_case(Hq, Hkv, P, d, q, k, sum(k))
    O, lse = fa.paged_attn_fwd(Q.cuda(), i32(prefix(q)), i32(k), i32(table), on_device(K, ks, V, vs), causal=causal)
    for b, n in enumerate(k):
        i = slice(prefix(q)[b], prefix(q)[b + 1])
        want = ref.attend(f64(Q[:, i]), ref.keys_of_pages(K, ks, table[b, :-(-n // P)], n, False), ref.keys_of_pages(V, vs, table[b, :-(-n // P)], n, True), causal, d ** -0.5)
        check(O[:, i], lse[:, i], want, n, d, True, f"sequence {b}")


@pytest.mark.parametrize("Hq,Hkv,P,d,q,k", SPREAD + [(8, 1, 16, 64, [1, 1], [9000, 9000]), (8, 1, 32, 128, [3], [9000]), (4, 2, 64, 128, [70], [9000])])
@pytest.mark.parametrize("causal", [True, False])
def test_keys_on_runs_of_pages_that_do_not_exist_are_left_out(Hq, Hkv, P, d, q, k, causal):
    """Single pages, a run of them that is longer than a share of the tiles, the first and the last; and sequences without any page that exists."""
    K, ks, V, vs, table, Q = spread_case(Hq, Hkv, P, d, q, k, sum(k) + 1)
    for gone in ([lambda per: [0], lambda per: [per // 2, per - 1], lambda per: list(range(per // 3, max(2 * per // 3, 1)))], [lambda per: list(range(per))] * 3):
        t = table.copy()
        for b, n in enumerate(k):
            t[b, gone[(b + len(k)) % 3](-(-n // P))] = (-1, 2 ** 30, -2 ** 31, K.shape[0])[b % 4]
        O, lse = fa.paged_attn_fwd(Q.cuda(), i32(prefix(q)), i32(k), i32(t), on_device(K, ks, V, vs), causal=causal)
        for b, n in enumerate(k):
            i, ids = slice(prefix(q)[b], prefix(q)[b + 1]), t[b, :-(-n // P)]
            live = np.repeat([0 <= p < K.shape[0] for p in ids], P)[:n]
            want = ref.attend(f64(Q[:, i]), ref.keys_of_pages(K, ks, ids, n, False), ref.keys_of_pages(V, vs, ids, n, True), causal, d ** -0.5, live)
            check(O[:, i], lse[:, i], want, n, d, True, f"sequence {b}")


WEIGHTS16 = [(8, 1, 16, 128, 1, 100), (12, 12, 64, 128, 1, 64), (4, 1, 32, 64, 2, 40), (5, 1, 64, 128, 1, 160), (6, 3, 16, 64, 4, 99)]


def weights16_case(Hq, Hkv, P, d, q, k):
    """Even weights and values of 1 and 2 of either sign, which leave little of each other: an output is some per cent of what rounding a
    weight is relative to.  Returns the pages, the table, the queries, the 64-bit result and the bound of weights of 16 bits: 2^-16 of a weight may be missing."""
    rng = np.random.default_rng(k)
    K, ks, V, vs, table = ref.spread_pages(rng, k, Hkv, P, d=d)
    V = (V & 0x80 | 0x38).astype(np.uint8)
    vs[:] = 1.0
    Q = torch.randn((q, Hq, d), generator=torch.Generator().manual_seed(k)).bfloat16().transpose(0, 1)
    k64, v64 = ref.keys_of_pages(K, ks, table, k, False), ref.keys_of_pages(V, vs, table, k, True)
    Or, _, A, S, vmax = ref.attend(f64(Q), k64, v64, False, d ** -0.5)
    delta = 2 * (d + 4) * 2.0 ** -24 * S[..., None] + 2.0 ** -20
    tol = 2.0 ** -8 * np.abs(Or) + (2.0 ** -16 + delta + k * 2.0 ** -24) * 1.02 * A + 2 * k * 2.0 ** -126 * vmax
    return (K, ks, V, vs), table, Q, k64, v64, Or, tol


@pytest.mark.parametrize("Hq,Hkv,P,d,q,k", WEIGHTS16)
def test_even_weights_of_few_rows_have_sixteen_bits(Hq, Hkv, P, d, q, k):
    """test_packed_host.py shows that weights of 8 bits would be seen.  Tables as long as the sequence and of 4096 keys (two launches)."""
    pages, table, Q, _, _, Or, tol = weights16_case(Hq, Hkv, P, d, q, k)
    for t in (table, np.concatenate([table, np.full(4096 // P - len(table), -1, np.int32)])):
        O, _ = fa.paged_attn_fwd(Q.cuda(), i32([0, q]), i32([k]), i32(t[None]), on_device(*pages), causal=False)
        assert (np.abs(f64(O) - Or) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("large", [1.0, 2.0 ** 127])
@pytest.mark.parametrize("Hkv,q,n", [(2, 5, 200), (2, 5, 256), (40, 420, 470)])
def test_infinities_and_no_numbers_that_every_query_sees(Hkv, q, n, large, dtype):
    """Not causal: sums that are not finite stand, unless values are so large that they may have left the range by themselves."""
    g = torch.Generator().manual_seed(n)
    d, Hq = 128, 2 * Hkv
    Q, K = (view(g, h, m, d, DT[dtype], "tokens") for h, m in ((Hq, q), (Hkv, n)))
    V = ((torch.rand((Hkv, n, d), generator=g) + 1.0) * large * 0.99).to(DT[dtype]).cuda()
    V[:, 9, 3], V[:, 100, 4], V[:, 101, 5], V[:, 102, 5], V[:, n - 1, 77] = math.inf, math.nan, math.inf, -math.inf, -math.inf
    K[Hkv - 1, 150] = math.nan     # a head whose rows are no numbers at all
    O, lse = fa.prompt_attn_fwd(Q, K, V, i32([0, q]), i32([0, n]), causal=False)
    for h in (0, Hq - 1):
        with np.errstate(invalid="ignore"):
            want = ref.attend(f64(Q[h:h + 1]), f64(K[h // 2:h // 2 + 1]), f64(V[h // 2:h // 2 + 1]), False, d ** -0.5)
        check_kinds(O[h:h + 1], lse[h:h + 1], want, n, d, dtype == "bf16", f"head {h}")


@pytest.mark.parametrize("Hq,Hkv,P,d,q,n", PAGED_ENDS + [(8, 2, 16, 128, 1, 300), (8, 1, 64, 64, 1, 20000)])
@pytest.mark.parametrize("vexp", [0, 119])
def test_codes_that_are_no_numbers_and_every_query_sees(Hq, Hkv, P, d, q, n, vexp):
    K, ks, V, vs, table = flat_pages(n, Hkv, P, d, n)
    V = ((V & 0x07) | 0x70).astype(np.uint8)
    V[V == 0x77] = 0x7E
    vs[:] = 2.0 ** vexp
    rows = ref.rows_of_cells(V, True).copy()
    for j, c in ((9, 3), (n // 2, 40), (n - 1, 41)):
        rows[table[0, j // P], :, j % P, c] = 0x7F
    V = ref.cells_of_rows(rows, True)
    Q = view(torch.Generator().manual_seed(n), Hq, q, d, torch.bfloat16, "tokens")
    O, lse = fa.paged_attn_fwd(Q, i32([0, q]), i32([n]), i32(table), on_device(K, ks, V, vs), causal=False)
    want = ref.attend(f64(Q), gather(K, ks, table[0], n, False), gather(V, vs, table[0], n, True), False, d ** -0.5)
    check_kinds(O, lse, want, n, d, True)
