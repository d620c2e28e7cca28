"""Norm and rotation of queries and keys (qk_norm_rope), and the same on the way into pages (kv_pages_write_rope), against 64 bits
(share_ref.py: the definitions, and the tolerances with their arithmetic)."""
import math

import numpy as np
import pytest
import torch

import packed_ref as ref
import paper_2602_01801_amd as fa
import share_ref as sref
from test_gpu_packed import DT, f64, i32, prefix, view

pytestmark = pytest.mark.gpu


def weights(g, d):
    return (1 + 0.3 * torch.randn(d, generator=g)).cuda()


def make_rope(g, d, rot, norm=True, interleaved=False, axes=1, eps=1e-6, weighted=True):
    freq = sref.frequencies(rot)
    axis = np.arange(rot // 2) % axes
    r = fa.Rope(torch.from_numpy(freq).cuda() if rot else None, axis=i32(axis.tolist()) if rot and axes > 1 else None, n_axes=axes, norm=norm,
                q_weight=weights(g, d) if weighted else None, k_weight=weights(g, d) if weighted else None, eps=eps, interleaved=interleaved)
    return r, freq, axis


def check_rows(got, x, w, rope, freq, at, bf16, what=""):
    """got, x [H, n, d]; at [n, rot/2] positions."""
    y, size = sref.rope(f64(x).transpose(1, 0, 2), None if w is None else f64(w), float(np.float32(rope.eps)), rope.norm, freq, at, rope.rot, rope.interleaved)
    got = f64(got).transpose(1, 0, 2)
    tol = sref.rope_tol(y, size, freq, at, bf16)
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(got - y) <= tol) & ~(np.isnan(got) & np.isnan(y)) & ~(got == y)
    assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], y[bad][:4], tol[bad][:4])


SHAPES = [   # new tokens, tokens before them
    ([1], [0]), ([1], [200000]), ([3, 0, 1, 17], [0, 9, 1559, 30]), ([64, 65, 1], [3, 0, 260000]), ([130], [7]), ([1] * 67, list(range(67))),
]


@pytest.mark.parametrize("q,k", SHAPES, ids=lambda x: "-".join(map(str, x[:5])))
@pytest.mark.parametrize("dtype,d,Hq,Hkv,layout,rot,norm,interleaved", [
    ("bf16", 128, 4, 2, "tokens", 128, True, False), ("bf16", 128, 5, 3, "fused", 128, True, True), ("bf16", 64, 9, 1, "heads", 64, True, False),
    ("bf16", 64, 3, 3, "fused", 48, False, True), ("bf16", 128, 40, 8, "fused", 32, True, False), ("f32", 128, 6, 2, "fused", 128, True, False),
    ("f32", 64, 2, 2, "heads", 64, True, True), ("f32", 128, 1, 1, "tokens", 96, False, False), ("f32", 64, 12, 4, "tokens", 16, True, False),
    ("bf16", 128, 7, 2, "tokens", 0, True, False), ("f32", 64, 1, 5, "tokens", 0, False, False)])
def test_norm_and_rotation(q, k, dtype, d, Hq, Hkv, layout, rot, norm, interleaved):
    g = torch.Generator().manual_seed(sum(q) * 7 + d + rot)
    pad, n = 3, sum(q) + 6
    Q, K = view(g, Hq, n, d, DT[dtype], layout, 2.0), view(g, Hkv, n, d, DT[dtype], layout)
    for t in (Q, K):   # rows of nobody
        t[:, :pad], t[:, n - pad:] = math.nan, math.inf
    rope, freq, _ = make_rope(g, d, rot, norm, interleaved)
    out = view(g, Hq, n, d, DT[dtype], layout), view(g, Hkv, n, d, DT[dtype], "heads")
    for o in out:
        o[:] = 7.0
    cu = prefix(q) + pad
    fa.qk_norm_rope(Q, K, rope, cu=i32(cu.tolist()), length=i32([a + b for a, b in zip(q, k)]), out=out)
    at = np.concatenate([b + np.arange(a) for a, b in zip(q, k)])[:, None].astype(float) * np.ones(rot // 2)
    rows = slice(pad, n - pad)
    for o, x, w in ((out[0], Q, rope.q_weight), (out[1], K, rope.k_weight)):
        check_rows(o[:, rows], x[:, rows], w, rope, freq, at, dtype == "bf16")
        assert (o[:, :pad] == 7.0).all() and (o[:, n - pad:] == 7.0).all()
        if rot < d and not norm:
            assert torch.equal(o[:, rows, rot:], x[:, rows, rot:])


@pytest.mark.parametrize("dtype,interleaved,axes", [("bf16", False, 3), ("f32", True, 3), ("f32", False, 4), ("bf16", True, 2), ("f32", False, 1)])
def test_positions_on_several_axes(dtype, interleaved, axes):
    g = torch.Generator().manual_seed(axes)
    d, n, rng = 128, 77, np.random.default_rng(axes)
    Q, K = view(g, 3, n, d, DT[dtype], "tokens"), view(g, 2, n, d, DT[dtype], "fused")
    rope, freq, axis = make_rope(g, d, 96, True, interleaved, axes)
    pos = rng.integers(-500, 5000, size=(axes, n))
    oq, ok = fa.qk_norm_rope(Q, K, rope, pos=i32(pos.tolist()))
    at = pos[axis].T.astype(float)
    check_rows(oq, Q, rope.q_weight, rope, freq, at, dtype == "bf16")
    check_rows(ok, K, rope.k_weight, rope, freq, at, dtype == "bf16")
    # rows outside of the sequences stay, with positions of their own too
    out = torch.full_like(Q, 5.0), torch.full_like(K, 5.0)
    fa.qk_norm_rope(Q, K, rope, pos=i32(pos.tolist()), cu=i32([4, 20, 60]), out=out)
    assert torch.equal(out[0][:, 4:60], oq[:, 4:60]) and torch.equal(out[1][:, 4:60], ok[:, 4:60])
    assert all((o[:, :4] == 5.0).all() and (o[:, 60:] == 5.0).all() for o in out)
    # either alone, and in place
    assert torch.equal(fa.qk_norm_rope(Q, None, rope, pos=i32(pos.tolist()))[0], oq)
    assert torch.equal(fa.qk_norm_rope(None, K, rope, pos=i32(pos.tolist()))[1], ok)
    fa.qk_norm_rope(Q, K, rope, pos=i32(pos.tolist()), out=(Q, K))
    assert torch.equal(Q, oq) and torch.equal(K, ok)


def test_positions_at_the_ends_of_the_range():
    g = torch.Generator().manual_seed(3)
    d, pos = 64, [0, -1, 1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 999983]
    Q = view(g, 2, len(pos), d, torch.float32, "tokens")
    rope, freq, _ = make_rope(g, d, 64, False)
    out = fa.qk_norm_rope(Q, None, rope, pos=i32([pos]))[0]
    check_rows(out, Q, None, rope, freq, np.array(pos, float)[:, None] * np.ones(32), False)
    assert torch.equal(out[:, 0], Q[:, 0])   # no turn


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6])
def test_rows_of_any_magnitude(dtype, eps):
    """Squares that leave the range of 32 bits, in either direction, beside ordinary rows."""
    g = torch.Generator().manual_seed(4)
    d, mags = 128, [1.0, 1e-30, 1e30, 1e-38, 1e37, 1e-15, 1e19, 3e-20, 1.0, 1e-45]
    Q = view(g, 5, len(mags), d, torch.float32, "tokens")
    Q *= torch.tensor(mags, device="cuda")[None, :, None]
    Q = Q.to(DT[dtype])
    rope, freq, _ = make_rope(g, d, 64, True, eps=eps)
    out = fa.qk_norm_rope(Q, None, rope, pos=i32([list(range(len(mags)))]))[0]
    check_rows(out, Q, rope.q_weight, rope, freq, np.arange(len(mags), dtype=float)[:, None] * np.ones(32), dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_numbers_that_are_not_finite_stay_in_their_rows(dtype):
    g = torch.Generator().manual_seed(5)
    d, n = 64, 12
    Q = view(g, 3, n, d, DT[dtype], "tokens")
    rope, freq, _ = make_rope(g, d, 64, True)
    clean = fa.qk_norm_rope(Q, None, rope, pos=i32([list(range(n))]))[0]
    Q[0, 3, 5], Q[1, 3, 40], Q[2, 7, 0], Q[0, 8] = math.nan, math.inf, -math.inf, 0.0
    out = fa.qk_norm_rope(Q, None, rope, pos=i32([list(range(n))]))[0]
    assert torch.isnan(out[0, 3]).all()                       # the norm is none
    for h, t, c in ((1, 3, 40), (2, 7, 0)):                   # infinite: the others of the row are divided by infinity
        pair = c % 32
        other = [i for i in range(d) if i % 32 != pair]
        assert (out[h, t, other] == 0).all() and torch.isnan(out[h, t, [pair, pair + 32]]).all()
    assert (out[0, 8] == 0).all()
    touched = torch.zeros(3, n, dtype=torch.bool)
    for h, t in ((0, 3), (1, 3), (2, 7), (0, 8)):
        touched[h, t] = True
    assert torch.equal(out[~touched.cuda()], clean[~touched.cuda()])
    Z = torch.zeros_like(Q)
    assert torch.isnan(fa.qk_norm_rope(Z, None, make_rope(g, d, 64, True, eps=0.0)[0], pos=i32([list(range(n))]))[0]).all()


def test_many_sequences_and_heads():
    """More sequences than one look finds, empty ones among them; heads that leave lanes over."""
    g = torch.Generator().manual_seed(6)
    rng = np.random.default_rng(6)
    q = rng.choice([0, 1, 1, 2, 5], size=9000).tolist()
    k = rng.integers(0, 9999, size=9000).tolist()
    n, d = sum(q), 64
    Q, K = view(g, 3, n, d, torch.bfloat16, "tokens"), view(g, 1, n, d, torch.bfloat16, "tokens")
    rope, freq, _ = make_rope(g, d, 64)
    oq, ok = fa.qk_norm_rope(Q, K, rope, cu=i32(prefix(q).tolist()), length=i32([a + b for a, b in zip(q, k)]))
    at = np.concatenate([b + np.arange(a) for a, b in zip(q, k)])[:, None].astype(float) * np.ones(32)
    check_rows(oq, Q, rope.q_weight, rope, freq, at, True)
    check_rows(ok, K, rope.k_weight, rope, freq, at, True)


def test_more_heads_than_a_wavefront_takes():
    """264 heads of 64 and 4100 tokens, some rows of magnitudes that are done again; the same in place."""
    g = torch.Generator().manual_seed(13)
    Hq, n, d = 264, 4100, 64
    Q = torch.randn((n, Hq, d), generator=g).bfloat16().cuda()
    rows = [0, 1, 77, 2050, 4099]
    for r in rows:
        Q[r, ::3] *= 1e30
        Q[r, 1::7] *= 1e-30
    rope, freq, _ = make_rope(g, d, 32, True)
    pos = i32([list(range(n))])
    Q = Q.transpose(0, 1)
    out = fa.qk_norm_rope(Q, None, rope, pos=pos)[0]
    some = rows + [5, 1000, 3333]
    check_rows(out[:, some], Q[:, some], rope.q_weight, rope, freq, np.array(some, float)[:, None] * np.ones(16), True)
    fa.qk_norm_rope(Q, None, rope, pos=pos, out=(Q, None))
    assert torch.equal(Q, out)


@pytest.mark.parametrize("weight", [1e-25, 1e25])
def test_in_place_rows_are_done_once(weight):
    """Rows whose outputs would be done again if they were inputs."""
    g = torch.Generator().manual_seed(14)
    d, n = 128, 9
    Q = view(g, 6, n, d, torch.float32, "tokens")
    Q[:, 4] *= 1e30
    rope = fa.Rope(torch.from_numpy(sref.frequencies(d)).cuda(), q_weight=weights(g, d) * weight)
    out = fa.qk_norm_rope(Q, None, rope, pos=i32([list(range(n))]))[0]
    fa.qk_norm_rope(Q, None, rope, pos=i32([list(range(n))]), out=(Q, None))
    assert torch.equal(Q, out) and torch.isfinite(Q).all()


# ------------------------------------------------------------------------------------------------ into pages


def make_pages(rng, n_pages, Hkv, P, d):
    shape = (n_pages, Hkv, P // 16, d // 16, 16, 16)
    code = lambda: torch.from_numpy((rng.integers(0, 0x7F, shape) | 128 * rng.integers(0, 2, shape)).astype(np.uint8)).cuda()
    scale = lambda: torch.from_numpy(2.0 ** rng.integers(-9, -4, (n_pages, Hkv))).float().cuda()
    return fa.Pages(code(), scale(), code(), scale())


def clone(p):
    return fa.Pages(p.K8.clone(), p.kscale.clone(), p.V8.clone(), p.vscale.clone())


def slots_of(rng, q, k, P, spare=2):
    per = [-(-(a + b) // P) - b // P for a, b in zip(q, k)]
    order, slot, at = rng.permutation(sum(per) + spare), [], 0
    for a, b, m in zip(q, k, per):
        slot += [int(order[at + (b % P + i) // P] * P + (b + i) % P) for i in range(a)]
        at += m
    return slot, sum(per) + spare


WRITES = [([1], [0]), ([1, 1, 1], [15, 16, 77]), ([5, 0, 40], [0, 3, 9]), ([100, 64], [30, 0]), ([1] * 40, list(range(40))), ([300], [0])]


@pytest.mark.parametrize("q,k", WRITES, ids=lambda x: "-".join(map(str, x[:5])))
@pytest.mark.parametrize("dtype,d,Hq,Hkv,layout,P,rot,norm,interleaved", [
    ("bf16", 128, 4, 2, "fused", 64, 128, True, False), ("bf16", 128, 3, 3, "tokens", 16, 64, True, True), ("bf16", 64, 8, 1, "heads", 32, 64, False, False),
    ("f32", 128, 2, 2, "fused", 32, 128, True, False), ("f32", 64, 5, 5, "tokens", 64, 48, True, False), ("bf16", 64, 2, 2, "fused", 16, 64, True, True),
    ("f32", 128, 0, 1, "heads", 16, 96, True, True), ("bf16", 128, 1, 1, "tokens", 32, 0, True, False)])
def test_write_rope_is_both_calls_in_32_bits(q, k, dtype, d, Hq, Hkv, layout, P, rot, norm, interleaved):
    """The codes and scales of qk_norm_rope in fp32 and kv_pages_write of its output; Q of qk_norm_rope.  Rows of nobody have slots."""
    g = torch.Generator().manual_seed(sum(q) + rot + d)
    rng = np.random.default_rng(sum(q) + P)
    pad, n = 2, sum(q) + 4
    slot, n_pages = slots_of(rng, q, k, P)
    lost = n_pages * P - 1   # of rows in front of the first sequence and behind the last one
    Q = view(g, Hq, n, d, DT[dtype], layout) if Hq else None
    K, V = view(g, Hkv, n, d, DT[dtype], layout, 3.0), view(g, Hkv, n, d, DT[dtype], layout, 0.2)
    rope, freq, _ = make_rope(g, d, rot, norm, interleaved)
    cu, length = i32((prefix(q) + pad).tolist()), i32([a + b for a, b in zip(q, k)])
    pages = make_pages(rng, n_pages, Hkv, P, d)
    want = clone(pages)
    out = None if Q is None else torch.full_like(Q, 7.0)
    fa.kv_pages_write_rope(pages, i32([lost] * pad + slot + [lost] * pad), Q, K, V, rope, cu=cu, length=length, out=out)
    K32, V32 = K.float(), V.float()
    turned = fa.qk_norm_rope(None, K32, rope, cu=cu, length=length)[1]
    fa.kv_pages_write(want, i32([-1] * pad + slot + [-1] * pad), turned, V32)
    for name in ("K8", "kscale", "V8", "vscale"):
        assert torch.equal(getattr(pages, name), getattr(want, name)), name
    if Q is not None:
        both = torch.full_like(Q, 7.0)
        fa.qk_norm_rope(Q, None, rope, cu=cu, length=length, out=(both, None))
        assert torch.equal(out, both)
    # and against 64 bits: the new keys' values within half a step of theirs
    at = np.concatenate([b + np.arange(a) for a, b in zip(q, k)])[:, None].astype(float) * np.ones(rot // 2)
    y, size = sref.rope(f64(K).transpose(1, 0, 2)[pad:n - pad], f64(rope.k_weight), float(np.float32(rope.eps)), norm, freq, at, rot, interleaved)
    tol = sref.rope_tol(y, size, freq, at, False)
    rows = ref.VALUES[ref.rows_of_cells(pages.K8.cpu().numpy(), False)]
    scale = f64(pages.kscale)
    for t, s in enumerate(slot):
        v, sc = rows[s // P, :, s % P], scale[s // P][:, None]
        assert (np.abs(v * sc - y[t]) <= np.maximum(2.0 ** -4 * np.abs(y[t]), 2.0 ** -10 * sc) + 1.1 * tol[t]).all(), t


@pytest.mark.parametrize("dtype,d,P", [("bf16", 128, 64), ("f32", 64, 16), ("bf16", 64, 32)])
def test_write_rope_of_numbers_that_are_not_finite(dtype, d, P):
    g = torch.Generator().manual_seed(8)
    rng = np.random.default_rng(8)
    q, k = [70, 1, 20], [5, 30, 0]
    n, Hkv = sum(q), 2
    slot, n_pages = slots_of(rng, q, k, P)
    K, V = view(g, Hkv, n, d, DT[dtype], "tokens"), view(g, Hkv, n, d, DT[dtype], "tokens")
    K[0, 3, 7], K[1, 40, 1], K[0, 70, d - 1], K[1, 75] = math.nan, math.inf, -math.inf, math.inf
    V[1, 9, 2] = math.inf
    for norm in (True, False):
        rope, _, _ = make_rope(g, d, d, norm)
        cu, length = i32(prefix(q).tolist()), i32([a + b for a, b in zip(q, k)])
        pages = make_pages(rng, n_pages, Hkv, P, d)
        want = clone(pages)
        fa.kv_pages_write_rope(pages, i32(slot), None, K, V, rope, cu=cu, length=length)
        fa.kv_pages_write(want, i32(slot), fa.qk_norm_rope(None, K.float(), rope, cu=cu, length=length)[1], V.float())
        for name in ("K8", "V8"):   # NaN has one code of either sign
            a, b = getattr(pages, name), getattr(want, name)
            assert torch.equal(torch.where(a & 127 == 127, 127, a), torch.where(b & 127 == 127, 127, b)), name
        assert torch.equal(pages.kscale, want.kscale) and torch.equal(pages.vscale, want.vscale)


@pytest.mark.parametrize("dtype,d,P,eps", [("bf16", 128, 64, 1e-6), ("f32", 64, 16, 0.0), ("f32", 128, 32, 1e-6)])
def test_write_rope_of_rows_of_any_magnitude(dtype, d, P, eps):
    """Keys of zeros, and those whose squares leave the range, among others of their pages and alone on one."""
    g = torch.Generator().manual_seed(16)
    rng = np.random.default_rng(16)
    q, k, Hkv = [70, 1, 33, 64], [5, 30, 0, 0], 2
    n = sum(q)
    slot, n_pages = slots_of(rng, q, k, P)
    K, V = view(g, Hkv, n, d, torch.float32, "tokens"), view(g, Hkv, n, d, torch.float32, "tokens")
    for t, x in ((3, 1e30), (20, 1e-30), (40, 1e-38), (70, 1e25), (80, 1e37), (81, 1e-45)):
        K[:, t] *= x
    if eps:
        K[:, 50], K[1, 104:168], V[0, 104:168] = 0.0, 0.0, 0.0
    K, V = K.to(DT[dtype]), V.to(DT[dtype])
    for norm in (True, False):
        rope, _, _ = make_rope(g, d, d // 2, norm, eps=eps)
        cu, length = i32(prefix(q).tolist()), i32([a + b for a, b in zip(q, k)])
        pages = make_pages(rng, n_pages, Hkv, P, d)
        want = clone(pages)
        fa.kv_pages_write_rope(pages, i32(slot), None, K, V, rope, cu=cu, length=length)
        fa.kv_pages_write(want, i32(slot), fa.qk_norm_rope(None, K.float(), rope, cu=cu, length=length)[1], V.float())
        for name in ("K8", "kscale", "V8", "vscale"):
            assert torch.equal(getattr(pages, name), getattr(want, name)), (norm, name)


def test_prompts_whose_queries_have_a_launch_of_their_own():
    g = torch.Generator().manual_seed(15)
    rng = np.random.default_rng(15)
    q, k, P, d, Hq, Hkv = [5000, 3, 3700], [0, 9, 5], 64, 128, 64, 2
    n = sum(q)
    slot, n_pages = slots_of(rng, q, k, P)
    x = torch.randn((n, Hq + 2 * Hkv, d), generator=g).bfloat16().cuda()
    assert x.numel() * 2 >= 150000000
    Q, K, V = (y.transpose(0, 1) for y in x.split([Hq, Hkv, Hkv], 1))
    rope, _, _ = make_rope(g, d, d)
    cu, length = i32(prefix(q).tolist()), i32([a + b for a, b in zip(q, k)])
    pages = make_pages(rng, n_pages, Hkv, P, d)
    want = clone(pages)
    out = fa.kv_pages_write_rope(pages, i32(slot), Q, K, V, rope, cu=cu, length=length)
    assert torch.equal(out, fa.qk_norm_rope(Q, None, rope, cu=cu, length=length)[0])
    fa.kv_pages_write(want, i32(slot), fa.qk_norm_rope(None, K.float(), rope, cu=cu, length=length)[1], V.float())
    for name in ("K8", "kscale", "V8", "vscale"):
        assert torch.equal(getattr(pages, name), getattr(want, name)), name


def test_positions_on_axes_into_pages():
    g = torch.Generator().manual_seed(9)
    rng = np.random.default_rng(9)
    q, P, d, Hkv = [90, 33], 64, 128, 2
    n = sum(q)
    slot, n_pages = slots_of(rng, q, [0, 7], P)
    K, V = view(g, Hkv, n, d, torch.bfloat16, "fused"), view(g, Hkv, n, d, torch.bfloat16, "fused")
    rope, _, _ = make_rope(g, d, 128, True, True, 3)
    pos = i32(rng.integers(0, 100, size=(3, n)).tolist())
    pages = make_pages(rng, n_pages, Hkv, P, d)
    want = clone(pages)
    fa.kv_pages_write_rope(pages, i32(slot), None, K, V, rope, pos=pos)
    fa.kv_pages_write(want, i32(slot), fa.qk_norm_rope(None, K.float(), rope, pos=pos)[1], V.float())
    for name in ("K8", "kscale", "V8", "vscale"):
        assert torch.equal(getattr(pages, name), getattr(want, name)), name


def test_a_run_of_rows_of_two_sequences():
    """Slots of one page that follow one another, though their rows are of different sequences: positions are each its own."""
    g = torch.Generator().manual_seed(10)
    rng = np.random.default_rng(10)
    K, V = view(g, 1, 12, 64, torch.float32, "tokens"), view(g, 1, 12, 64, torch.float32, "tokens")
    rope, _, _ = make_rope(g, 64, 64)
    cu, length = i32([0, 3, 3, 7, 12]), i32([900, 0, 40, 77777])
    pages = make_pages(rng, 3, 1, 16, 64)
    want = clone(pages)
    slot = i32(list(range(16, 28)))
    fa.kv_pages_write_rope(pages, slot, None, K, V, rope, cu=cu, length=length)
    fa.kv_pages_write(want, slot, fa.qk_norm_rope(None, K, rope, cu=cu, length=length)[1], V)
    assert torch.equal(pages.K8, want.K8) and torch.equal(pages.kscale, want.kscale)


def test_replayed_from_a_graph_while_requests_grow():
    """One token per request and step, its position from the device: captured once, replayed with the program's own work between."""
    g = torch.Generator().manual_seed(11)
    rng = np.random.default_rng(11)
    B, P, d, Hq, Hkv, W = 3, 16, 64, 4, 2, 4
    rope, freq, _ = make_rope(g, d, d)
    K, V, Q = (torch.zeros((B, h, d), dtype=torch.bfloat16, device="cuda").transpose(0, 1) for h in (Hkv, Hkv, Hq))
    out = torch.zeros_like(Q)
    table, pool, pool_n = i32([[-1] * W] * B), i32(list(range(12))), i32([12])
    n_new, length, cu, slot, status = i32([1] * B), i32([0] * B), i32([0] * (B + 1)), i32([-1] * B), i32([0] * B)
    pages = fa.Pages.empty(12, Hkv, P, d)
    side = torch.cuda.Stream()

    def step():
        fa.kv_pages_plan(n_new, length, table, pool, pool_n, P, B, out=(length, pool_n, cu, slot, status))
        fa.kv_pages_write_rope(pages, slot, Q, K, V, rope, cu=cu, length=length, out=out)

    fa.init()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        length.zero_(), pool_n.fill_(12), table.fill_(-1)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for i in range(20):
            new = [torch.randn(x.shape, generator=g).to(torch.bfloat16) for x in (Q, K, V)]
            for x, y in zip((Q, K, V), new):
                x.copy_(y)
            graph.replay()
            side.synchronize()
            assert length.tolist() == [i + 1] * B
            at = np.full((B, d // 2), float(i))
            check_rows(out, Q, rope.q_weight, rope, freq, at, True)
            want = fa.Pages.empty(12, Hkv, P, d) if i == 0 else want
            fa.kv_pages_write_rope(want, slot, None, K, V, rope, cu=cu, length=length)
            for name in ("K8", "kscale", "V8", "vscale"):
                assert torch.equal(getattr(pages, name), getattr(want, name)), (i, name)


def test_arguments_that_do_not_fit_are_refused():
    g = torch.Generator().manual_seed(12)
    Q, K = view(g, 2, 8, 64, torch.float32, "tokens"), view(g, 1, 8, 64, torch.float32, "tokens")
    rope, _, _ = make_rope(g, 64, 64)
    pos = i32([list(range(8))])
    for bad in (dict(pos=pos[:, :7]), dict(pos=pos.long()), dict(pos=pos.cpu()), dict(cu=i32([0, 8])), dict(), dict(cu=i32([0, 8]), length=i32([8, 8])),
                dict(pos=pos, out=(Q, K[:, :4])), dict(pos=pos, out=(Q.bfloat16(), K)), dict(pos=pos, out=(Q, torch.empty(1, 8, 64)))):
        with pytest.raises((ValueError, TypeError, fa.FastarError)):
            fa.qk_norm_rope(Q, K, rope, **bad)
    with pytest.raises(ValueError):
        fa.qk_norm_rope(view(g, 2, 8, 128, torch.float32, "tokens"), None, rope, pos=pos)   # weights of 64
    with pytest.raises(ValueError):
        fa.qk_norm_rope(None, None, rope, pos=pos)
    with pytest.raises(TypeError):
        fa.Rope(torch.ones(4, device="cuda"))
    with pytest.raises(ValueError):
        fa.Rope(torch.ones(4, dtype=torch.float64, device="cuda"), axis=i32([0, 0, 0]))
