"""Forking, freeing and compacting of pages, against plain loops (share_ref.py): tables, pools, counts and codes are exact."""
import numpy as np
import pytest
import torch

import packed_ref as ref
import paper_2602_01801_amd as fa
import share_ref as sref
from test_gpu_packed import check, f64, i32, prefix, view
from test_gpu_rope import clone, make_pages, make_rope

pytestmark = pytest.mark.gpu


def ints(t):
    return t.cpu().tolist()


def layout(rng, lens, W, P, n_free, share=0.0, junk=False):
    """Tables of requests of these lengths, some of whose full pages are those of an earlier request; pool and its count."""
    table, at, total = [], 0, 0
    for b, n in enumerate(lens):
        n = min(max(n, 0), W * P)
        row = [None] * -(-n // P)
        if b and rng.random() < share:
            a = int(rng.integers(b))
            m = int(rng.integers(0, min(n, min(max(lens[a], 0), W * P)) // P + 1))
            row[:m] = table[a][:m]
        for j, p in enumerate(row):
            if p is None:
                row[j], total = total, total + 1
        table.append(row)
    n_pages = total + n_free
    order = rng.permutation(n_pages).tolist()
    table = [[order[p] if p >= 0 else p for p in row] + [int(rng.choice([-1, -7, 0, n_pages, 2 ** 31 - 1])) for _ in range(W - len(row))] for row in table]
    if junk:   # entries that name no page
        for row, n in zip(table, lens):
            for j in range(-(-min(max(n, 0), W * P) // P)):
                if rng.random() < 0.1:
                    row[j] = int(rng.choice([-1, n_pages, -2 ** 31]))
    return table, order[total:] + [-5] * total, n_free, n_pages


# ------------------------------------------------------------------------------------------------ forking


def run_fork(rng, pages, parent, child, keep, length, table, pool, pool_n, P, in_place=False):
    n_pages = len(pool)
    K, ks, V, vs = (x.cpu().numpy().copy() for x in (pages.K8, pages.kscale, pages.V8, pages.vscale))
    want_table = [list(r) for r in table]
    after, free, status, copies = sref.fork(parent, child, keep, length, want_table, pool, pool_n, P, n_pages)
    for x in (K, ks, V, vs):
        old = x.copy()
        for a, b in copies:
            x[b] = old[a]
    t, ln, pn, pl = i32(table), i32(length), i32([pool_n]), i32(pool)
    st = i32([77] * len(parent))
    out = (ln, pn, st) if in_place else None
    got = fa.kv_pages_fork(pages, i32(parent), i32(child), ln, t, pl, pn, keep=None if keep is None else i32(keep), out=out)
    assert ints(got[2]) == status
    assert ints(got[0]) == after and ints(got[1]) == [free] and ints(t) == want_table and ints(pl) == pool
    for got, want in ((pages.K8, K), (pages.kscale, ks), (pages.V8, V), (pages.vscale, vs)):
        assert np.array_equal(got.cpu().numpy(), want)
    return status


@pytest.mark.parametrize("P,d,Hkv", [(16, 64, 1), (64, 128, 3), (32, 128, 8)])
@pytest.mark.parametrize("in_place", [False, True])
def test_fork(P, d, Hkv, in_place):
    rng = np.random.default_rng(P + Hkv)
    lens, W = [3 * P + 5, 0, 1, 0, 0, 2 * P, 0, 0, 5 * P - 1, 0], 6
    table, pool, free, n_pages = layout(rng, lens, W, P, 4)
    pages = make_pages(rng, n_pages, Hkv, P, d)
    # ends, full pages, one token, beyond the end, none, a parent that is a child too, children that hold tokens or are named twice, nobody
    parent = [0, 5, 8, 2, 0, 1, 0, 0, -1, 10, 0, 8]
    child = [1, 3, 4, 6, 0, 7, 1, 9, 7, 9, 10, 9]
    keep = [3 * P + 5, 2 * P, 2 * P + 3, 99 * P, 7, 4, 2, -4, 5, 5, 5, 9]
    status = run_fork(rng, pages, parent, child, keep, lens, table, pool, free, P, in_place)
    assert status.count(0) > 4 and status.count(2) > 4


@pytest.mark.parametrize("free", [0, 1, 7, 30])
def test_forks_until_the_pages_run_out(free):
    rng = np.random.default_rng(free)
    P, B, W = 16, 60, 9
    lens = [int(rng.integers(1, W * P)) if b % 3 == 0 else 0 for b in range(B)]
    table, pool, _, n_pages = layout(rng, lens, W, P, 30, junk=True)
    pages = make_pages(rng, n_pages, 2, P, 64)
    child = [b for b in range(B) if not lens[b]]
    parent = [3 * int(rng.integers(B // 3)) for _ in child]
    keep = [int(rng.integers(0, W * P + 9)) for _ in child]
    run_fork(rng, pages, parent, child, keep, lens, table, pool, free, P)


def test_as_many_forks_as_a_call_can_have():
    rng = np.random.default_rng(7)
    P, W, n = 16, 3, 1024
    lens = [W * P - 3] + [0] * 1500
    table, pool, free, n_pages = layout(rng, lens, W, P, 700)
    pages = make_pages(rng, n_pages, 1, P, 64)
    child = (1 + rng.permutation(1500)[:n]).tolist()
    child[900] = child[3]    # named before, in another round of threads
    keep = rng.integers(0, W * P, n).tolist()
    status = run_fork(rng, pages, [0] * n, child, keep, lens, table, pool, free, P)
    assert status[900] == 2 and 1 in status
    run_fork(rng, pages, [], [], None, lens, table, pool, free, P)            # nobody
    run_fork(rng, pages, [], [], [], lens, table, pool, free, P, True)


# ------------------------------------------------------------------------------------------------ freeing


def run_free(keep, length, table, pool, pool_n, P, in_place=False):
    n_pages = len(pool)
    want_pool = list(pool)
    after, free, status = sref.free(keep, length, table, want_pool, pool_n, P, n_pages)
    t, ln, pn, pl = i32(table), i32(length), i32([pool_n]), i32(pool)
    out = (ln, pn, i32([9] * len(length))) if in_place else None
    got = fa.kv_pages_free(i32(keep), ln, t, pl, pn, P, out=out)
    assert ints(got[2]) == status
    assert ints(got[0]) == after and ints(got[1]) == [free]
    assert ints(pl) == want_pool and ints(t) == [list(r) for r in table]
    return status


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("P,B,W", [(16, 5, 7), (64, 40, 3), (32, 1, 2500), (16, 300, 30), (16, 3, 5000)])
def test_free(seed, P, B, W):
    rng = np.random.default_rng(1000 * seed + B)
    lens = [int(rng.choice([0, 1, P, 2 * P + 3, rng.integers(0, W * P + 1)])) for _ in range(B)]
    table, pool, free, n_pages = layout(rng, lens, W, P, 3, share=[0, 0.5, 0.9][seed % 3], junk=seed >= 3)
    if seed == 5:
        lens[0] += 10 ** 9   # cut to the table
        lens[-1] = -3
    keep = [int(rng.choice([-5, 0, n, max(0, n - 1), rng.integers(0, max(n, 0) + 9), 2 ** 31 - 1])) for n in lens]
    run_free(keep, lens, table, pool, free, P, in_place=seed % 2 == 1)


def test_what_others_hold_stays_with_them():
    P = 16
    table = [[0, 1, 2, -1], [0, 1, 3, -1], [0, 4, 5, 6], [0, 1, 3, -1]]
    length = [40, 48, 64, 48]
    pool = [9, 8, 7, 10] + [-1] * 7
    assert run_free([0, 48, 64, 48], length, table, pool, 4, P) == [0, 0, 0, 0]
    assert run_free([0, 0, 0, 0], length, table, pool, 4, P) == [0, 0, 0, 0]          # shared pages at the last holder's place
    assert run_free([20, 48, 17, 0], length, table, pool, 4, P) == [1, 0, 0, 0]       # into a page that others hold, one of whom ends
    assert run_free([16, 32, 1, 48], length, table, pool, 4, P) == [0, 0, 1, 0]       # at a page's end
    assert run_free([0, 0, 0, 0], length, table, pool[:8] + [-1] * 3, 8, P) == [0, 0, 0, 0]   # more than the pool can hold


def test_free_of_nobody():
    n = i32([3])
    got = fa.kv_pages_free(i32([]), i32([]), i32([]).view(0, 4), i32([1, 2, 3, -1]), n, 16)
    assert ints(got[1]) == [3]


# ------------------------------------------------------------------------------------------------ thinning out


def run_compact(pages, keep, length, table, pool, pool_n, P, in_place=False, boolean=False):
    n_pages = len(pool)
    want = sref.compact(keep, length, table, pool, pool_n, P, n_pages)
    K, ks, V, vs = (x.cpu().numpy().copy() for x in (pages.K8, pages.kscale, pages.V8, pages.vscale))
    sref.compact_codes(K, ks, False, want[5])
    sref.compact_codes(V, vs, True, want[5])
    t, ln, pn, pl = i32(table), i32(length), i32([pool_n]), i32(pool)
    mask = torch.from_numpy(keep.astype(np.uint8)).cuda()
    out = (ln, t, pl, pn, i32([9] * len(length))) if in_place else None
    got = fa.kv_pages_compact(pages, mask.bool() if boolean else mask, ln, t, pl, pn, out=out)
    assert ints(got[4]) == want[4]
    assert ints(got[0]) == want[0] and ints(got[3]) == [want[3]]
    assert ints(got[1]) == want[1]
    assert ints(got[2]) == want[2]
    if not in_place:
        assert ints(t) == [list(r) for r in table] and ints(pl) == pool and ints(ln) == list(length)
    for name, x, y in (("K8", pages.K8, K), ("kscale", pages.kscale, ks), ("V8", pages.V8, V), ("vscale", pages.vscale, vs)):
        assert np.array_equal(x.cpu().numpy(), y), name
    return want


MASKS = {
    "half": lambda rng, B, T: rng.random((B, T)) < 0.5,
    "few": lambda rng, B, T: rng.random((B, T)) < 0.03,
    "most": lambda rng, B, T: rng.random((B, T)) < 0.98,
    "all": lambda rng, B, T: np.ones((B, T), bool),
    "none": lambda rng, B, T: np.zeros((B, T), bool),
    "window": lambda rng, B, T: (np.arange(T) < 5) | (np.arange(T)[None] >= rng.integers(0, T, B)[:, None]),
    "pages": lambda rng, B, T: np.repeat(rng.random((B, T // 16)) < 0.7, 16, 1),
    "runs": lambda rng, B, T: np.repeat(rng.random((B, T // 4)) < 0.5, 4, 1),
}


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("P,d,Hkv,B,W", [(16, 64, 1, 4, 6), (64, 128, 2, 3, 5), (32, 128, 5, 7, 4), (64, 64, 2, 1, 40)])
def test_compact(mask, P, d, Hkv, B, W):
    rng = np.random.default_rng(len(mask) * 31 + P + B)
    for turn in range(3):
        lens = [int(rng.choice([0, 1, P, W * P, rng.integers(0, W * P + 1)])) for _ in range(B)]
        lens[0] = W * P - 3
        n_free = B * W if turn else W + 1
        table, pool, free, n_pages = layout(rng, lens, W, P, n_free, share=0.5 if turn else 0.0, junk=turn == 2)
        pages = make_pages(rng, n_pages, Hkv, P, d)
        keep = MASKS[mask](rng, B, W * P)
        run_compact(pages, np.broadcast_to(keep, (B, W * P)), lens, table, pool, free, P, in_place=turn == 1, boolean=turn == 2)


def test_compact_of_a_long_request():
    rng = np.random.default_rng(3)
    P, W = 16, 4000
    lens = [W * P - 9, 20011]
    table, pool, free, n_pages = layout(rng, lens, W, P, 5000)
    pages = make_pages(rng, n_pages, 1, P, 64)
    keep = np.repeat(rng.random((2, W * P // 32)) < 0.5, 32, 1)
    keep[0, :1000] = True
    run_compact(pages, keep, lens, table, pool, free, P)


def test_compact_of_many_requests():
    rng = np.random.default_rng(4)
    P, W, B = 16, 2, 1100
    lens = [int(rng.integers(0, W * P + 1)) for _ in range(B)]
    table, pool, free, n_pages = layout(rng, lens, W, P, 900, share=0.3)
    pages = make_pages(rng, n_pages, 1, P, 64)
    want = run_compact(pages, rng.random((B, W * P)) < 0.6, lens, table, pool, free, P)
    assert 0 in want[4] and 1 in want[4]


def test_more_requests_than_workgroups_sum_up():
    """Blocks of entries whose counts are summed by a launch of their own."""
    rng = np.random.default_rng(8)
    P, W, B = 16, 2, 4500
    lens = [int(rng.integers(0, W * P + 1)) for _ in range(B)]
    table, pool, free, n_pages = layout(rng, lens, W, P, 5000, share=0.2)
    keep = [int(rng.choice([0, n, max(0, n - 1), n // 2])) for n in lens]
    run_free(keep, lens, table, pool, free, P)
    pages = make_pages(rng, n_pages, 1, P, 64)
    run_compact(pages, rng.random((B, W * P)) < 0.7, lens, table, pool, free, P, in_place=True)


@pytest.mark.parametrize("P,d,Hkv", [(16, 64, 20), (32, 64, 9), (16, 128, 9), (64, 128, 1), (32, 128, 4)])
def test_compact_of_many_heads(P, d, Hkv):
    """More heads than an item takes, and fewer."""
    rng = np.random.default_rng(P + Hkv)
    lens = [5 * P - 2, 3 * P + 1]
    table, pool, free, n_pages = layout(rng, lens, 6, P, 12)
    pages = make_pages(rng, n_pages, Hkv, P, d)
    run_compact(pages, rng.random((2, 6 * P)) < 0.6, lens, table, pool, free, P)


def test_compact_keeps_what_a_code_says():
    """Every code, NaN and both zeros among them, over pages of equal scales: carried bit by bit, and rounded where the scales differ."""
    rng = np.random.default_rng(5)
    P, d = 16, 64
    pages = make_pages(rng, 8, 1, P, d)
    every = torch.arange(256, dtype=torch.uint8).repeat(P * d // 256).view(1, 1, 1, d // 16, 16, 16)
    for x in (pages.K8, pages.V8):
        x[:4] = every
    for x in (pages.kscale, pages.vscale):
        x[:] = torch.tensor([1.0, 1.0, 0.25, 2.0 ** 20, 1, 1, 1, 1])[:, None]
    keep = np.ones((1, 64), bool)
    keep[0, [1, 18, 33, 40]] = False
    table, pool = [[0, 1, 2, 3]], [4, 5, 6, 7, -1, -1, -1, -1]
    n = sref.compact(keep, [64], table, pool, 4, P, 8)
    K, ks = pages.K8.cpu().numpy().copy(), pages.kscale.cpu().numpy().copy()
    V, vs = pages.V8.cpu().numpy().copy(), pages.vscale.cpu().numpy().copy()
    fa.kv_pages_compact(pages, torch.from_numpy(keep).cuda(), i32([64]), i32(table), i32(pool), i32([4]))
    sref.compact_codes(K, ks, False, n[5])
    sref.compact_codes(V, vs, True, n[5])
    for got, want in ((pages.K8, K), (pages.V8, V)):
        got = got.cpu().numpy()
        got, want = (np.where(x & 127 == 127, 127, x) for x in (got, want))   # one NaN
        assert np.array_equal(got, want)
    assert np.array_equal(pages.kscale.cpu().numpy(), ks) and np.array_equal(pages.vscale.cpu().numpy(), vs)


def test_compact_of_pages_that_nothing_was_written_to():
    """Tokens that have been counted but not written: scales are zero, alone in a fresh page or beside others."""
    rng = np.random.default_rng(12)
    P, W = 16, 5
    table, pool, free, n_pages = layout(rng, [5 * P, 4 * P + 3], W, P, 12)
    pages = make_pages(rng, n_pages, 3, P, 64)
    for code, scale in ((pages.K8, pages.kscale), (pages.V8, pages.vscale)):
        for p in table[0][1:] + table[1][3:]:
            if 0 <= p < n_pages:
                code[p], scale[p] = 0, 0
    keep = np.ones((2, W * P), bool)
    keep[:, ::3] = False
    run_compact(pages, keep, [5 * P, 4 * P + 3], table, pool, free, P)
    assert (pages.kscale == 0).any() and not ((pages.K8 & 127) == 127).any() and not ((pages.V8 & 127) == 127).any()


@pytest.mark.parametrize("P,B,W", [(16, 4, 9), (16, 300, 30), (64, 12, 1000), (16, 4500, 2)])
def test_more_pages_than_the_pool_can_hold(P, B, W):
    """A count that says that more is free than the tables leave: pages are lost, and nothing is written behind the pool, which is longer than the call's."""
    rng = np.random.default_rng(B + W)
    lens = [int(rng.integers(1, min(W, 40) * P + 1)) for _ in range(B)]
    table, pool, free, n_pages = layout(rng, lens, W, P, 9, share=0.3)
    held = n_pages - free
    pool = [p if p >= 0 else int(rng.integers(n_pages)) for p in pool]
    for pool_n in (n_pages, n_pages - 1, n_pages - held // 3):
        behind = i32(pool + [-77] * 5000)
        want_pool = list(pool)
        after, n, status = sref.free([0] * B, lens, table, want_pool, pool_n, P, n_pages)
        got = fa.kv_pages_free(i32([0] * B), i32(lens), i32(table), behind[:n_pages], i32([pool_n]), P)
        assert n == n_pages and ints(got[1]) == [n] and ints(got[0]) == after and ints(got[2]) == status
        assert ints(behind) == want_pool + [-77] * 5000
    pages = make_pages(rng, n_pages, 1, P, 64)
    keep = np.zeros((B, W * P), bool)
    keep[:, :P] = True      # whole pages stay: no page is taken
    run_compact(pages, keep, [n // P * P for n in lens], table, pool, n_pages - held // 3, P, in_place=True)


def test_compact_of_nobody():
    pages = fa.Pages.empty(4, 1, 16, 64)
    got = fa.kv_pages_compact(pages, torch.zeros((0, 32), dtype=torch.uint8, device="cuda"), i32([]), i32([]).view(0, 2), i32([1, 2, 3, -1]), i32([3]))
    assert ints(got[3]) == [3] and ints(got[2]) == [1, 2, 3, -1]


# ------------------------------------------------------------------------------------------------ together


def test_requests_that_share_grow_thin_out_and_end():
    """A prompt, two forks of it, tokens for all three, one thinned out, one ended: attention over every cache against 64 bits, and no page
    lost or held by two who write to it."""
    g = torch.Generator().manual_seed(1)
    rng = np.random.default_rng(1)
    P, d, Hq, Hkv, B, W, n_pages = 16, 128, 4, 2, 4, 12, 40
    rope, freq, _ = make_rope(g, d, d)
    pages = fa.Pages.empty(n_pages, Hkv, P, d)
    table, length = i32([[-1] * W] * B), i32([0] * B)
    pool, pool_n = i32(rng.permutation(n_pages).tolist()), i32([n_pages])
    cache = [[np.zeros((Hkv, 0, d))] * 2 for _ in range(B)]    # what every request's cache stands for

    def stand_for():
        K, V = pages.K8.cpu().numpy(), pages.V8.cpu().numpy()
        ks, vs, t, n = f64(pages.kscale), f64(pages.vscale), table.cpu().numpy(), ints(length)
        return [(ref.keys_of_pages(K, ks, t[b, :-(-n[b] // P)], n[b], False), ref.keys_of_pages(V, vs, t[b, :-(-n[b] // P)], n[b], True)) for b in range(B)]

    def accounts():
        n, free = ints(length), ints(pool_n)[0]
        holders = [p for row in sref.held(ints(table), n, n_pages, P) for p in row]
        assert sorted(set(holders) | set(ints(pool)[:free])) == list(range(n_pages)) and not set(holders) & set(ints(pool)[:free])

    def grow(n_new):
        nonlocal cache
        n = sum(n_new)
        Q, K, V = view(g, Hq, n, d, torch.bfloat16, "fused"), view(g, Hkv, n, d, torch.bfloat16, "fused"), view(g, Hkv, n, d, torch.bfloat16, "fused")
        before = stand_for()
        _, _, cu, slot, status = fa.kv_pages_plan(i32(n_new), length, table, pool, pool_n, P, n, out=(length, pool_n, i32([0] * (B + 1)), i32([-1] * n), i32([0] * B)))
        assert ints(status) == [0] * B
        Qr = fa.kv_pages_write_rope(pages, slot, Q, K, V, rope, cu=cu, length=length)
        cache = stand_for()
        for b in range(B):   # what was there stays, but for a page's larger scale
            m = before[b][0].shape[1]
            assert np.abs(cache[b][0][:, :m] - before[b][0]).max(initial=0) <= 2.0 ** -4 * np.abs(before[b][0]).max(initial=1)
        O, lse = fa.paged_attn_fwd(Qr, cu, length, table, pages)
        at = prefix(n_new)
        for b in range(B):
            if n_new[b]:
                i = slice(at[b], at[b + 1])
                want = ref.attend(f64(Qr[:, i]), *cache[b], True, d ** -0.5)
                check(O[:, i], lse[:, i], want, cache[b][0].shape[1], d, True, f"request {b}")
        accounts()

    grow([70, 0, 0, 9])
    before = stand_for()
    _, _, status = fa.kv_pages_fork(pages, i32([0, 0]), i32([1, 2]), length, table, pool, pool_n, keep=i32([70, 40]), out=(length, pool_n, i32([0, 0])))
    assert ints(status) == [0, 0] and ints(length) == [70, 70, 40, 9]
    after = stand_for()
    for b, n in ((0, 70), (1, 70), (2, 40)):
        for x, y in zip(before[0], after[b]):
            assert np.array_equal(x[:, :n], y)
    accounts()
    grow([1, 1, 1, 1])
    grow([3, 20, 30, 1])
    keep = torch.zeros((B, W * P), dtype=torch.uint8)
    keep[0, :16], keep[0, 33:] = 1, 1
    keep[1:] = 1
    before = stand_for()
    _, _, _, _, status = fa.kv_pages_compact(pages, keep.cuda(), length, table, pool, pool_n, out=(length, table, pool, pool_n, i32([0] * B)))
    assert ints(status) == [0] * B and ints(length) == [74 - 17, 91, 71, 11]
    after = stand_for()
    kept = np.r_[0:16, 33:74]
    for x, y in zip(before[0], after[0]):   # scales are powers of two: only codes that became subnormal are rounded
        assert np.abs(x[:, kept] - y).max() <= 2.0 ** -4 * np.abs(x).max()
    for b in (1, 2, 3):
        assert all(np.array_equal(x, y) for x, y in zip(before[b], after[b]))
    accounts()
    grow([2, 1, 1, 0])
    _, _, status = fa.kv_pages_free(i32([99, 0, 99, 4]), length, table, pool, pool_n, P, out=(length, pool_n, i32([0] * B)))
    assert ints(status) == [0] * B and ints(length) == [59, 0, 72, 4]
    accounts()
    grow([1, 15, 1, 1])
    fa.kv_pages_free(i32([0] * B), length, table, pool, pool_n, P, out=(length, pool_n, i32([0] * B)))
    assert ints(pool_n) == [n_pages]
    accounts()


@pytest.mark.parametrize("seed,P,B,W,n_pages", [(0, 16, 9, 14, 40), (1, 32, 40, 6, 150), (2, 16, 20, 500, 3000), (3, 64, 3, 9, 20)])
def test_a_long_life_of_many_requests(seed, P, B, W, n_pages):
    """Plans, forks, cuts and masks in any order, everything in place, step by step against the references; codes go where tables say."""
    rng = np.random.default_rng(seed)
    pages = make_pages(rng, n_pages, 1, P, 64)
    K, ks, V, vs = (x.cpu().numpy().copy() for x in (pages.K8, pages.kscale, pages.V8, pages.vscale))
    table, length = [[-1] * W for _ in range(B)], [0] * B
    pool, free = [int(p) for p in rng.permutation(n_pages)], n_pages
    dt, dl, dp, dn = i32(table), i32(length), i32(pool), i32([free])
    for step in range(80):
        what = rng.choice(4, p=[0.4, 0.25, 0.15, 0.2])
        if what == 0:
            n_new = [int(rng.choice([0, 1, P, rng.integers(0, W * P // 2 + 1)])) for _ in range(B)]
            after, free, _, _, status = ref.plan(n_new, length, table, pool, free, P, 10 ** 6)
            got = fa.kv_pages_plan(i32(n_new), dl, dt, dp, dn, P, sum(n_new), out=(dl, dn, i32([0] * (B + 1)), i32([-1] * sum(n_new)), i32([0] * B)))[4]
        elif what == 1:
            n = int(rng.integers(1, 6))
            parent, empty = rng.integers(-1, B + 1, n).tolist(), [b for b in range(B) if not length[b]]
            child, keep = rng.choice(empty + [-1, B, 0], n).tolist(), rng.integers(-3, W * P, n).tolist()
            after, free, status, copies = sref.fork(parent, child, keep, length, table, pool, free, P, n_pages)
            for x in (K, ks, V, vs):
                old = x.copy()
                for a, b in copies:
                    x[b] = old[a]
            got = fa.kv_pages_fork(pages, i32(parent), i32(child), dl, dt, dp, dn, keep=i32(keep), out=(dl, dn, i32([9] * n)))[2]
        elif what == 2:
            keep = [int(rng.choice([0, n, max(0, n - rng.integers(40))], p=[0.2, 0.4, 0.4])) for n in length]
            after, free, status = sref.free(keep, length, table, pool, free, P, n_pages)
            got = fa.kv_pages_free(i32(keep), dl, dt, dp, dn, P, out=(dl, dn, i32([9] * B)))[2]
        else:
            keep = np.repeat(rng.random((B, W * P // 16)) < rng.choice([0.5, 0.9]), 16, 1) ^ (rng.random((B, W * P)) < 0.01)
            after, table, pool, free, status, made = sref.compact(keep, length, table, pool, free, P, n_pages)
            sref.compact_codes(K, ks, False, made)
            sref.compact_codes(V, vs, True, made)
            got = fa.kv_pages_compact(pages, torch.from_numpy(keep.astype(np.uint8)).cuda(), dl, dt, dp, dn, out=(dl, dt, dp, dn, i32([9] * B)))[4]
        length = after
        assert ints(got) == status, step
        assert ints(dl) == length and ints(dn) == [free] and ints(dp)[:free] == pool[:free], step
        assert sref.held(ints(dt), length, n_pages, P) == sref.held(table, length, n_pages, P), step
        for x, y in ((pages.K8, K), (pages.kscale, ks), (pages.V8, V), (pages.vscale, vs)):
            assert np.array_equal(x.cpu().numpy(), y), step
        holders = [p for row in sref.held(table, length, n_pages, P) for p in row]
        assert not set(holders) & set(pool[:free]) and sorted(set(holders) | set(pool[:free])) == list(range(n_pages)), step


def test_replayed_from_a_graph():
    """Fork, thin out and end, captured once with everything in place and replayed on other lengths and masks."""
    rng = np.random.default_rng(6)
    P, d, Hkv, B, W = 16, 64, 2, 6, 9
    side = torch.cuda.Stream()
    n_pages = B * W * 2
    state = dict(length=i32([0] * B), table=i32([[-1] * W] * B), pool=i32([0] * n_pages), pool_n=i32([0]), parent=i32([0, 1]), child=i32([4, 5]),
                 keep=i32([0, 0]), mask=torch.zeros((B, W * P), dtype=torch.uint8, device="cuda"), stay=i32([0] * B))
    pages = make_pages(rng, n_pages, Hkv, P, d)
    ws = torch.empty(fa.workspace_bytes(fa.OP_PAGES, B, W, n_pages, P), dtype=torch.uint8, device="cuda")
    st = [i32([0] * 2), i32([0] * B), i32([0] * B)]

    def calls(s):
        fa.kv_pages_fork(pages, s["parent"], s["child"], s["length"], s["table"], s["pool"], s["pool_n"], keep=s["keep"], out=(s["length"], s["pool_n"], st[0]))
        fa.kv_pages_compact(pages, s["mask"], s["length"], s["table"], s["pool"], s["pool_n"], out=(s["length"], s["table"], s["pool"], s["pool_n"], st[1]), ws=ws)
        fa.kv_pages_free(s["stay"], s["length"], s["table"], s["pool"], s["pool_n"], P, out=(s["length"], s["pool_n"], st[2]), ws=ws)

    fa.init()
    with torch.cuda.stream(side):
        calls(state)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls(state)
        for turn in range(6):
            lens = [int(rng.integers(1, W * P)) for _ in range(4)] + [0, 0]
            table, pool, free, _ = layout(rng, lens, W, P, n_pages)
            pool = [p for p in pool if p < n_pages and p >= 0]
            table, pool = [[p if 0 <= p < n_pages else -1 for p in r] for r in table], pool[:n_pages // 2]
            free = len(pool)
            pool += [-1] * (n_pages - free)
            keep, stay = [int(rng.integers(0, W * P)) for _ in range(2)], [int(rng.integers(0, W * P)) for _ in range(B)]
            mask = rng.random((B, W * P)) < 0.7
            for name, x in dict(length=lens, table=table, pool=pool, pool_n=[free], keep=keep, stay=stay).items():
                state[name].copy_(i32(x))
            state["mask"].copy_(torch.from_numpy(mask.astype(np.uint8)))
            graph.replay()
            side.synchronize()
            t = [list(r) for r in table]
            after, free, s0, _ = sref.fork([0, 1], [4, 5], keep, lens, t, pool, free, P, n_pages)
            after, t, pool, free, s1, _ = sref.compact(mask, after, t, pool, free, P, n_pages)
            after, free, s2 = sref.free(stay, after, t, pool, free, P, n_pages)
            assert [ints(x) for x in st] == [s0, s1, s2]
            assert ints(state["length"]) == after and ints(state["pool_n"]) == [free] and ints(state["pool"])[:free] == pool[:free]


def test_arguments_that_do_not_fit_are_refused():
    pages = fa.Pages.empty(6, 1, 16, 64)
    table, n, pool, free = i32([[0, 1], [2, 3]]), i32([20, 20]), i32([4, 5, 0, 0, 0, 0]), i32([2])
    mask = torch.ones((2, 32), dtype=torch.uint8, device="cuda")
    for call in (lambda: fa.kv_pages_fork(pages, i32([0]), i32([1, 1]), n, table, pool, free),
                 lambda: fa.kv_pages_fork(pages, i32([0]), i32([1]), n, table, pool[:5], free),
                 lambda: fa.kv_pages_fork(pages, i32([0]), i32([1]).cpu(), n, table, pool, free),
                 lambda: fa.kv_pages_free(i32([0]), n, table, pool, free, 16),
                 lambda: fa.kv_pages_free(i32([0, 0]), n, table, pool, free, 17),
                 lambda: fa.kv_pages_free(i32([0, 0]), n, table, pool, free, 16, ws=torch.empty(256, dtype=torch.uint8, device="cuda")),
                 lambda: fa.kv_pages_free(i32([0, 0]), n, table, pool, free, 16, ws=torch.empty(1 << 20, dtype=torch.uint8)),
                 lambda: fa.kv_pages_compact(pages, mask[:, :31], n, table, pool, free),
                 lambda: fa.kv_pages_compact(pages, mask.float(), n, table, pool, free),
                 lambda: fa.kv_pages_compact(pages, mask.cpu(), n, table, pool, free),
                 lambda: fa.kv_pages_compact(pages, mask, n.long(), table, pool, free)):
        with pytest.raises((ValueError, TypeError, fa.FastarError)):
            call()
