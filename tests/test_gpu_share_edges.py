"""Forking, freeing and compacting of pages where a call is at an edge of what it allows, against plain loops (share_ref.py): exact."""
import math

import numpy as np
import pytest
import torch

import packed_ref as ref
import paper_2602_01801_amd as fa
import share_ref as sref
from test_gpu_packed import i32
from test_gpu_rope import make_pages
from test_gpu_share import ints, layout, run_compact, run_fork, run_free

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P,d,Hkv", [(16, 64, 3), (64, 128, 2), (32, 128, 5)])
def test_scales_that_are_no_numbers_stay_with_their_tokens(P, d, Hkv):
    """Tokens counted on pages whose scales were never written: NaN.  Theirs become NaN; those of other pages that move into the same fresh page keep
    their values, against the largest scale that is a number."""
    rng = np.random.default_rng(P + Hkv)
    W = 9
    lens = [W * P - 3, 5 * P]
    for share in (0.2, 0.6):
        table, pool, free, n_pages = layout(rng, lens, W, P, 2 * W)
        pages = make_pages(rng, n_pages, Hkv, P, d)
        for code, scale in ((pages.K8, pages.kscale), (pages.V8, pages.vscale)):   # no mantissas, so that fewer codes are rounded
            scale[torch.from_numpy(rng.random((n_pages, Hkv)) < share).cuda()] = math.nan
            code &= 0xF8
        K, ks, V, vs = (x.cpu().numpy().copy() for x in (pages.K8, pages.kscale, pages.V8, pages.vscale))
        keep = rng.random((2, W * P)) < 0.4
        length, new, left, n, status, made = sref.compact(keep, lens, table, pool, free, P, n_pages)
        got = fa.kv_pages_compact(pages, torch.from_numpy(keep.astype(np.uint8)).cuda(), i32(lens), i32(table), i32(pool), i32([free]))
        assert [ints(x) for x in got] == [length, new, left, [n], status] and made
        for x, xs, y, ys, transposed in ((K, ks, pages.K8, pages.kscale, False), (V, vs, pages.V8, pages.vscale, True)):
            was, now = ref.rows_of_cells(x, transposed), ref.rows_of_cells(y.cpu().numpy(), transposed)
            scale = ys.cpu().numpy()
            for page, src in made.items():
                old = np.array([xs[p] for p, _ in src])
                numbers = np.where(np.isnan(old), 0, old).max(0)
                for h in range(Hkv):
                    assert scale[page, h] == numbers[h]
                    for t, (p, o) in enumerate(src):
                        value = ref.VALUES[now[page, h, t]]
                        if np.isnan(xs[p, h]):
                            assert np.isnan(value).all()
                        else:
                            want = ref.round_e4m3(ref.VALUES[was[p, h, o]] * (xs[p, h] / numbers[h]))
                            assert np.array_equal(value, want, equal_nan=True)


# ------------------------------------------------------------------------------------------------ masks of several rounds

ROUND = 65536   # tokens of a request that its mask's workgroup looks at before it goes on


@pytest.mark.parametrize("P,beside", [(16, True), (16, False), (64, True), (64, False)])
def test_compact_of_requests_of_several_rounds(P, beside):
    """Two requests of more than twice as many tokens as a round has, neither a multiple of 64: counts of tokens and of fresh pages go from one round to the
    next.  Whole pages and fresh ones on both sides of every round's end, or a stretch of fresh ones across it."""
    rng = np.random.default_rng(P + beside)
    W = (2 * ROUND + 4000) // P
    T = W * P
    lens = [T - 27, 2 * ROUND + 1001]
    keep = np.repeat(rng.random((2, T // P)) < 0.9, P, 1)
    for b in range(2):
        for end in (ROUND, 2 * ROUND):
            keep[b, end - 1024:end + 1024] = True
            for lo, hi in ([(end - 512, end - 320), (end + 320, end + 512)] if beside else [(end - 192, end + 192)]):
                keep[b, lo:hi] = rng.random(hi - lo) < 0.5
                spare = np.flatnonzero(keep[b, lo:hi])[: int(keep[b, :hi].sum() % P)]   # so that the pages behind are whole again
                keep[b, lo + spare] = False
    table, pool, free, n_pages = layout(rng, lens, W, P, 200)
    pages = make_pages(rng, n_pages, 1, P, 64)
    want = run_compact(pages, keep, lens, table, pool, free, P)
    assert want[4] == [0, 0] and len(want[5]) >= 2 * 2 * 192 // P // 2
    for b in range(2):   # what the mask was made for
        rank = np.concatenate([[0], np.cumsum(keep[b])])
        old = {p: j for j, p in enumerate(table[b][: -(-lens[b] // P)])}
        kind = [old.get(p, -1) >= 0 for p in want[1][b][: -(-want[0][b] // P)]]
        for end in (ROUND, 2 * ROUND):
            at = int(rank[end]) // P
            before, behind = kind[at - 768 // P:at], kind[at + 1:at + 768 // P]
            assert any(before) and any(behind)
            assert not all(before) and not all(behind) if beside else not kind[at]


@pytest.mark.parametrize("B,first", [(700, 300), (700, 600), (1000, 800), (257, 256), (700, 255), (512, 511)])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact_of_requests_whose_pages_run_out_in_a_later_round(B, first, in_place):
    """Fresh pages are summed up 256 requests a round: the pool suffices for the requests before `first`."""
    rng = np.random.default_rng(B + first)
    P, W = 16, 2
    lens = [int(rng.integers(1, W * P + 1)) for _ in range(B)]
    table, pool, free, n_pages = layout(rng, lens, W, P, 2 * B, share=0.2)
    keep = rng.random((B, W * P)) < 0.6
    keep[first, :] = [0, 1] * P      # needs one
    lens[first] = max(lens[first], 5)
    all_of_it = sref.compact(keep, lens, table, pool, free, P, n_pages)
    assert 1 not in all_of_it[4]
    have = [set(p for p in row if p is not None) for row in sref.held(table, lens, n_pages, P)]
    need = [sum(p not in have[b] for p in all_of_it[1][b][: -(-all_of_it[0][b] // P)]) for b in range(B)]
    assert need[first] > 0
    pages = make_pages(rng, n_pages, 1, P, 64)
    want = run_compact(pages, keep, lens, table, pool, sum(need[:first]), P, in_place=in_place)
    assert want[4].index(1) == first and all(s == 0 or need[b] for b, s in enumerate(want[4]))


@pytest.mark.parametrize("n_free,lens", [(150_000, [37]), (150_000, [40, 0, 1, 33]), (1_100_000, [48])])
def test_compact_of_few_tokens_in_a_large_pool(n_free, lens):
    """Far more pages than the tables name, a workspace full of junk, and the same one again."""
    rng = np.random.default_rng(n_free + len(lens))
    P, W = 16, 3
    table, pool, free, n_pages = layout(rng, lens, W, P, n_free)
    pages = fa.Pages(*(torch.zeros(s, dtype=t, device="cuda") for s, t in (((n_pages, 1, 1, 4, 16, 16), torch.uint8), ((n_pages, 1), torch.float32)) * 2))
    ws = torch.randint(0, 256, (fa.workspace_bytes(fa.OP_PAGES, len(lens), W, n_pages, P),), dtype=torch.uint8, device="cuda")
    for turn in range(3):
        keep = rng.random((len(lens), W * P)) < 0.6
        keep[:, :P] = True
        want = sref.compact(keep, lens, table, pool, free, P, n_pages)
        t, ln, pn, pl = i32(table), i32(lens), i32([free]), i32(pool)
        out = (ln, t, pl, pn, i32([9] * len(lens))) if turn == 1 else None
        got = fa.kv_pages_compact(pages, torch.from_numpy(keep.astype(np.uint8)).cuda(), ln, t, pl, pn, out=out, ws=ws)
        for x, y in zip(got, want[:5]):
            assert torch.equal(x.cpu().view(-1), torch.tensor(y, dtype=torch.int32).view(-1))
        assert len(want[5])


# ------------------------------------------------------------------------------------------------ freeing by one workgroup and by several launches


@pytest.mark.parametrize("B,W,n_pages,share", [
    (1024, 8, 0, 0.5), (1024, 8, 0, 0.0), (1, 8192, 0, 0.0), (64, 128, 0, 0.7), (1023, 8, 16384, 0.0), (3, 5, 16384, 0.0),    # the most that one workgroup does
    (1025, 7, 0, 0.5), (2731, 3, 0, 0.5), (1, 8193, 0, 0.0), (1025, 8, 0, 0.0), (3, 5, 16385, 0.0), (1024, 8, 16385, 0.0)])   # the least that it does not
@pytest.mark.parametrize("full", [True, False])
def test_free_on_both_sides_of_what_one_workgroup_does(B, W, n_pages, share, full):
    rng = np.random.default_rng(B + W + n_pages)
    P = 16
    lens = [W * P - int(rng.integers(0, P)) if full else int(rng.choice([0, 1, P, rng.integers(0, W * P + 1)])) for _ in range(B)]
    held = sum(-(-n // P) for n in lens)
    table, pool, free, got = layout(rng, lens, W, P, n_pages - held if n_pages else 5, share=share, junk=not full)
    assert not n_pages or got == n_pages
    for in_place in (False, True):
        keep = [int(rng.choice([-5, 0, n, max(0, n - 1), rng.integers(0, n + 9), 2 ** 31 - 1], p=[0.1, 0.3, 0.2, 0.15, 0.15, 0.1])) for n in lens]
        status = run_free(keep, lens, table, pool, free, P, in_place=in_place)
        assert share == 0 or full is False or 1 in status
    run_free([0] * B, lens, table, pool, free, P)


# ------------------------------------------------------------------------------------------------ two calls at once


def test_two_calls_at_once():
    """Two caches on two streams, with a workspace each, step by step in turn: neither sees the other."""
    rng = np.random.default_rng(9)
    P, B, W = 16, 30, 12
    sides = []
    for i in range(2):
        lens = [int(rng.integers(1, W * P + 1)) for _ in range(B)]
        table, pool, free, n_pages = layout(rng, lens, W, P, 200, share=0.3)
        pages = make_pages(rng, n_pages, 2, P, 64)
        mask = rng.random((B, W * P)) < 0.6
        keep = [int(rng.integers(0, W * P)) for _ in range(B)]
        after, t, pl, n, s0, made = sref.compact(mask, lens, table, pool, free, P, n_pages)
        K, ks = pages.K8.cpu().numpy().copy(), pages.kscale.cpu().numpy().copy()
        sref.compact_codes(K, ks, False, made)
        after, n, s1 = sref.free(keep, after, t, pl, n, P, n_pages)
        state = dict(length=i32(lens), table=i32(table), pool=i32(pool), pool_n=i32([free]), mask=torch.from_numpy(mask.astype(np.uint8)).cuda(), keep=i32(keep),
                     status=[i32([9] * B), i32([9] * B)], pages=pages, stream=torch.cuda.Stream(),
                     ws=torch.empty(fa.workspace_bytes(fa.OP_PAGES, B, W, n_pages, P), dtype=torch.uint8, device="cuda"))
        sides.append((state, (after, n, pl, s0, s1, K, ks)))
    torch.cuda.synchronize()
    for what in range(2):
        for s, _ in sides:
            with torch.cuda.stream(s["stream"]):
                if what == 0:
                    fa.kv_pages_compact(s["pages"], s["mask"], s["length"], s["table"], s["pool"], s["pool_n"],
                                        out=(s["length"], s["table"], s["pool"], s["pool_n"], s["status"][0]), ws=s["ws"])
                else:
                    fa.kv_pages_free(s["keep"], s["length"], s["table"], s["pool"], s["pool_n"], P, out=(s["length"], s["pool_n"], s["status"][1]), ws=s["ws"])
    torch.cuda.synchronize()
    for s, (after, n, pl, s0, s1, K, ks) in sides:
        assert ints(s["length"]) == after and ints(s["pool_n"]) == [n] and ints(s["pool"])[:n] == pl[:n]
        assert [ints(x) for x in s["status"]] == [s0, s1]
        assert np.array_equal(s["pages"].K8.cpu().numpy(), K) and np.array_equal(s["pages"].kscale.cpu().numpy(), ks)


# ------------------------------------------------------------------------------------------------ pages named twice, pages far out, many requests from a graph


@pytest.mark.parametrize("B,W", [(1, 6), (9, 5), (40, 300)])
def test_pages_that_a_table_names_twice(B, W):
    """Any entry may name any page, its own request's among them: holders are counted by entries."""
    rng = np.random.default_rng(B + W)
    P, n_pages = 16, 8 * B + 30
    held = 2 * B + 3
    for turn in range(6):
        lens = [int(rng.choice([0, 1, P, W * P, rng.integers(0, W * P + 1)])) for _ in range(B)]
        order = rng.permutation(n_pages).tolist()
        table = [[order[int(rng.integers(held))] for _ in range(W)] for _ in range(B)]
        pool, free = order[held:] + [-1] * held, n_pages - held
        keep = [int(rng.choice([0, n, max(0, n - 1), n // 2, n // P * P])) for n in lens]
        run_free(keep, lens, table, pool, free, P, in_place=turn % 2 == 1)
        pages = make_pages(rng, n_pages, 2, P, 64)
        mask = np.repeat(rng.random((B, W)) < 0.7, P, 1) & (rng.random((B, W * P)) < (1.0 if turn < 3 else 0.97))
        run_compact(pages, mask, lens, table, pool, free, P, in_place=turn % 2 == 1)
        empty = [b for b in range(B) if lens[b] == 0]
        run_fork(rng, pages, rng.integers(0, B, len(empty)).tolist(), empty, rng.integers(0, W * P, len(empty)).tolist(), lens, table, pool, free, P)


def test_pages_beyond_32_bits():
    """Caches of more than 2^32 bytes: the last pages are forked, and move to each other."""
    rng = np.random.default_rng(17)
    P, d, Hkv, n_pages = 64, 128, 8, 70_000
    assert n_pages * P * d * Hkv > 2 ** 32
    pages = fa.Pages(*(torch.zeros(s, dtype=t, device="cuda") for s, t in (((n_pages, Hkv, P // 16, d // 16, 16, 16), torch.uint8), ((n_pages, Hkv), torch.float32)) * 2))
    few = 12
    at = [n_pages - 1, 0, n_pages - 2, 1, 65_535, 65_536, 65_537, n_pages - 3, 33_000, 2, n_pages - 4, 32_767]   # where the pages of a small cache lie in the large one
    small = make_pages(rng, few, Hkv, P, d)
    for big, x in ((pages.K8, small.K8), (pages.kscale, small.kscale), (pages.V8, small.V8), (pages.vscale, small.vscale)):
        big[at] = x
    def far(rows):
        return [[at[p] if 0 <= p < few else -1 for p in row] for row in rows]
    # a fork of 2 P + 5 tokens, then both requests thinned out
    table, pool = [[0, 1, 2, -1], [-1] * 4], [3, 4, 5, 6, 7, 8, 9, 10, 11, -1, -1, -1]
    lens, keep = i32([2 * P + 50, 0]), i32([2 * P + 5])
    st, tb, pl, pn = i32(table), i32(far(table)), i32([at[p] if p >= 0 else -1 for p in pool] + [-1] * (n_pages - few)), i32([9])
    spl, spn = i32(pool), i32([9])
    mask = torch.from_numpy((rng.random((2, 4 * P)) < 0.7).astype(np.uint8)).cuda()
    for pg, t, pool_t, n in ((small, st, spl, spn), (pages, tb, pl, pn)):
        ln = lens.clone()
        fa.kv_pages_fork(pg, i32([0]), i32([1]), ln, t, pool_t, n, keep=keep, out=(ln, n, i32([9])))
        got = fa.kv_pages_compact(pg, mask, ln, t, pool_t, n)
        t.copy_(got[1])
        assert ints(got[4]) == [0, 0]
    assert ints(tb) == far(ints(st))
    for name in ("K8", "kscale", "V8", "vscale"):
        assert torch.equal(getattr(pages, name)[at], getattr(small, name)), name
    for x in (pages.K8, pages.V8):
        x[at] = 0
        assert all(not x[a:a + 4096].any() for a in range(0, n_pages, 4096))


@pytest.mark.parametrize("B,W", [(1100, 3), (300, 30), (2100, 2)])
def test_many_requests_replayed_from_a_graph(B, W):
    """Thinning out and freeing by their launches for many requests, captured once, replayed on other lengths and masks with the program's own work between."""
    rng = np.random.default_rng(B)
    P, n_pages = 16, 3 * B * W
    state = dict(length=i32([0] * B), table=i32([[-1] * W] * B), pool=i32([0] * n_pages), pool_n=i32([0]), stay=i32([0] * B),
                 mask=torch.zeros((B, W * P), dtype=torch.uint8, device="cuda"))
    pages = make_pages(rng, n_pages, 1, P, 64)
    ws = torch.empty(fa.workspace_bytes(fa.OP_PAGES, B, W, n_pages, P), dtype=torch.uint8, device="cuda")
    st = [i32([0] * B), i32([0] * B)]
    side = torch.cuda.Stream()

    def calls(s):
        fa.kv_pages_compact(pages, s["mask"], s["length"], s["table"], s["pool"], s["pool_n"], out=(s["length"], s["table"], s["pool"], s["pool_n"], st[0]), ws=ws)
        fa.kv_pages_free(s["stay"], s["length"], s["table"], s["pool"], s["pool_n"], P, out=(s["length"], s["pool_n"], st[1]), ws=ws)

    fa.init()
    with torch.cuda.stream(side):
        calls(state)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls(state)
        for turn in range(4):
            lens = [int(rng.integers(0, W * P + 1)) for _ in range(B)]
            table, pool, _, total = layout(rng, lens, W, P, 10, share=0.3)
            assert total <= n_pages
            table = [[p if 0 <= p < total else -1 for p in row] for row in table]
            free = [10, B // 3 + 10, n_pages - total + 10, 0][turn]   # from then on pages that no table names
            pool = pool[:10] + list(range(total, n_pages)) + [-1] * (total - 10)
            stay = [int(rng.integers(0, W * P + 9)) for _ in range(B)]
            mask = rng.random((B, W * P)) < 0.7
            K, ks = pages.K8.cpu().numpy().copy(), pages.kscale.cpu().numpy().copy()
            for name, x in dict(length=lens, table=table, pool=pool, pool_n=[free], stay=stay).items():
                state[name].copy_(i32(x))
            state["mask"].copy_(torch.from_numpy(mask.astype(np.uint8)))
            graph.replay()
            side.synchronize()
            after, t, pool, n, s0, made = sref.compact(mask, lens, table, pool, free, P, n_pages)
            sref.compact_codes(K, ks, False, made)
            after, n, s1 = sref.free(stay, after, t, pool, n, P, n_pages)
            assert [ints(x) for x in st] == [s0, s1]
            assert ints(state["length"]) == after and ints(state["pool_n"]) == [n] and ints(state["pool"])[:n] == pool[:n]
            assert np.array_equal(pages.K8.cpu().numpy(), K) and np.array_equal(pages.kscale.cpu().numpy(), ks)
