"""Norm and rotation, and calls on pages that requests share: what the host refuses (nothing is launched: the pointers are never
used), and the references of the GPU tests against their own definitions.  No GPU."""
import math
import os

import numpy as np
import pytest

import packed_ref as ref
import share_ref as sref
from test_packed_host import BAD, P, UNSUPPORTED, WORKSPACE, pages, rows


@pytest.fixture(scope="module")
def L():
    from paper_2602_01801_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2602_01801_amd.build import build
        build()
    return binding.lib()


def rope(**over):
    from paper_2602_01801_amd.binding import _RopeStruct
    f = dict(qw=P, kw=P, freq=P, axis=P, eps=1e-6, norm=1, rot=128, interleaved=0, n_axes=1)
    f.update(over)
    return _RopeStruct(*[f[k] for k in ("qw", "kw", "freq", "axis", "eps", "norm", "rot", "interleaved", "n_axes")])


R = 0   # rope() is made in the test: the fixture has loaded the package by then


def norm_rope(L, Q=R, K=R, pos=P, cu=P, length=P, B=1, n=100, Hq=4, Hkv=2, d=128, dtype=1, rp=R, Qo=R, Ko=R):
    pick = lambda x: rows() if x is R else x
    return L.qk_norm_rope(pick(Q), pick(K), pos, cu, length, B, n, Hq, Hkv, d, dtype, rope() if rp is R else rp, pick(Qo), pick(Ko), None)


ROPE_BAD = [
    (dict(rp=None), BAD), (dict(B=-1), BAD), (dict(n=-1), BAD), (dict(Hq=-1), BAD), (dict(Hkv=-1), BAD), (dict(dtype=2), BAD),
    (dict(Q=None), BAD), (dict(Ko=None), BAD), (dict(Q=rows(p=P + 8)), BAD), (dict(K=rows(row=132)), BAD), (dict(Qo=rows(row=64)), BAD),
    (dict(Ko=rows(head=64)), BAD), (dict(Qo=rows(row=0)), BAD), (dict(pos=None, cu=None, B=0), BAD), (dict(pos=None, length=None), BAD),
    (dict(cu=None), BAD), (dict(d=96), UNSUPPORTED), (dict(d=256), UNSUPPORTED), (dict(n=(1 << 30) + 1), UNSUPPORTED)]
STRUCT_BAD = [
    (dict(norm=2), BAD), (dict(norm=-1), BAD), (dict(interleaved=2), BAD), (dict(eps=-1e-9), BAD), (dict(eps=math.nan), BAD),
    (dict(eps=math.inf), BAD), (dict(rot=-16), BAD), (dict(rot=144), BAD), (dict(freq=None), BAD), (dict(n_axes=0), BAD),
    (dict(rot=24), UNSUPPORTED), (dict(rot=2), UNSUPPORTED), (dict(n_axes=5), UNSUPPORTED)]


@pytest.mark.parametrize("over,code", ROPE_BAD)
def test_norm_rope_refuses(L, over, code):
    assert norm_rope(L, **over) == code


@pytest.mark.parametrize("over,code", STRUCT_BAD)
def test_a_rotation_that_is_none_is_refused(L, over, code):
    assert norm_rope(L, rp=rope(**over)) == code
    assert write_rope(L, rp=rope(**over)) == code


def test_norm_rope_of_nothing_is_done_at_once(L):
    assert norm_rope(L, n=0) == 0 and norm_rope(L, B=0) == 0 and norm_rope(L, Hq=0, Hkv=0, Q=None, K=None, Qo=None, Ko=None) == 0


def test_launches_of_more_workgroups_than_there_can_be_are_refused(L):
    apart = rows(head=128, row=512)
    assert norm_rope(L, n=1 << 27, pos=None, Qo=apart, Ko=apart) == UNSUPPORTED
    assert write_rope(L, n=1 << 28, Hq=0) == UNSUPPORTED


def write_rope(L, pg=None, Q=R, K=R, V=R, dtype=1, slot=P, pos=P, cu=P, length=P, B=1, n=5, Hq=4, rp=R, Qo=R):
    pick = lambda x: rows() if x is R else x
    return L.kv_pages_write_rope(pg or pages(), pick(Q), pick(K), pick(V), dtype, slot, pos, cu, length, B, n, Hq, rope() if rp is R else rp,
                                 pick(Qo), None)


@pytest.mark.parametrize("over,code", [
    (dict(slot=None), BAD), (dict(n=-1), BAD), (dict(B=-1), BAD), (dict(dtype=3), BAD), (dict(Hq=-1), BAD), (dict(Q=None), BAD), (dict(Qo=None), BAD),
    (dict(K=None), BAD), (dict(V=rows(p=P + 8)), BAD), (dict(K=rows(row=4)), BAD), (dict(V=rows(row=1 << 24)), UNSUPPORTED), (dict(Qo=rows(row=8)), BAD),
    (dict(pos=None, length=None), BAD), (dict(cu=None), BAD), (dict(pg=pages(P=20)), UNSUPPORTED), (dict(pg=pages(d=80)), UNSUPPORTED),
    (dict(pg=pages(vscale=None)), BAD)])
def test_write_rope_refuses(L, over, code):
    assert write_rope(L, **over) == code


def test_write_rope_of_nothing_is_done_at_once(L):
    assert write_rope(L, n=0) == 0 and write_rope(L, B=0) == 0


def fork(L, pg=None, parent=P, child=P, keep=P, n=3, length=P, table=P, B=8, max_pages=4, pool=P, pool_n=P, after=P, free=P, status=P):
    return L.kv_pages_fork(pg or pages(), parent, child, keep, n, length, table, B, max_pages, pool, pool_n, after, free, status, None)


@pytest.mark.parametrize("over,code", [
    (dict(parent=None), BAD), (dict(child=None), BAD), (dict(length=None), BAD), (dict(table=None), BAD), (dict(pool=None), BAD),
    (dict(pool_n=None), BAD), (dict(after=None), BAD), (dict(free=None), BAD), (dict(status=None), BAD), (dict(n=-1), BAD), (dict(B=-1), BAD),
    (dict(max_pages=0), BAD), (dict(n=1025), UNSUPPORTED), (dict(max_pages=1 << 26), UNSUPPORTED), (dict(B=1 << 20, max_pages=1 << 11), UNSUPPORTED),
    (dict(pg=pages(P=8)), UNSUPPORTED), (dict(pg=pages(d=32)), UNSUPPORTED), (dict(pg=pages(K8=None)), BAD)])
def test_fork_refuses(L, over, code):
    assert fork(L, **over) == code


BIG = 1 << 40


def give(L, keep=P, length=P, table=P, B=3, max_pages=4, pool=P, pool_n=P, n_pages=10, size=64, after=P, free=P, status=P, ws=P, ws_bytes=BIG):
    return L.kv_pages_free(keep, length, table, B, max_pages, pool, pool_n, n_pages, size, after, free, status, ws, ws_bytes, None)


def thin(L, pg=None, keep=P, length=P, table=P, B=3, max_pages=4, pool=P, pool_n=P, after=P, table_out=P, pool_out=P, free=P, status=P, ws=P,
         ws_bytes=BIG):
    return L.kv_pages_compact(pg or pages(), keep, length, table, B, max_pages, pool, pool_n, after, table_out, pool_out, free, status, ws,
                              ws_bytes, None)


BOTH = [(dict(keep=None), BAD), (dict(length=None), BAD), (dict(table=None), BAD), (dict(pool=None), BAD), (dict(pool_n=None), BAD),
        (dict(after=None), BAD), (dict(free=None), BAD), (dict(status=None), BAD), (dict(ws=None), BAD), (dict(ws=P + 16), BAD),
        (dict(ws_bytes=0), WORKSPACE), (dict(B=-1), BAD), (dict(max_pages=0), BAD), (dict(max_pages=1 << 26), UNSUPPORTED),
        (dict(B=1 << 20, max_pages=1 << 11), UNSUPPORTED), (dict(B=1 << 23, max_pages=1), UNSUPPORTED)]


@pytest.mark.parametrize("over,code", BOTH + [(dict(size=8), UNSUPPORTED), (dict(size=128), UNSUPPORTED), (dict(n_pages=0), BAD), (dict(n_pages=1 << 26), UNSUPPORTED)])
def test_free_refuses(L, over, code):
    assert give(L, **over) == code


@pytest.mark.parametrize("over,code", BOTH + [(dict(keep=P + 8), BAD), (dict(table_out=None), BAD), (dict(pool_out=None), BAD),
                                              (dict(pg=pages(P=8)), UNSUPPORTED), (dict(pg=pages(V8=P + 4)), BAD)])
def test_compact_refuses(L, over, code):
    assert thin(L, **over) == code


def test_positions_of_a_mask_stay_in_32_bits_a_round_ahead(L):
    assert thin(L, B=1, max_pages=(1 << 24) + 1) == UNSUPPORTED and thin(L, B=1, max_pages=(1 << 25) - 1) == UNSUPPORTED


def test_workspace_of_shared_pages(L):
    from paper_2602_01801_amd import OP_PAGES, workspace_bytes
    need = workspace_bytes(OP_PAGES, 3, 4, 10, 64)
    assert need % 256 == 0 and need >= 4 * (3 * 10 + 3 * 4 + 3 * 12 + 2 * 10 + 12 * 64)
    assert workspace_bytes(OP_PAGES, 3, 4, 10, 20) == 0 and workspace_bytes(OP_PAGES, -1, 4, 10, 64) == 0
    assert give(L, ws_bytes=need - 1) == WORKSPACE and thin(L, ws_bytes=need - 1) == WORKSPACE


def test_what_a_rotation_is_made_of_is_looked_at():
    import torch
    import paper_2602_01801_amd as fa
    with pytest.raises(ValueError):
        fa.Rope(torch.ones(64, dtype=torch.float64))   # on the host
    assert fa.Rope(None).struct(128, 0).rot == 0


# ------------------------------------------------------------------------------------------------ the references


def test_rotation_reference_is_a_rotation():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(5, 3, 64))
    freq, pos = sref.frequencies(32), rng.integers(-9, 9999, size=(5, 1)).astype(float)
    for inter in (False, True):
        y, size = sref.rope(x, None, 0.0, False, freq, pos, 32, inter)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 32:], x[..., 32:])
        back, _ = sref.rope(y, None, 0.0, False, -freq, pos, 32, inter)
        assert np.allclose(back, x) and (np.abs(y) <= size + 1e-12).all()
        # products of two rotated rows go by the distance of their positions
        a, b = x[:1], x[1:2]
        dot = [float((sref.rope(a, None, 0, False, freq, np.array([[p]]), 32, inter)[0] * sref.rope(b, None, 0, False, freq, np.array([[p - 7.0]]), 32, inter)[0]).sum())
               for p in (7.0, 1000.0)]
        assert abs(dot[0] - dot[1]) < 1e-9
    z, _ = sref.rope(x * 1e30, np.full(64, 2.0), 1e-6, True, freq[:0], pos[:, :0], 0, False)
    assert np.allclose((z ** 2).mean(-1), 4.0)


def check_pages(table, length, pool, free, n_pages, P):
    """Every page is held or free, never both."""
    holders = [p for pages in sref.held(table, length, n_pages, P) for p in pages]
    assert sorted(set(holders) | set(pool[:free])) == list(range(n_pages))
    assert not set(holders) & set(pool[:free]) and len(set(pool[:free])) == free


def test_references_of_shared_pages_lose_no_page_and_hand_none_out_twice():
    rng = np.random.default_rng(2)
    Psz, n_pages, B, W = 16, 30, 9, 14
    table, length = [[-1] * W for _ in range(B)], [0] * B
    pool, free = [int(p) for p in rng.permutation(n_pages)], n_pages
    done, refused = [0] * 4, [0] * 4
    for step in range(600):
        what = rng.choice(4, p=[0.4, 0.3, 0.1, 0.2])
        if what == 0:
            n_new = [int(rng.choice([0, 1, 5, 40])) for _ in range(B)]
            length, free, _, _, status = ref.plan(n_new, length, table, pool, free, Psz, 400)
        elif what == 1:
            n = int(rng.integers(1, 4))
            parent, child = rng.integers(-1, B + 1, n).tolist(), rng.choice([b for b in range(B) if not length[b]] + [-1, B, 0], n).tolist()
            keep = None if rng.random() < 0.3 else rng.integers(-3, 60, n).tolist()
            length, free, status, _ = sref.fork(parent, child, keep, length, table, pool, free, Psz, n_pages)
        elif what == 2:
            keep = [int(rng.choice([0, length[b], max(0, length[b] - rng.integers(40))], p=[0.1, 0.5, 0.4])) for b in range(B)]
            length, free, status = sref.free(keep, length, table, pool, free, Psz, n_pages)
        else:
            keep = rng.random((B, W * Psz)) < rng.choice([0.3, 0.9])
            keep[:, :rng.integers(0, 60)] = True
            length, table, pool, free, status, _ = sref.compact(keep, length, table, pool, free, Psz, n_pages)
        done[what] += status.count(0)
        refused[what] += status.count(1)
        check_pages(table, length, pool, free, n_pages, Psz)
    assert min(done) > 20 and min(refused) > 3, (done, refused)
