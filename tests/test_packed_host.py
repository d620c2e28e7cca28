"""Calls over packed sequences and paged caches: what the host refuses (nothing is launched: the pointers are never used), and
the references of the GPU tests against their own definitions.  No GPU."""
import ctypes
import math
import os

import numpy as np
import pytest

import packed_ref as ref


@pytest.fixture(scope="module")
def L():
    from paper_2602_01801_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2602_01801_amd.build import build
        build()
    return binding.lib()


P = 0x10000   # an address that is never read


def rows(p=P, head=128 * 100, row=128):
    from paper_2602_01801_amd.binding import _RowsStruct
    return _RowsStruct(p, head, row)


def pages(**over):
    from paper_2602_01801_amd.binding import _PagesStruct
    f = dict(K8=P, V8=P, kscale=P, vscale=P, n_pages=10, Hkv=2, P=64, d=128)
    f.update(over)
    return _PagesStruct(*[f[k] for k in ("K8", "V8", "kscale", "vscale", "n_pages", "Hkv", "P", "d")])


def prompt(L, Q=None, K=None, V=None, O=None, cu=P, B=1, n_q=100, n_k=100, Hq=4, Hkv=2, d=128, dtype=1, causal=1, scale=0.1):
    r = rows()
    return L.prompt_attn_fwd(Q or r, K or r, V or r, cu, None, B, n_q, n_k, Hq, Hkv, d, dtype, causal, scale, O or r, None, None)


BAD, UNSUPPORTED, WORKSPACE = -1, -2, -3


@pytest.mark.parametrize("over,code", [
    (dict(cu=None), BAD), (dict(B=-1), BAD), (dict(n_q=-1), BAD), (dict(n_k=-1), BAD), (dict(Hq=5), BAD), (dict(Hq=0), BAD),
    (dict(Hkv=0), BAD), (dict(dtype=2), BAD), (dict(causal=2), BAD), (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD),
    (dict(scale=math.nan), BAD), (dict(scale=math.inf), BAD), (dict(scale=3e38), BAD), (dict(d=96), UNSUPPORTED),
    (dict(d=256), UNSUPPORTED), (dict(K=rows(row=1 << 24)), UNSUPPORTED), (dict(n_q=1 << 28), UNSUPPORTED), (dict(Q=rows(p=None)), BAD), (dict(K=rows(p=None)), BAD), (dict(V=rows(p=P + 8)), BAD),
    (dict(Q=rows(row=132)), BAD), (dict(K=rows(head=12804)), BAD), (dict(V=rows(row=-128)), BAD),
    (dict(O=rows(p=P + 2)), BAD), (dict(O=rows(row=0)), BAD), (dict(O=rows(row=64)), BAD), (dict(O=rows(head=64)), BAD),
    (dict(O=rows(head=99 * 128)), BAD), (dict(O=rows(head=128, row=3 * 128)), BAD)])
def test_prompt_attn_refuses(L, over, code):
    assert prompt(L, **over) == code


def test_key_positions_stay_in_32_bits_tiles_ahead(L):
    assert prompt(L, n_k=(1 << 30) + 1) == UNSUPPORTED and prompt(L, n_k=(1 << 31) - 1, dtype=0) == UNSUPPORTED
    assert paged(L, max_pages=(1 << 24) + 1) == UNSUPPORTED and paged(L, max_pages=(1 << 27) - 1, pg=pages(P=16)) == UNSUPPORTED


def test_prompt_attn_of_nothing_is_done_at_once(L):
    assert prompt(L, B=0) == 0 and prompt(L, n_q=0) == 0 and prompt(L, B=0, cu=None) == 0


def paged(L, Q=None, O=None, cu=P, length=P, table=P, B=1, max_pages=4, n=100, Hq=4, pg=None, dtype=1, causal=1, scale=0.1, ws=P,
          ws_bytes=1 << 40):
    r = rows()
    return L.paged_attn_fwd(Q or r, cu, length, table, B, max_pages, n, Hq, pg or pages(), dtype, causal, scale, O or r, None, ws,
                            ws_bytes, None)


@pytest.mark.parametrize("over,code", [
    (dict(cu=None), BAD), (dict(length=None), BAD), (dict(table=None), BAD), (dict(B=-1), BAD), (dict(max_pages=0), BAD),
    (dict(n=-1), BAD), (dict(Hq=3), BAD), (dict(Hq=0), BAD), (dict(dtype=0), UNSUPPORTED), (dict(dtype=5), BAD),
    (dict(causal=-1), BAD), (dict(scale=0.0), BAD), (dict(ws=None), BAD), (dict(ws=P + 16), BAD), (dict(ws_bytes=0), WORKSPACE),
    (dict(n=1 << 28), UNSUPPORTED), (dict(max_pages=1 << 26), UNSUPPORTED), (dict(pg=pages(P=48)), UNSUPPORTED), (dict(pg=pages(P=128)), UNSUPPORTED),
    (dict(pg=pages(d=32)), UNSUPPORTED), (dict(pg=pages(K8=None)), BAD), (dict(pg=pages(V8=P + 4)), BAD),
    (dict(pg=pages(kscale=None)), BAD), (dict(pg=pages(n_pages=0)), BAD), (dict(pg=pages(Hkv=0)), BAD),
    (dict(pg=pages(n_pages=1 << 26)), UNSUPPORTED), (dict(O=rows(row=0)), BAD), (dict(Q=rows(p=P + 4)), BAD)])
def test_paged_attn_refuses(L, over, code):
    assert paged(L, **over) == code


def test_paged_attn_of_nothing_is_done_at_once(L):
    assert paged(L, B=0) == 0 and paged(L, n=0) == 0


def plan(L, n_new=P, length=P, table=P, B=3, max_pages=4, pool=P, pool_n=P, n_pages=10, size=64, n_tok=5, after=P, free=P, cu=P,
         slot=P, status=P):
    return L.kv_pages_plan(n_new, length, table, B, max_pages, pool, pool_n, n_pages, size, n_tok, after, free, cu, slot, status, None)


@pytest.mark.parametrize("over,code", [
    (dict(n_new=None), BAD), (dict(length=None), BAD), (dict(table=None), BAD), (dict(pool=None), BAD), (dict(pool_n=None), BAD),
    (dict(after=None), BAD), (dict(free=None), BAD), (dict(cu=None), BAD), (dict(slot=None), BAD), (dict(status=None), BAD),
    (dict(B=-1), BAD), (dict(n_tok=-1), BAD), (dict(max_pages=0), BAD), (dict(n_pages=0), BAD), (dict(size=8), UNSUPPORTED),
    (dict(size=128), UNSUPPORTED), (dict(max_pages=1 << 26), UNSUPPORTED), (dict(n_pages=1 << 26), UNSUPPORTED)])
def test_plan_refuses(L, over, code):
    assert plan(L, **over) == code


def write(L, pg=None, K=None, V=None, dtype=1, slot=P, n=5):
    return L.kv_pages_write(pg or pages(), K or rows(), V or rows(), dtype, slot, n, None)


@pytest.mark.parametrize("over,code", [
    (dict(slot=None), BAD), (dict(n=-1), BAD), (dict(dtype=3), BAD), (dict(K=rows(p=None)), BAD), (dict(V=rows(p=P + 8)), BAD),
    (dict(K=rows(row=4)), BAD), (dict(V=rows(row=1 << 24)), UNSUPPORTED), (dict(pg=pages(P=20)), UNSUPPORTED), (dict(pg=pages(d=80)), UNSUPPORTED),
    (dict(pg=pages(vscale=None)), BAD), (dict(pg=pages(Hkv=-1)), BAD)])
def test_write_refuses(L, over, code):
    assert write(L, **over) == code


def test_write_of_nothing_is_done_at_once(L):
    assert write(L, n=0) == 0 and write(L, n=0, slot=None) == 0


def test_launches_of_more_workgroups_than_there_can_be_are_refused(L):
    """Threads are counted in 32 bits along a launch's first dimension."""
    for dtype, B in ((1, 1 << 23), (0, 1 << 24)):
        assert prompt(L, n_q=1, Hq=1, Hkv=1, B=B, dtype=dtype) == UNSUPPORTED
        assert prompt(L, n_q=1, Hq=64, Hkv=64, B=B // 64, dtype=dtype) == UNSUPPORTED
    assert prompt(L, n_q=(1 << 30) - 1, Hq=1, Hkv=1, B=1 << 22) == UNSUPPORTED
    assert write(L, n=1 << 28) == UNSUPPORTED and write(L, n=1 << 29, pg=pages(Hkv=1, P=16, d=64)) == UNSUPPORTED


def test_a_workspace_that_a_kernel_cannot_write_to_is_refused():
    """Its size alone was looked at: the address of a host tensor went to the kernel."""
    import torch
    from paper_2602_01801_amd.binding import _workspace
    dev = torch.device("cuda", 0)
    with pytest.raises(ValueError):
        _workspace(torch.empty(4096, dtype=torch.uint8), 256, dev)
    with pytest.raises(ValueError):
        _workspace(torch.empty(4096, dtype=torch.uint8, device="meta"), 256, dev)


# ------------------------------------------------------------------------------------------------ the references


def test_e4m3_rounding_is_to_the_nearest_code_ties_to_even():
    import torch
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.normal(0, 1, 4000), rng.normal(0, 200, 2000), np.ldexp(rng.normal(0, 1, 2000), -9),
                        (ref.VALUES[:126] + ref.VALUES[1:127]) / 2, ref.VALUES[:127]]).astype(np.float32)
    x = np.clip(x, -448, 448)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.code_of(ref.round_e4m3(x)), want)


def test_scale_is_the_least_power_of_two_that_fits():
    for a in (1e-20, 0.3, 1.0, 447.9, 448.0, 448.1, 896.0, 3e38):
        e = ref.scale_exp(a)
        assert 448 * 2.0 ** e >= a > 448 * 2.0 ** (e - 1)
    assert ref.scale_exp(0.0) == ref.scale_exp(1e-40) == ref.scale_exp(1e-30) == -100


def test_cells_and_rows_are_inverse():
    x = np.arange(2 * 3 * 32 * 64).reshape(2, 3, 32, 64)
    for tr in (False, True):
        c = ref.cells_of_rows(x, tr)
        assert np.array_equal(ref.rows_of_cells(c, tr), x)
        tok, co = 17, 35
        assert c[1, 2, 1, 2, 3 if tr else 1, 1 if tr else 3] == x[1, 2, tok, co]


def test_plan_reference_hands_every_page_to_one_request():
    rng = np.random.default_rng(3)
    Psz, n_pages, B = 16, 60, 7
    table, length = [[-1] * 12 for _ in range(B)], [0] * B
    pool, free = list(rng.permutation(n_pages)), n_pages
    for step in range(40):
        n_new = [int(rng.choice([-1, 0, 1, 5, 40], p=[0.1, 0.2, 0.4, 0.2, 0.1])) for _ in range(B)]
        length, free, cu, slot, status = ref.plan(n_new, length, table, pool, free, Psz, 150)
        held = [p for b in range(B) for p in table[b][: -(-length[b] // Psz)]]
        assert sorted(held + pool[:free]) == list(range(n_pages))
        assert len(set(s for s in slot.values() if s >= 0)) == sum(s >= 0 for s in slot.values())


def test_attend_leaves_out_what_a_query_does_not_see():
    rng = np.random.default_rng(5)
    Q, K, V = rng.normal(size=(2, 5, 8)), rng.normal(size=(1, 3, 8)), rng.normal(size=(1, 3, 8))
    O, lse = ref.attend(Q, K, V, True, 0.5)[:2]
    assert (O[:, :2] == 0).all() and np.isneginf(lse[:, :2]).all()
    assert np.allclose(O[:, 2], V[0, 0])
    K2, V2 = K.copy(), V.copy()
    K2[:, 2], V2[:, 2] = math.nan, math.inf
    O2, lse2 = ref.attend(Q, K2, V2, True, 0.5)[:2]
    assert np.array_equal(O2[:, :4], O[:, :4]) and np.array_equal(lse2[:, :4], lse[:, :4])
    O3 = ref.attend(Q, K, V, False, 0.5, live=np.array([True, False, True]))[0]
    assert np.allclose(O3, ref.attend(Q, K[:, ::2], V[:, ::2], False, 0.5)[0])


# ------------------------------------------------------------------------------------------------ what the GPU tests' data shows


def spread_cases():
    from test_gpu_packed import SPREAD
    return [c for c in SPREAD if sum(c[4]) < 20]   # the chunks' pages are made the same way


@pytest.mark.parametrize("case", spread_cases(), ids=str)
def test_data_of_the_paged_attention_tests_shows_a_lost_tile(case):
    """Mistakes planted in the 64-bit result: one tile of 64 keys left out, and its values those of the next tile, for every tile."""
    import torch
    from test_gpu_packed import check, prefix, spread_case
    Hq, Hkv, P, d, q, k = case
    K, ks, V, vs, table, Q = spread_case(*case, sum(k))
    b = int(np.argmax(k))
    n, ids = k[b], table[b, :-(-k[b] // P)]
    Q = Q[:, prefix(q)[b]:prefix(q)[b] + 1].double().numpy()
    K, V = ref.keys_of_pages(K, ks, ids, n, False), ref.keys_of_pages(V, vs, ids, n, True)
    want = ref.attend(Q, K, V, False, d ** -0.5)
    check(torch.from_numpy(want[0]), torch.from_numpy(want[1]), want, n, d, True)
    for t in range(-(-n // 64)):
        tile = np.arange(n) // 64 == t
        lost = ref.attend(Q, K[:, ~tile], V[:, ~tile], False, d ** -0.5)
        for o, l in ((lost[0], None), (want[0], lost[1])):
            with pytest.raises(AssertionError):
                check(torch.from_numpy(o), None if l is None else torch.from_numpy(l), want, n, d, True)
        if (t + 2) * 64 <= n:
            V2 = V.copy()
            V2[:, t * 64:(t + 1) * 64] = V[:, (t + 1) * 64:(t + 2) * 64]
            with pytest.raises(AssertionError):
                check(torch.from_numpy(ref.attend(Q, K, V2, False, d ** -0.5)[0]), None, want, n, d, True)


def weights16_cases():
    from test_gpu_packed import WEIGHTS16
    return WEIGHTS16


@pytest.mark.parametrize("case", weights16_cases(), ids=str)
def test_data_of_the_test_of_sixteen_bits_shows_eight(case):
    """The 64-bit result with every weight rounded to bf16 is outside of the bound."""
    import torch
    from test_gpu_packed import weights16_case
    Hq, Hkv, P, d, q, k = case
    _, _, Q, K, V, Or, tol = weights16_case(*case)
    off = 0
    for h in range(Hq):
        for i in range(q):
            l = K[h // (Hq // Hkv)] @ Q[h, i].double().numpy() * d ** -0.5
            w = np.exp(l - l.max())
            r = torch.from_numpy(w).bfloat16().double().numpy()
            off += (np.abs(r @ V[h // (Hq // Hkv)] / w.sum() - Or[h, i]) > tol[h, i]).sum()
            assert (np.abs(w @ V[h // (Hq // Hkv)] / w.sum() - Or[h, i]) <= tol[h, i]).all()
    assert off >= 10, off
