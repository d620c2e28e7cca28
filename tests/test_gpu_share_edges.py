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
from test_gpu_share import ints, layout

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
