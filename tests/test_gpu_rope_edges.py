"""Norm and rotation, and the same on the way into pages, where a call is at an edge of what it allows: weights that are not ordinary numbers.
References and tolerances are those of share_ref.py."""
import math

import numpy as np
import pytest
import torch

import paper_2602_01801_amd as fa
import share_ref as sref
from test_gpu_packed import DT, f64, i32, prefix, view
from test_gpu_rope import check_rows, clone, make_pages, slots_of, weights

pytestmark = pytest.mark.gpu


def odd_weights(g, d, rot):
    """Ordinary weights but for a few: in coordinates that turn and in those that do not, in a lane's first piece of four and in its second."""
    w = weights(g, d)
    w[rot + 1], w[d - 2], w[5], w[rot // 2 + 9] = math.inf, math.nan, -math.inf, 2.0 ** 110
    return w


@pytest.mark.parametrize("dtype,d,rot,interleaved", [("bf16", 128, 48, False), ("f32", 128, 64, True), ("f32", 64, 32, False), ("bf16", 64, 48, True)])
def test_weights_that_are_not_finite_stay_in_their_coordinates(dtype, d, rot, interleaved):
    g = torch.Generator().manual_seed(d + rot)
    rng = np.random.default_rng(d + rot)
    q, k, P, Hkv = [37, 1, 20], [5, 30, 0], 16, 2
    n = sum(q)
    Q, K, V = view(g, 6, n, d, DT[dtype], "tokens"), view(g, Hkv, n, d, DT[dtype], "fused"), view(g, Hkv, n, d, DT[dtype], "tokens")
    freq = sref.frequencies(rot)
    rope = fa.Rope(torch.from_numpy(freq).cuda(), q_weight=odd_weights(g, d, rot), k_weight=odd_weights(g, d, rot), interleaved=interleaved)
    cu, length = i32(prefix(q).tolist()), i32([a + b for a, b in zip(q, k)])
    oq, ok = fa.qk_norm_rope(Q, K, rope, cu=cu, length=length)
    at = np.concatenate([b + np.arange(a) for a, b in zip(q, k)])[:, None].astype(float) * np.ones(rot // 2)
    with np.errstate(invalid="ignore", over="ignore"):
        check_rows(oq, Q, rope.q_weight, rope, freq, at, dtype == "bf16", "Q")
        check_rows(ok, K, rope.k_weight, rope, freq, at, dtype == "bf16", "K")
    ordinary = [c for c in range(rot, d) if c not in (rot + 1, d - 2)]
    assert torch.isfinite(oq[..., ordinary]).all() and torch.isfinite(ok[..., ordinary]).all()
    # the same in place, and on the way into pages
    again = Q.clone(), K.clone()
    fa.qk_norm_rope(*again, rope, cu=cu, length=length, out=again)
    for x, y in zip(again, (oq, ok)):
        assert np.array_equal(f64(x), f64(y), equal_nan=True)
    slot, n_pages = slots_of(rng, q, k, P)
    pages = make_pages(rng, n_pages, Hkv, P, d)
    want = clone(pages)
    fa.kv_pages_write_rope(pages, i32(slot), None, K, V, rope, cu=cu, length=length)
    fa.kv_pages_write(want, i32(slot), fa.qk_norm_rope(None, K.float(), rope, cu=cu, length=length)[1], V.float())
    for name in ("K8", "V8"):   # NaN has one code of either sign
        a, b = getattr(pages, name), getattr(want, name)
        assert torch.equal(torch.where(a & 127 == 127, 127, a), torch.where(b & 127 == 127, 127, b)), name
    assert torch.equal(pages.kscale, want.kscale) and torch.equal(pages.vscale, want.vscale)
