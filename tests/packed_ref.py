"""References of the calls over packed sequences and paged caches: plain loops in 64 bits (test infrastructure)."""
import math

import numpy as np

SCALE_MIN_EXP = -100


def e4m3_values() -> np.ndarray:
    """The 256 codes: sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7F and 0xFF are no numbers."""
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = math.nan if (c & 127) == 127 else (-x if c >> 7 else x)
    return v


VALUES = e4m3_values()


def round_e4m3(x):
    """Nearest value of the format, ties to even; beyond 448 the largest; NaN stays."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.maximum(np.floor(np.log2(np.where(a > 0, a, 1.0))), -6)
    step = 2.0 ** (e - 3)
    return np.copysign(np.minimum(np.round(a / step) * step, 448.0), x)   # zeros keep their sign


def scale_exp(amax: float) -> int:
    """Exponent of the least power of two, 2^-100 at least, whose 448-fold is not below amax."""
    if amax == 0:
        return SCALE_MIN_EXP
    m, e = math.frexp(amax)
    return max(SCALE_MIN_EXP, e - 9 if m <= 0.875 else e - 8)


def rows_of_cells(code, transposed):
    """[n, H, P/16, d/16, 16, 16] -> [n, H, P, d]."""
    n, H, pb, db = code.shape[:4]
    if transposed:
        code = code.swapaxes(4, 5)
    return code.transpose(0, 1, 2, 4, 3, 5).reshape(n, H, 16 * pb, 16 * db)


def cells_of_rows(x, transposed):
    n, H, P, d = x.shape
    x = x.reshape(n, H, P // 16, 16, d // 16, 16).transpose(0, 1, 2, 4, 3, 5)
    return np.ascontiguousarray(x.swapaxes(4, 5) if transposed else x)


def attend(Q, K, V, causal, scale, live=None):
    """One sequence.  Q [Hq,a,d], K, V [Hkv,n,d] float64; live [n] keys that exist (None: all).  Returns (O, lse, A, S, max|v|):
    A = sum of weights times |v| per output, S = the largest sum |q||k| * scale of a query, for tolerances."""
    Hq, a, d = Q.shape
    Hkv, n, _ = K.shape
    O, A = np.zeros((Hq, a, d)), np.zeros((Hq, a, d))
    lse, S = np.full((Hq, a), -math.inf), np.zeros((Hq, a))
    live = np.ones(n, bool) if live is None else live
    for h in range(Hq):
        k, v = K[h // (Hq // Hkv)], V[h // (Hq // Hkv)]
        for i in range(a):
            see = live & (np.arange(n) <= n - a + i) if causal else live
            if not see.any():
                continue
            l = k[see] @ Q[h, i] * scale
            m = l.max()
            w = np.exp(l - m)
            z = w.sum()
            O[h, i], A[h, i] = w @ v[see] / z, w @ np.abs(v[see]) / z
            lse[h, i] = m + math.log(z)
            S[h, i] = (np.abs(k[see]) @ np.abs(Q[h, i])).max() * scale
    fin = np.abs(V[np.isfinite(V)])
    return O, lse, A, S, fin.max() if fin.size else 0.0


def plan(n_new, length, table, pool, pool_n, P, n_tok):
    """kv_pages_plan, request by request; table and pool (lists) are changed."""
    B, n_pages = len(n_new), len(pool)
    max_pages = len(table[0]) if B else 0
    held = [min(max(x, 0), max_pages * P) for x in length]
    free = min(max(pool_n, 0), n_pages)
    for b in range(B):
        if n_new[b] < 0:
            for j in range(-(-held[b] // P)):
                if free < n_pages:
                    pool[free] = table[b][j]
                    free += 1
    cu, slot, status, after = [0], {}, [], []
    rows = asked = 0
    top = free
    for b in range(B):
        n, st = max(n_new[b], 0), 0
        have, want = -(-held[b] // P), -(-(held[b] + n) // P)
        rows += n
        if want > max_pages:
            st = 2
        elif n > 0 and rows > n_tok:
            st = 3
        ask = 0 if st or n_new[b] < 0 else want - have
        asked += ask
        if ask and asked > free:
            st = 1
        if ask and not st:
            for j in range(ask):
                top -= 1
                table[b][have + j] = pool[top]
        cu.append(min(rows, n_tok))
        for i in range(cu[b + 1] - cu[b]):
            page = -1 if st else table[b][(held[b] + i) // P]
            slot[cu[b] + i] = page * P + (held[b] + i) % P if 0 <= page < n_pages else -1
        status.append(st)
        after.append(0 if n_new[b] < 0 else held[b] if st else held[b] + n)
    return after, top, cu, slot, status


def write(code, scale, transposed, x, slot, P):
    """kv_pages_write for one of the tensors, run by run: code [n,H,...] and scale [n,H] are changed; x [H,n,d] float64."""
    n_pages, H = scale.shape
    rows = rows_of_cells(code, transposed).copy()
    t, n = 0, len(slot)
    ok = lambda i: 0 <= slot[i] < n_pages * P
    while t < n:
        if not ok(t):
            t += 1
            continue
        e = t + 1
        while e < n and ok(e) and slot[e] == slot[e - 1] + 1 and slot[e] % P:
            e += 1
        page, o = slot[t] // P, slot[t] % P
        for h in range(H):
            v = x[h, t:e]
            fin = np.abs(v[np.isfinite(v)])
            s = 2.0 ** scale_exp(fin.max() if fin.size else 0.0)
            if o > 0:
                old = float(scale[page, h])
                if old >= s:
                    s = old
                else:
                    rows[page, h] = code_of(round_e4m3(VALUES[rows[page, h]] * (old / s)))
            scale[page, h] = s
            rows[page, h, o:o + e - t] = code_of(round_e4m3(v / s))
        t = e
    code[...] = cells_of_rows(rows, transposed)


def code_of(v):
    """Codes of values of the format; zeros keep their sign, NaN is 0x7F."""
    v = np.asarray(v, np.float64)
    a = np.abs(v)
    order = VALUES[:127]
    c = np.searchsorted(order, np.where(np.isnan(a), 0, a))
    c = np.where(np.isnan(v), 127, np.minimum(c, 126))
    return np.where(~np.isnan(v) & np.signbit(v), c | 128, c).astype(np.uint8)


def spread_pages(rng, n, Hkv, P, spare=2, d=128):
    """Pages of n tokens in any order and their block table, for tests that notice a tile of 64 keys that is lost or read wrongly: keys of 0.5 to 2, so that
    scores of ordinary queries spread by about one and no key rules a row; values of 1 to 2 of either sign and, in one coordinate that is
    the tile's, of 256.  Page by page a scale of its own."""
    per = -(-n // P)
    n_pages = per + spare
    sign = lambda: 128 * rng.integers(0, 2, size=(n_pages, Hkv, P, d))
    K = rng.integers(0x30, 0x40, size=(n_pages, Hkv, P, d)) | sign()
    V = rng.integers(0x38, 0x40, size=K.shape) | sign()
    table = rng.permutation(n_pages)[:per].astype(np.int32)
    for j in range(n):
        V[table[j // P], :, j % P, j // 64 % d] = 0x78
    scale = lambda: 2.0 ** rng.integers(-1, 2, size=(n_pages, Hkv))
    return cells_of_rows(K.astype(np.uint8), False), scale(), cells_of_rows(V.astype(np.uint8), True), scale(), table


def keys_of_pages(code, scale, table, n, transposed):
    """[Hkv, n, d] float64 of a sequence; zeros for pages that do not exist."""
    n_pages = code.shape[0]
    rows = VALUES[rows_of_cells(code, transposed)] * scale[:, :, None, None]
    out = [rows[p] if 0 <= p < n_pages else np.zeros_like(rows[0]) for p in table]
    return np.concatenate(out, 1)[:, :n] if out else rows[0][:, :0]
