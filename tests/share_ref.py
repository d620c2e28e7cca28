"""References of norm and rotation, and of forking, freeing and compacting pages: plain loops in 64 bits (test infrastructure)."""
import numpy as np

import packed_ref as ref


def rope(x, w, eps, norm, freq, pos, rot, interleaved):
    """x [n, H, d] float64, w [d] or None, freq [rot/2], pos [n, rot/2] -> [n, H, d], and the sum of a pair's magnitudes at every
    coordinate that is turned (its own elsewhere), for tolerances."""
    x = np.asarray(x, np.float64).copy()
    with np.errstate(all="ignore"):
        if norm:
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
            if w is not None:
                x = x * w
        size = np.abs(x)
        if rot:
            t = pos * freq
            c, s = np.cos(t)[:, None], np.sin(t)[:, None]
            i = np.arange(rot // 2)
            ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
            a, b = x[..., ia], x[..., ib]
            x[..., ia], x[..., ib] = a * c - b * s, a * s + b * c
            size[..., ia] = size[..., ib] = np.abs(a) + np.abs(b)
    return x, size


def rope_tol(y, size, freq, pos, bf16):
    """u = 2^-24.  The sum of squares is 8 fused steps and 4 additions of what is not negative (12 u), the mean and eps 2 u, of which the
    root takes half; root and division 2 u; two products 2 u: 11 u of a coordinate.  An angle in turns is off by 2^-52 of itself (two
    products in 64 bits, here and in the reference) and by 2^-26 when its fraction (at most 1/2) goes to 32 bits: 2 pi times that; sine and
    cosine by 2^-22 beside that (bf16: 2^-16).  Products and the fused step of the turn 3 u.  Then the rounding to the type, and the
    least steps: six roundings of subnormal numbers, half a step each, in fp32; one in bf16."""
    u = 2.0 ** -24
    far = np.abs(pos * freq).max() if freq.size and pos.size else 0.0
    delta = (2.0 ** -16 if bf16 else 2.0 ** -22) + 2.0 ** -23 + far * 2.0 ** -50
    return (14 * u + delta) * size + (2.0 ** -8 if bf16 else u) * np.abs(y) + (2.0 ** -133 if bf16 else 2.0 ** -147)


def held(table, length, n_pages, P):
    """Pages that every request holds, by table entries: [(entry, page or None)] per request."""
    W = len(table[0]) if len(table) else 0
    out = []
    for row, n in zip(table, length):
        n = min(max(n, 0), W * P)
        out.append([p if 0 <= p < n_pages else None for p in row[:-(-n // P)]])
    return out


def cut(n, hi):
    return min(max(n, 0), hi)


def fork(parent, child, keep, length, table, pool, pool_n, P, n_pages):
    """kv_pages_fork, one after the other; table (lists) is changed.  Returns lengths, free pages, status, copies [(from, to)]."""
    B, W = len(table), len(table[0]) if len(table) else 0
    before = [list(r) for r in table]
    after, status, copies, seen = list(length), [], [], set()
    free = cut(pool_n, n_pages)
    asked = taken = 0
    for i, (p, c) in enumerate(zip(parent, child)):
        if not (0 <= p < B and 0 <= c < B) or length[c] > 0 or c in seen:
            status.append(2)
            if 0 <= c < B:
                seen.add(c)
            continue
        seen.add(c)
        L = cut(length[p], W * P)
        m = L if keep is None else cut(keep[i], L)
        last = before[p][m // P] if m % P else None
        need = last is not None and 0 <= last < n_pages
        asked += need
        if need and asked > free:
            status.append(1)
            continue
        status.append(0)
        after[c] = m
        table[c][:m // P] = before[p][:m // P]
        if need:
            taken += 1
            page = pool[free - asked]
            table[c][m // P] = page
            if 0 <= page < n_pages:
                copies.append((last, page))
        elif last is not None:
            table[c][m // P] = last
    return after, free - taken, status, copies


def give_back(before, gone, pool, free, n_pages):
    """gone: [(page)] in the order of requests and tables.  A page whose holders all give it up goes to the pool with the last of them."""
    count = {}
    for pages in before:
        for p in pages:
            if p is not None:
                count[p] = count.get(p, 0) + 1
    for p in gone:
        count[p] -= 1
        if count[p] == 0 and free < n_pages:
            pool[free] = p
            free += 1
    return free


def free(keep, length, table, pool, pool_n, P, n_pages):
    """kv_pages_free; pool (a list) is changed."""
    W = len(table[0]) if len(table) else 0
    before = held(table, length, n_pages, P)
    flat = [p for pages in before for p in pages]
    after, status, gone = [], [], []
    for b, pages in enumerate(before):
        L = cut(length[b], W * P)
        stay = cut(keep[b], L)
        refused = stay < L and stay % P and pages[stay // P] is not None and flat.count(pages[stay // P]) > 1
        if refused:
            stay = L
        gone += [p for p in pages[-(-stay // P):] if p is not None]
        after.append(stay)
        status.append(int(bool(refused)))
    return after, give_back(before, gone, pool, cut(pool_n, n_pages), n_pages), status


def compact(keep, length, table, pool, pool_n, P, n_pages):
    """kv_pages_compact.  Returns lengths, tables, pool, free pages, status, made {fresh page: [(old page, offset)]}."""
    W = len(table[0]) if len(table) else 0
    before = held(table, length, n_pages, P)
    free0 = cut(pool_n, n_pages)
    out, new, status, gone, made = [], [], [], [], {}
    asked = top = 0
    for b, pages in enumerate(before):
        L = cut(length[b], W * P)
        tokens = [i for i in range(L) if keep[b][i] and pages[i // P] is not None]
        groups = [tokens[j:j + P] for j in range(0, len(tokens), P)]
        whole = {}
        for j, g in enumerate(groups):
            s = g[0] // P
            if g == list(range(s * P, min(s * P + P, L))):
                whole[j] = s
        need = len(groups) - len(whole)
        asked += need
        if need and asked > free0:
            out.append(L)
            new.append(list(table[b]))
            status.append(1)
            continue
        row = []
        for j, g in enumerate(groups):
            if j in whole:
                row.append(pages[whole[j]])
                continue
            page = pool[free0 - 1 - top]
            top += 1
            row.append(page)
            made[page] = [(pages[i // P], i % P) for i in g]
        new.append(row + [-1] * (W - len(row)))
        out.append(len(tokens))
        status.append(0)
        gone += [p for s, p in enumerate(pages) if p is not None and s not in whole.values()]
    pool = list(pool)
    return out, new, pool, give_back(before, gone, pool, free0 - top, n_pages), status, made


def compact_codes(code, scale, transposed, made):
    """The fresh pages' codes and scales; code [n,H,...] and scale [n,H] are changed."""
    old, old_scale = ref.rows_of_cells(code, transposed).copy(), scale.copy()
    rows = old.copy()
    for page, src in made.items():
        if not 0 <= page < len(code):
            continue
        s = np.max([old_scale[p] for p, _ in src], 0)
        rows[page] = 0
        for t, (p, o) in enumerate(src):
            for h in range(scale.shape[1]):
                x = old[p, h, o]
                if old_scale[p, h] != s[h]:
                    x = ref.code_of(ref.round_e4m3(ref.VALUES[x] * (old_scale[p, h] / s[h])))
                rows[page, h, t] = x
        scale[page] = s
    code[...] = ref.cells_of_rows(rows, transposed)


def frequencies(rot, base=10000.0):
    return base ** (-np.arange(0, rot, 2) / max(rot, 1))


