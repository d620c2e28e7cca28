"""Attention for several requests at a time: prompts in one piece, and a paged cache in 8 bits.

Four operators that a serving program calls one after the other: kv_pages_plan (block tables and slot maps from the
requests' lengths), kv_pages_write (new keys and values into pages of E4M3 codes with a scale per page and head),
paged_attn_fwd (attention over those pages, for single tokens and chunks), and prompt_attn_fwd (attention over whole
packed prompts).  Every case is one call of one of them.

Sequence lengths of a case follow from its own numbers alone (`lens`); values come from the seed.  Keys lie in clusters,
a few coordinates are much larger than the others, and heads differ in magnitude, as trained projections do; values
differ in magnitude between heads by powers of ten.
"""
import math
import random

import torch

own = False

ROWS_AT_ONCE = 1 << 28   # scores that the plain form holds at a time (elements)


# ---------------------------------------------------------------------------------------------------- cases

def _prompt(**over):
    return dict(dict(op="prompt", dtype="bf16", d=128, Hq=12, Hkv=12, causal=True, B=1, q_lo=64, q_hi=64, k_lo=0, k_hi=0,
                     lens_seed=1, fused=False), **over)


def _paged(**over):
    return dict(dict(op="paged", d=128, Hq=40, Hkv=8, P=64, causal=True, B=1, q_lo=1, q_hi=1, k_lo=1560, k_hi=1560,
                     lens_seed=1), **over)


def _write(**over):
    return dict(dict(op="write", dtype="bf16", d=128, Hkv=8, P=64, B=1, q_lo=1, q_hi=1, k_lo=0, k_hi=0, lens_seed=1),
                **over)


def _plan(**over):
    return dict(dict(op="plan", P=64, B=64, q_lo=1, q_hi=1, k_lo=0, k_hi=4680, max_pages=512, ended=0, short=0,
                     lens_seed=1), **over)


def listed():
    return [
        # three short prompts of a small model with 64-wide heads, one of them a single token: launch latency
        _prompt(name="prompt_tiny", d=64, Hq=4, Hkv=2, B=3, q_lo=1, q_hi=77, lens_seed=4),
        # fp32: frames of two videos and their prompts of different lengths, every token sees the whole prompt
        _prompt(name="prompt_cross_f32", dtype="f32", Hq=4, Hkv=4, causal=False, B=4, q_lo=390, q_hi=780, k_lo=64, k_hi=512),
        # a batch of ragged prompts at the world-model layer with grouped heads, read from a fused projection's output
        _prompt(name="prompt_batch", Hq=40, Hkv=8, B=14, q_lo=65, q_hi=3600, fused=True, lens_seed=2),
        # the longest prompt: 21 frames of 1560 tokens at the Wan-shaped layer's heads, three of them on a key head
        _prompt(name="prompt_long", Hq=12, Hkv=4, q_lo=32760, q_hi=32760),
        # the next token of one request with a short cache and pages of 16: launch latency
        _paged(name="token_one", Hq=12, Hkv=12, P=16),
        # the next token of a batch of requests of very different lengths
        _paged(name="token_batch", B=48, k_lo=100, k_hi=37440, lens_seed=3),
        # the next token of two requests at the end of a long rollout: few heads, a long axis
        _paged(name="token_long", B=2, k_lo=199999, k_hi=230400),
        # the next chunk of five requests: 201 to 780 new tokens each over caches of many frames
        _paged(name="chunk_batch", Hq=12, Hkv=4, P=32, B=5, q_lo=201, q_hi=780, k_lo=4680, k_hi=37440, lens_seed=5),
        # one token each of a batch of requests into their half-filled pages
        _write(name="write_token", P=16, B=96, k_lo=1, k_hi=4680),
        # prompts of a batch of requests into fresh pages, some of them behind tokens that are there
        _write(name="write_prompt", B=20, q_lo=201, q_hi=4680, k_lo=0, k_hi=99, lens_seed=2),
        # a step of a batch of requests: one token each, some requests have ended
        _plan(name="plan_step", P=16, B=192, ended=9, max_pages=2340),
        # a batch of prompts is admitted, until the pages run out
        _plan(name="plan_prompt", B=64, q_lo=201, q_hi=4680, k_lo=0, k_hi=0, short=40),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    op = rng.choice(["prompt", "prompt", "paged", "paged", "paged", "write", "plan"])
    heads = rng.choice([(12, 12), (12, 4), (40, 8), (40, 40), (8, 1), (4, 2), (14, 2), (5, 5), (24, 3)])
    seed = rng.randrange(1 << 30)
    if op == "prompt":
        f32 = rng.random() < 0.25
        hi = log(16, 8000 if f32 else 16000)
        B = min(log(1, 32), max(1, 40000 // hi))
        c = _prompt(dtype="f32" if f32 else "bf16", d=rng.choice([64, 128]), Hq=heads[0], Hkv=heads[1],
                    causal=rng.random() < 0.7, B=B, q_lo=max(1, hi // rng.choice([1, 3, 40])), q_hi=hi, lens_seed=seed,
                    fused=rng.random() < 0.4)
        if rng.random() < 0.3:
            c.update(k_lo=log(1, 512), fused=False)
            c["k_hi"] = c["k_lo"] + log(1, 2000)
        while work(c)["flops"] > (2.5e11 if f32 else 1.5e12):
            c["q_hi"] = max(16, c["q_hi"] // 2)
            c["q_lo"] = min(c["q_lo"], c["q_hi"])
        return c
    if op == "paged":
        token = rng.random() < 0.65
        hi = log(16, 200000 if token else 30000)
        B = min(log(1, 128), max(1, 400000 // hi))
        q = (1, rng.choice([1, 1, 1, 3, 8])) if token else (1, log(16, 900))
        c = _paged(d=rng.choice([64, 128, 128]), Hq=heads[0], Hkv=heads[1], P=rng.choice([16, 32, 64]),
                   causal=rng.random() < 0.8, B=B, q_lo=q[0], q_hi=q[1], k_lo=max(1, hi // rng.choice([1, 3, 40])), k_hi=hi,
                   lens_seed=seed)
        while work(c)["flops"] > 6e11 or work(c)["bytes"] > 9e8:
            c["k_hi"] = max(16, c["k_hi"] // 2)
            c["k_lo"] = min(c["k_lo"], c["k_hi"])
        return c
    if op == "write":
        hi = log(1, 8000)
        B = min(log(1, 256), max(1, 50000 // hi))
        return _write(dtype=rng.choice(["bf16", "bf16", "f32"]), d=rng.choice([64, 128]), Hkv=rng.choice([1, 4, 5, 8, 12]),
                      P=rng.choice([16, 32, 64]), B=B, q_lo=max(1, hi // rng.choice([1, 3, 40])), q_hi=hi,
                      k_lo=0, k_hi=log(1, 4680), lens_seed=seed)
    B = log(1, 1500)
    hi = log(1, 4680)
    return _plan(P=rng.choice([16, 32, 64]), B=B, q_lo=0 if rng.random() < 0.3 else 1, q_hi=max(1, min(hi, 150000 // B)),
                 k_lo=0, k_hi=log(1, 8000), max_pages=rng.choice([200, 700]), ended=rng.choice([0, 0, B // 9]),
                 short=rng.choice([0, 0, 30, 60]), lens_seed=seed)


def _spread(rng, lo, hi):
    """A length between the two, spread over its logarithm."""
    lo1 = max(lo, 1)
    n = int(math.exp(rng.uniform(math.log(lo1), math.log(hi + 1)))) if hi >= lo1 else hi
    if lo < 1 and rng.random() < 0.2:
        n = 0
    return max(lo, min(hi, n))


def lens(case):
    """(queries or new tokens, keys or tokens that are there) of every sequence; the first is the longest, the last the shortest."""
    rng = random.Random(case["lens_seed"])
    B = case["B"]
    q = [_spread(rng, case["q_lo"], case["q_hi"]) for _ in range(B)]
    k = [_spread(rng, case["k_lo"], case["k_hi"]) for _ in range(B)]
    q[0], k[0] = case["q_hi"], case["k_hi"]
    if B > 1:
        q[-1], k[-1] = case["q_lo"], case["k_lo"]
    if case["op"] == "prompt" and case["k_hi"] == 0:
        k = list(q)
    if case["op"] == "paged":   # the keys hold the queries' own, but for a sequence now and then
        k = [max(a, b) if i % 7 else b for i, (a, b) in enumerate(zip(q, k))]
    return q, k


def _pairs(case):
    """(query, key) pairs that are not masked."""
    q, k = lens(case)
    n = 0
    for a, b in zip(q, k):
        if not case["causal"]:
            n += a * b
        else:   # query i sees the keys up to b - a + i
            lo = max(0, a - b)
            n += sum_range(b - a + lo + 1, b)
    return n


def sum_range(lo, hi):
    return (lo + hi) * (hi - lo + 1) // 2 if hi >= lo else 0


def work(case):
    q, k = lens(case)
    nq, nk = sum(q), sum(k)
    if case["op"] in ("prompt", "paged"):
        d, Hq, Hkv = case["d"], case["Hq"], case["Hkv"]
        elt = 2 if case["op"] == "paged" or case["dtype"] == "bf16" else 4
        kv = 1 if case["op"] == "paged" else elt
        return {"bytes": 2 * elt * nq * Hq * d + 2 * kv * nk * Hkv * d + 4 * nq * Hq, "flops": 4 * d * Hq * _pairs(case)}
    if case["op"] == "write":
        elt = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * nq * case["Hkv"] * case["d"] * (elt + 1), "flops": 4 * nq * case["Hkv"] * case["d"]}
    return {"bytes": 4 * nq + 28 * case["B"] + 8 * nq // case["P"], "flops": nq}


# ---------------------------------------------------------------------------------------------------- inputs

def _prefix(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


def _ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def _heads(g, H, n, d, dtype, spread, cluster):
    """[n, H, d]: clusters of neighbouring rows, some large coordinates, heads of different magnitude."""
    dev = "cuda"
    mag = torch.exp2((torch.rand(H, generator=g, device=dev) - 0.5) * spread)
    coord = torch.ones(d, device=dev)
    coord[torch.randperm(d, generator=g, device=dev)[: d // 32]] = 4.0
    out = torch.empty((n, H, d), dtype=dtype, device=dev)
    cen = torch.randn((64, H, d), generator=g, device=dev)
    step = max(1, (1 << 27) // (H * d))
    for a in range(0, n, step):
        b = min(n, a + step)
        x = torch.randn((b - a, H, d), generator=g, device=dev)
        if cluster:
            which = (torch.arange(a, b, device=dev) // 13) % 64
            x = 0.8 * x + 0.6 * cen[which]
        out[a:b] = (x * coord * mag[:, None]).to(dtype)
    return out


def _queries(g, H, n, d, dtype):
    return torch.randn((n, H, d), generator=g, device="cuda").mul_(1.3).to(dtype)


def _cells(x, P, transposed):
    """[n_pages * P, H, d] -> [n_pages, H, P/16, d/16, 16, 16]: tokens before coordinates in a cell, or coordinates first."""
    n, H, d = x.shape
    x = x.reshape(n // P, P // 16, 16, H, d // 16, 16)
    return x.permute(0, 3, 1, 4, 5, 2).contiguous() if transposed else x.permute(0, 3, 1, 4, 2, 5).contiguous()


def _scale_of(amax):
    """Least power of two (2^-100 at least) whose 448-fold is not below amax."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return ((e.clamp(min=-100).to(torch.int32) + 127) << 23).view(torch.float32)


def _pages(g, n_pages, Hkv, P, d):
    """Pages of codes and their scales, the values between heads and pages of different magnitude."""
    out = []
    for spread, transposed in ((2.0, False), (8.0, True)):
        code = torch.empty((n_pages, Hkv, P // 16, d // 16, 16, 16), dtype=torch.uint8, device="cuda")
        scale = torch.empty((n_pages, Hkv), dtype=torch.float32, device="cuda")
        mag = torch.exp2((torch.rand(Hkv, generator=g, device="cuda") - 0.5) * spread)
        step = max(1, (1 << 26) // (Hkv * P * d))
        for a in range(0, n_pages, step):
            b = min(n_pages, a + step)
            x = torch.randn(((b - a), Hkv, P * d), generator=g, device="cuda") * mag[:, None]
            if not transposed:
                x *= torch.exp2(torch.randn((b - a, Hkv, 1), generator=g, device="cuda") * 0.3)
            s = _scale_of(x.abs().amax(-1))
            c = (x / s[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
            code[a:b] = c.view(b - a, Hkv, P // 16, d // 16, 16, 16)
            scale[a:b] = s
        out += [code, scale]
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * (seed + 1) + case["lens_seed"] % 1000)
    q, k = lens(case)
    s = {"case": case, "q": q, "k": k, "cu_q": _ints(_prefix(q))}
    nq = sum(q)
    if case["op"] == "prompt":
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        d, Hq, Hkv, nk = case["d"], case["Hq"], case["Hkv"], sum(k)
        Q, K, V = _queries(g, Hq, nq, d, dt), _heads(g, Hkv, nk, d, dt, 2.0, True), _heads(g, Hkv, nk, d, dt, 8.0, False)
        if case["fused"]:   # views of one projection's output
            Q, K, V = torch.cat([Q, K, V], 1).split([Hq, Hkv, Hkv], 1)
        s.update(Q=Q.transpose(0, 1), K=K.transpose(0, 1), V=V.transpose(0, 1), cu_k=_ints(_prefix(k)), scale=d ** -0.5,
                 out=(torch.empty((nq, Hq, d), dtype=dt, device="cuda").transpose(0, 1),
                      torch.empty((Hq, nq), dtype=torch.float32, device="cuda")))
        return s
    P = case["P"]
    if case["op"] == "paged":
        d, Hq, Hkv = case["d"], case["Hq"], case["Hkv"]
        per = [-(-x // P) for x in k]
        n_pages = sum(per) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).cpu()
        table = torch.full((case["B"], max(1, max(per))), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(per):
            table[b, :n] = order[at:at + n]
            at += n
        s.update(Q=_queries(g, Hq, nq, d, torch.bfloat16).transpose(0, 1), table=table.cuda(), len=_ints(k), scale=d ** -0.5,
                 pages=_pages(g, n_pages, Hkv, P, d),
                 out=(torch.empty((nq, Hq, d), dtype=torch.bfloat16, device="cuda").transpose(0, 1),
                      torch.empty((Hq, nq), dtype=torch.float32, device="cuda")))
        if own:
            import paper_2602_01801_amd as fa
            s["handle"] = fa.Pages(*s["pages"])
            s["ws"] = torch.empty(fa.workspace_bytes(fa.OP_PAGED_ATTN, Hq, nq, 0), dtype=torch.uint8, device="cuda")
        return s
    if case["op"] == "write":
        d, Hkv = case["d"], case["Hkv"]
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        per = [-(-(a + b) // P) - b // P for a, b in zip(q, k)]   # pages that are written to
        n_pages = sum(per) + 2
        order = torch.randperm(n_pages, generator=g, device="cuda").cpu().tolist()
        slot, at = [], 0
        for a, b, n in zip(q, k, per):
            o = b % P
            slot += [order[at + (o + i) // P] * P + (o + i) % P for i in range(a)]
            at += n
        kv = torch.cat([_heads(g, Hkv, nq, d, dt, 2.0, True), _heads(g, Hkv, nq, d, dt, 8.0, False)], 1)
        s.update(K=kv[:, :Hkv].transpose(0, 1), V=kv[:, Hkv:].transpose(0, 1), slot=_ints(slot),
                 pages=_pages(g, n_pages, Hkv, P, d))
        if own:
            import paper_2602_01801_amd as fa
            s["handle"] = fa.Pages(*s["pages"])
        return s
    # plan: which pages a request holds, and the free ones, in an order that a long run leaves behind
    rng = random.Random(case["lens_seed"] + 77)
    gone = set(rng.sample(range(case["B"]), min(case["ended"], case["B"])))
    n_new = [-1 if b in gone else n for b, n in enumerate(q)]
    per = [-(-x // P) for x in k]
    need = sum(-(-(a + b) // P) for a, b in zip(q, k))
    free = need * (100 - case["short"]) // 100 + 5
    n_pages = sum(per) + free
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).cpu()
    table = torch.full((case["B"], case["max_pages"]), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(per):
        m = min(n, case["max_pages"])
        table[b, :m] = order[at:at + m]
        k[b] = min(k[b], m * P)
        at += m
    pool = torch.full((n_pages,), -1, dtype=torch.int32)
    pool[: n_pages - at] = order[at:]
    i32 = lambda *n: torch.empty(n, dtype=torch.int32, device="cuda")
    n_tok = sum(max(x, 0) for x in n_new)
    s.update(n_new=_ints(n_new), len=_ints(k), table=table.cuda(), pool=pool.cuda(), pool_n=_ints([n_pages - at]), n_tok=n_tok,
             out=(i32(case["B"]), i32(1), i32(case["B"] + 1), i32(n_tok), i32(case["B"])))
    return s


# ---------------------------------------------------------------------------------------------------- plain forms

def _decode(code, scale, ids, n, transposed, dtype=torch.float32, table=None):
    """Rows 0 .. n-1 of the pages `ids`: [Hkv, n, d]."""
    x = code[ids]
    x = x.view(torch.float8_e4m3fn).to(dtype) if table is None else table[x.long()]
    x = x * scale[ids].to(dtype)[:, :, None, None, None, None]
    x = x.permute(1, 0, 2, 5, 3, 4) if transposed else x.permute(1, 0, 2, 4, 3, 5)
    H, npg, pb, _, db, _ = x.shape
    return x.reshape(H, npg * pb * 16, db * 16)[:, :n]


def _attend(Q, K, V, causal, scale, dtype=torch.float32):
    """Q [Hq,a,d], K, V [Hkv,b,d] -> O [Hq,a,d], lse [Hq,a]; query i sees the keys up to b - a + i if causal."""
    Hq, a, d = Q.shape
    Hkv, b, _ = K.shape
    O = torch.zeros((Hq, a, d), dtype=dtype, device=Q.device)
    lse = torch.full((Hq, a), -math.inf, dtype=dtype, device=Q.device)
    if a == 0 or b == 0:
        return O, lse
    K, V = K.to(dtype), V.to(dtype)
    per = Hq // Hkv
    rows = max(1, ROWS_AT_ONCE // (per * b))
    for h in range(Hkv):
        Kt, Vh = K[h].t().contiguous(), V[h].contiguous()
        for r in range(0, a, rows):
            e = min(a, r + rows)
            q = Q[h * per:(h + 1) * per, r:e].to(dtype).reshape(per * (e - r), d)
            x = (q @ Kt).mul_(scale).view(per, e - r, b)
            if causal:
                i = torch.arange(r, e, device=Q.device)[:, None] + (b - a)
                x.masked_fill_(torch.arange(b, device=Q.device)[None] > i, -math.inf)
            m = x.amax(-1, keepdim=True)
            m = torch.where(m == -math.inf, torch.zeros_like(m), m)
            x = x.sub_(m).exp_()
            l = x.sum(-1, keepdim=True)
            o = (x.view(per * (e - r), b) @ Vh).view(per, e - r, d)
            O[h * per:(h + 1) * per, r:e] = torch.where(l > 0, o / l, torch.zeros_like(o))
            lse[h * per:(h + 1) * per, r:e] = (torch.log(l) + m)[..., 0]
    return O, lse


def _plain_prompt(s, dtype=torch.float32):
    Q, K, V, case = s["Q"], s["K"], s["V"], s["case"]
    O = torch.empty(Q.shape, dtype=dtype, device="cuda")
    lse = torch.empty(Q.shape[:2], dtype=dtype, device="cuda")
    cq, ck = _prefix(s["q"]), _prefix(s["k"])
    for b in range(case["B"]):
        i, j = slice(cq[b], cq[b + 1]), slice(ck[b], ck[b + 1])
        O[:, i], lse[:, i] = _attend(Q[:, i], K[:, j], V[:, j], case["causal"], s["scale"], dtype)
    return O, lse


def _plain_paged(s, dtype=torch.float32, table=None):
    Q, case = s["Q"], s["case"]
    K8, ks, V8, vs = s["pages"]
    O = torch.empty(Q.shape, dtype=dtype, device="cuda")
    lse = torch.empty(Q.shape[:2], dtype=dtype, device="cuda")
    cq = _prefix(s["q"])
    for b in range(case["B"]):
        i, n = slice(cq[b], cq[b + 1]), s["k"][b]
        ids = s["table"][b, : -(-n // case["P"])].long()
        K, V = _decode(K8, ks, ids, n, False, dtype, table), _decode(V8, vs, ids, n, True, dtype, table)
        O[:, i], lse[:, i] = _attend(Q[:, i], K, V, case["causal"], s["scale"], dtype)
    return O, lse


def _to_rows(code):
    """Cells [n, H, P/16, d/16, 16, 16] of keys -> [n, P, H, d]."""
    n, H, pb, db, _, _ = code.shape
    return code.permute(0, 2, 4, 1, 3, 5).reshape(n, pb * 16, H, db * 16)


def _plain_write(s):
    P, slot = s["case"]["P"], s["slot"].long()
    page, off = slot // P, slot % P
    K8, ks, V8, vs = s["pages"]
    fresh = torch.zeros(K8.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, page[off == 0], True)
    touched = torch.zeros(K8.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, page, True)
    for x, code, scale, tr in ((s["K"], K8, ks, False), (s["V"], V8, vs, True)):
        x = x.transpose(0, 1).float()
        amax = torch.zeros_like(scale).scatter_reduce_(0, page[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
        need = _scale_of(amax)
        new = torch.where(fresh[:, None], need, torch.maximum(scale, need))
        new = torch.where(touched[:, None], new, scale)
        ratio = torch.where(fresh[:, None], torch.ones_like(new), scale / new)
        rows = code.transpose(4, 5) if tr else code
        rows = _to_rows(rows).view(torch.float8_e4m3fn).float() * ratio[:, None, :, None]
        rows[page, off] = (x / new[page][..., None]).clamp(-448.0, 448.0)
        rows = rows.to(torch.float8_e4m3fn).view(torch.uint8)
        code.copy_(_cells(rows.reshape(-1, *rows.shape[2:]), P, tr))
        scale.copy_(new)
    return K8.view(torch.float8_e4m3fn), ks, V8.view(torch.float8_e4m3fn), vs


def _plain_plan(s):
    P, n_new, length, table, pool = s["case"]["P"], s["n_new"].long(), s["len"].long(), s["table"], s["pool"]
    free = s["pool_n"].long()
    B, max_pages = table.shape
    col = torch.arange(max_pages, device="cuda")[None]
    ended = n_new < 0
    n = n_new.clamp(min=0)
    have = torch.minimum((length + P - 1) // P, torch.full_like(length, max_pages))
    # pages of ended requests go on top of the pool, in the order of requests and of their tables
    back = torch.where(ended, have, torch.zeros_like(have))
    first = back.cumsum(0) - back
    give = col < back[:, None]
    pool[(free + first[:, None] + col)[give]] = table[give]
    free = free + back.sum()
    # requests in order take pages from the top; one whose pages are not there (or do not fit its table) stays as it is
    want = (length + n + P - 1) // P
    long = ~ended & (want > max_pages)
    need = torch.where(ended | long, torch.zeros_like(want), (want - have).clamp(min=0))
    upto = need.cumsum(0)
    refused = long | ((need > 0) & (upto > free))
    take = torch.where(refused, torch.zeros_like(need), need)
    first = take.cumsum(0) - take
    j = col - have[:, None]
    new = (j >= 0) & (j < take[:, None])
    table[new] = pool[(free - 1 - first[:, None] - j)[new]]
    after = torch.where(ended, torch.zeros_like(length), torch.where(refused, length, length + n))
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), n.cumsum(0)])
    t = torch.arange(s["n_tok"], device="cuda")
    b = torch.searchsorted(cu[1:], t, right=True)
    pos = length[b] + t - cu[b]
    page = table[b, (pos // P).clamp(max=max_pages - 1)].long()
    slot = torch.where(refused[b], torch.full_like(t, -1), page * P + pos % P)
    status = torch.where(long, 2, refused.long())
    i = lambda x: x.to(torch.int32)
    return table, pool, i(after), i(free - take.sum()), i(cu), i(slot), i(status)


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == "plan":
            return _plain_plan(s)
        if op == "write":
            return _plain_write(s)
        O, lse = _plain_prompt(s) if op == "prompt" else _plain_paged(s)
        return O.to(s["Q"].dtype), lse
    import paper_2602_01801_amd as fa
    case = s["case"]
    if op == "prompt":
        return fa.prompt_attn_fwd(s["Q"], s["K"], s["V"], s["cu_q"], s["cu_k"], causal=case["causal"], scale=s["scale"], out=s["out"])
    if op == "paged":
        return fa.paged_attn_fwd(s["Q"], s["cu_q"], s["len"], s["table"], s["handle"], causal=case["causal"], scale=s["scale"],
                                 out=s["out"], ws=s["ws"])
    if op == "write":
        fa.kv_pages_write(s["handle"], s["slot"], s["K"], s["V"])
        K8, ks, V8, vs = s["pages"]
        return K8.view(torch.float8_e4m3fn), ks, V8.view(torch.float8_e4m3fn), vs
    after, free, cu, slot, status = fa.kv_pages_plan(s["n_new"], s["len"], s["table"], s["pool"], s["pool_n"], case["P"],
                                                     s["n_tok"], out=s["out"])
    return s["table"], s["pool"], after, free, cu, slot, status


# ---------------------------------------------------------------------------------------------------- in 64 bits

def _e4m3_values():
    """The 256 codes: sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7F and 0xFF are no numbers."""
    v = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v.append(math.nan if c & 127 == 127 else -x if c >> 7 else x)
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def _power(e):
    """2^e in float64, by its bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _round_e4m3(x):
    """float64 to the nearest value of the format, ties to even, beyond 448 the largest."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -30))).clamp(min=-6)
    step = _power(e - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _exact_attention(Q, K, V, causal, scale):
    """O, lse of one sequence from the definition, head by head; a query's weights are e^(l - lse)."""
    Hq, a, d = Q.shape
    Hkv, b, _ = K.shape
    O, lse = Q.new_zeros((Hq, a, d)), Q.new_full((Hq, a), -math.inf)
    step = max(1, (1 << 27) // max(b, 1))
    for h in range(Hq):
        k, v = K[h // (Hq // Hkv)], V[h // (Hq // Hkv)]
        for r in range(0, a if b else 0, step):
            e = min(a, r + step)
            last = b if not causal else min(b, b - a + e)
            if last <= 0:
                continue
            l = torch.matmul(Q[h, r:e] * scale, k[:last].t())
            if causal:
                seen = torch.arange(last, device=Q.device)[None] <= (torch.arange(r, e, device=Q.device) + b - a)[:, None]
                l = torch.where(seen, l, torch.full_like(l, -math.inf))
            z = torch.logsumexp(l, 1)
            w = torch.exp(l - torch.where(z == -math.inf, torch.zeros_like(z), z)[:, None])
            O[h, r:e], lse[h, r:e] = torch.matmul(w, v[:last]), z
    return O, lse


def exact(case, seed):
    if case["op"] == "plan":
        return None
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "write":
        values, P = _e4m3_values(), case["P"]
        K8, ks, V8, vs = s["pages"]
        out = []
        runs, slot = {}, s["slot"].tolist()
        for t, x in enumerate(slot):
            runs.setdefault(x // P, []).append(t)
        ids = torch.tensor(list(runs), device="cuda")
        begun = torch.tensor([any(slot[t] % P == 0 for t in r) for r in runs.values()], device="cuda")
        which = torch.tensor([i for i, r in enumerate(runs.values()) for _ in r], device="cuda")
        rows = torch.tensor([t for r in runs.values() for t in r], device="cuda")
        for x, code, scale, tr in ((s["K"], K8, ks, False), (s["V"], V8, vs, True)):
            x = x.to(f64).permute(1, 0, 2)[rows]
            top = torch.zeros((len(runs), x.shape[1]), dtype=f64, device="cuda").index_reduce_(0, which, x.abs().amax(2), "amax")
            power = torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -130)))
            power = torch.where(_power(power - 1) * 448 >= top, power - 1, power).clamp(min=-100)
            was = scale[ids].to(f64)
            now = torch.where(begun[:, None], _power(power), torch.maximum(was, _power(power)))
            val = values[code.long()]
            old = val[ids]
            shrunk = _round_e4m3(old * (was / now)[:, :, None, None, None, None])
            old = torch.where(begun.view(-1, 1, 1, 1, 1, 1), old, shrunk)
            fit = _round_e4m3(x / now[which][..., None])                    # [rows, H, d]
            fit = fit.view(fit.shape[0], fit.shape[1], -1, 16)
            off = torch.tensor(slot, device="cuda")[rows] % P
            if tr:
                old[which, :, off // 16, :, :, off % 16] = fit
            else:
                old[which, :, off // 16, :, off % 16, :] = fit
            val[ids] = old
            sc = scale.to(f64)
            sc[ids] = now
            out += [val, sc]
        return out
    Q = s["Q"].to(f64)
    O, lse = torch.empty_like(Q), torch.empty(Q.shape[:2], dtype=f64, device="cuda")
    values = _e4m3_values()
    a0 = k0 = 0
    for b, (a, n) in enumerate(zip(s["q"], s["k"])):
        if case["op"] == "prompt":
            K, V = (x[:, k0:k0 + n].to(f64) for x in (s["K"], s["V"]))
        else:
            K8, ks, V8, vs = s["pages"]
            ids = s["table"][b, : (n + case["P"] - 1) // case["P"]].long()
            K, V = _decode(K8, ks, ids, n, False, f64, values), _decode(V8, vs, ids, n, True, f64, values)
        O[:, a0:a0 + a], lse[:, a0:a0 + a] = _exact_attention(Q[:, a0:a0 + a], K, V, case["causal"], s["scale"])
        a0, k0 = a0 + a, k0 + n
    return O, lse
