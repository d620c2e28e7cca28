// Pages that requests share: forking (kv_pages_fork), giving pages up (kv_pages_free) and thinning out (kv_pages_compact).
#include <algorithm>

#include "packed.hpp"

namespace fastar {

int pages_check(const fastar_pages *pg);

namespace share {

__device__ __forceinline__ int clipped(int x, int hi) { return min(max(x, 0), hi); }

// Inclusive prefix sum over a workgroup of NT threads; the total in *all.
template <int NT>
__device__ __forceinline__ int wg_incl_scan(int v, int *part, int *all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v = (int)wave_incl_scan((unsigned)v);
    __syncthreads();   // the last call's partial sums have been read
    if (lane == 63) part[wave] = v;
    __syncthreads();
    int base = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const int x = part[w];
        if (w < wave) base += x;
        sum += x;
    }
    *all = sum;
    return v + base;
}

// ---- forking ----------------------------------------------------------------------------------------------------

constexpr int FORKS = 1024;        // of a call
constexpr int FT = 256;            // threads
constexpr int SLOTS = 2 * FORKS;   // of the table of children: half of them stay empty, so that a search ends
constexpr int COPY = 4;            // 16-byte pieces per thread of a page's copy

struct ForkArgs {
    fastar_pages pg;
    const int32_t *parent, *child, *keep, *len, *pool, *pool_n;
    int32_t *table, *len_out, *pool_n_out, *status;
    int32_t n, B, max_pages, pshift, parts;   // parts: workgroups per fork
};

// Every workgroup works the whole call out for itself: which forks are refused, and which pages the others take.  Then the first one
// of a fork writes its table row, the others a part each of its last page's copy, and the first of all lengths and counts,
// or, where those are written in place, a workgroup of a second launch (FINISH), so that nobody reads them changed.
template <bool FINISH>
__global__ __launch_bounds__(FT) void fork_kernel(ForkArgs a, bool finish_here) {
    __shared__ int part[FT / 64];
    __shared__ int s_child[SLOTS], s_first[SLOTS], s_m[FORKS], s_upto[FORKS];   // s_m: tokens, or -1 - status
    const int tid = threadIdx.x, P = 1 << a.pshift;
    const int f = FINISH ? 0 : blockIdx.x / a.parts, mine = FINISH ? 0 : blockIdx.x % a.parts;
    const long long cap = (long long)a.max_pages << a.pshift;
    const int n_pages = a.pg.n_pages, free0 = clipped(a.pool_n[0], n_pages);
    for (int i = tid; i < SLOTS; i += FT) s_child[i] = -1, s_first[i] = FORKS;
    __syncthreads();
    auto slot_of = [&](int c) { return (unsigned)c * 2654435761u >> 21; };   // 2^11 slots
    auto find = [&](int c) {   // the first fork that names child c, or FORKS
        unsigned s = slot_of(c);
        while (s_child[s] != -1 && s_child[s] != c) s = (s + 1) % SLOTS;
        return s_child[s] == c ? s_first[s] : FORKS;
    };
    for (int i = tid; i < a.n; i += FT) {
        const int c = a.child[i];
        if ((unsigned)c >= (unsigned)a.B) continue;
        unsigned s = slot_of(c);
        for (;; s = (s + 1) % SLOTS) {   // at most FORKS children in twice as many slots
            const int was = atomicCAS(&s_child[s], -1, c);
            if (was == -1 || was == c) break;
        }
        atomicMin(&s_first[s], i);
    }
    __syncthreads();
    int asked = 0;
    for (int i0 = 0; i0 < a.n; i0 += FT) {
        const int i = i0 + tid;
        int m = -3, need = 0;
        if (i < a.n) {
            const int p = a.parent[i], c = a.child[i];
            if ((unsigned)p < (unsigned)a.B && (unsigned)c < (unsigned)a.B && a.len[c] <= 0 && find(c) == i) {
                const int L = (int)min((long long)max(a.len[p], 0), cap);
                m = a.keep ? clipped(a.keep[i], L) : L;
                if (m & (P - 1)) need = (unsigned)a.table[(size_t)p * a.max_pages + (m >> a.pshift)] < (unsigned)n_pages;
            }
        }
        int all;
        const int upto = asked + wg_incl_scan<FT>(need, part, &all);
        if (i < a.n) {
            s_m[i] = need && upto > free0 ? -2 : m;
            s_upto[i] = need ? upto : 0;
        }
        asked += all;
    }
    __syncthreads();
    if (finish_here && (FINISH || blockIdx.x == 0)) {
        for (int b = tid; b < a.B; b += FT) {
            const int i = find(b);
            a.len_out[b] = i < FORKS && s_m[i] >= 0 ? s_m[i] : a.len[b];
        }
        if (tid == 0) a.pool_n_out[0] = free0 - min(asked, free0);   // those that were given a page come first among those that ask
    }
    if (FINISH) return;
    const int m = s_m[f], nth = s_upto[f];
    if (mine == 0 && tid == 0) a.status[f] = m < 0 ? -1 - m : 0;
    if (m < 0) return;
    const int p = a.parent[f], c = a.child[f], full = m >> a.pshift;
    const int32_t *from = a.table + (size_t)p * a.max_pages;
    int32_t *row = a.table + (size_t)c * a.max_pages;
    const int page = nth ? a.pool[free0 - nth] : -1;
    if (mine == 0) {
        for (int j = tid; j < full; j += FT) row[j] = from[j];
        if (tid == 0 && (m & (P - 1))) row[full] = nth ? page : from[full];
        return;
    }
    if (!nth || (unsigned)page >= (unsigned)n_pages) return;
    const int src = from[full];
    const size_t page_units = (size_t)a.pg.Hkv * P * a.pg.d / 16;   // 16-byte pieces of a page of K8 or V8
    const size_t u0 = (size_t)(mine - 1) * (FT * COPY) + tid;
    auto at = [&](uint8_t *x, int pg, size_t u) { return (u32x4 *)x + (size_t)pg * page_units + u; };
    u32x4 w[COPY];
#pragma unroll
    for (int i = 0; i < COPY; ++i) {
        const size_t u = u0 + i * FT;
        if (u < 2 * page_units) w[i] = u < page_units ? *at(a.pg.K8, src, u) : *at(a.pg.V8, src, u - page_units);
    }
#pragma unroll
    for (int i = 0; i < COPY; ++i) {
        const size_t u = u0 + i * FT;
        if (u < 2 * page_units) *(u < page_units ? at(a.pg.K8, page, u) : at(a.pg.V8, page, u - page_units)) = w[i];
    }
    if (mine == 1)
        for (int h = tid; h < a.pg.Hkv; h += FT) {
            a.pg.kscale[(size_t)page * a.pg.Hkv + h] = a.pg.kscale[(size_t)src * a.pg.Hkv + h];
            a.pg.vscale[(size_t)page * a.pg.Hkv + h] = a.pg.vscale[(size_t)src * a.pg.Hkv + h];
        }
}

// ---- giving pages up --------------------------------------------------------------------------------------------

// Table entries are looked at in blocks of ET, each within a request's row: entry e of request b has number b * max_pages + e.
constexpr int ET = 1024;

// What a call needs in memory between its launches, cut out of the workspace.
struct Work {
    int32_t *hold, *gone, *last;             // [n_pages] holders before the call; those that give the page up; the last of them
    int32_t *have, *stay, *need, *base;      // [B] pages and tokens before and after, fresh pages needed and where they begin (-1: refused)
    int32_t *head;                           // [4] free pages before, fresh pages in all
    int32_t *block;                          // pages that a block gives back, then those before it
    int32_t *old, *link, *from;              // [B, max_pages] table before the call; new page of an old one; old page of a new one, or ~(which fresh one)
    int32_t *made, *page;                    // [n_pages] fresh pages: entry of the new table, number
    int32_t *token;                          // [B, max_pages * P] old place of the request's new tokens
};
inline size_t rounded(size_t n) { return (n + 63) / 64 * 64; }   // 256 bytes
inline size_t lay_out(Work &w, int32_t *p, int64_t B, int64_t max_pages, int64_t n_pages, int64_t P) {
    size_t at = 0;
    auto take = [&](int32_t *&x, size_t n) {
        x = p ? p + at : nullptr;
        at += rounded(n);
    };
    take(w.head, 4);
    take(w.hold, n_pages);
    take(w.gone, n_pages);
    take(w.last, n_pages);
    take(w.have, B);
    take(w.stay, B);
    take(w.need, B);
    take(w.base, B);
    take(w.block, B * ((max_pages + ET - 1) / ET) + 1);
    take(w.old, B * max_pages);
    take(w.link, B * max_pages);
    take(w.from, B * max_pages);
    take(w.made, n_pages);
    take(w.page, n_pages);
    take(w.token, (size_t)(B * max_pages) * P);
    return at * sizeof(int32_t);
}

struct Args {
    fastar_pages pg;   // compaction only
    const uint8_t *mask;
    const int32_t *keep, *len, *table, *pool, *pool_n;
    int32_t *len_out, *table_out, *pool_out, *pool_n_out, *status;
    int32_t B, max_pages, n_pages, pshift, segs;   // segs: blocks of entries per row
    Work w;
};

__global__ __launch_bounds__(256) void clear_kernel(Work w, int n_pages) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n_pages) return;
    w.hold[i] = 0;
    w.gone[i] = 0;
    w.last[i] = -1;
}

// A block of entries: request, first entry.
__device__ __forceinline__ void block_of(const Args &a, int &b, int &e0) {
    b = blockIdx.x / a.segs;
    e0 = blockIdx.x % a.segs * ET;
}
__device__ __forceinline__ int tokens_of(const Args &a, int b) {
    return (int)min((long long)max(a.len[b], 0), (long long)a.max_pages << a.pshift);
}

__global__ __launch_bounds__(256) void hold_kernel(Args a) {
    int b, e0;
    block_of(a, b, e0);
    const int have = (tokens_of(a, b) + (1 << a.pshift) - 1) >> a.pshift;
    const int32_t *row = a.table + (size_t)b * a.max_pages;
    for (int e = e0 + threadIdx.x; e < min(e0 + ET, have); e += 256) {
        const int p = row[e];
        if ((unsigned)p < (unsigned)a.n_pages) atomicAdd(&a.w.hold[p], 1);
    }
}

__device__ __forceinline__ void give_up(const Args &a, int p, int number) {
    atomicAdd(&a.w.gone[p], 1);
    atomicMax(&a.w.last[p], number);
}
// Which requests are refused, and the pages that the others give up.
__global__ __launch_bounds__(256) void cut_kernel(Args a) {
    int b, e0;
    block_of(a, b, e0);
    const int P = 1 << a.pshift, L = tokens_of(a, b), have = (L + P - 1) >> a.pshift;
    const int32_t *row = a.table + (size_t)b * a.max_pages;
    int stay = min(max(a.keep[b], 0), L);
    bool refused = false;
    if (stay < L && (stay & (P - 1))) {
        const int p = row[stay >> a.pshift];
        refused = (unsigned)p < (unsigned)a.n_pages && a.w.hold[p] > 1;
    }
    if (refused) stay = L;
    if (e0 == 0 && threadIdx.x == 0) {
        a.w.have[b] = have;
        a.w.stay[b] = stay;
        a.status[b] = refused;
        if (b == 0) a.w.head[0] = clipped(a.pool_n[0], a.n_pages);
    }
    const int left = (stay + P - 1) >> a.pshift;
    for (int e = max(e0, left / 256 * 256) + threadIdx.x; e < min(e0 + ET, have); e += 256) {
        if (e < left) continue;
        const int p = row[e];
        if ((unsigned)p < (unsigned)a.n_pages) give_up(a, p, b * a.max_pages + e);
    }
}

// The page of entry e, if the call gives it back to the pool there: all its holders give it up, and this is the last one.
template <bool COMPACT>
__device__ __forceinline__ int given_back(const Args &a, int b, int e, int left, int have) {
    if (e < left || e >= have) return -1;
    const size_t at = (size_t)b * a.max_pages + e;
    const int p = COMPACT ? a.w.old[at] : a.table[at];
    if ((unsigned)p >= (unsigned)a.n_pages || (COMPACT && a.w.link[at] >= 0)) return -1;
    return a.w.gone[p] == a.w.hold[p] && a.w.last[p] == (int)at ? p : -1;
}
template <bool COMPACT>
__device__ __forceinline__ int first_given(const Args &a, int b, int have) {
    if (COMPACT) return a.w.base[b] < 0 ? have : 0;   // refused requests give nothing up
    return (a.w.stay[b] + (1 << a.pshift) - 1) >> a.pshift;
}
// PUSH false: how many pages every block gives back;  true: they go to the pool.
template <bool COMPACT, bool PUSH>
__global__ __launch_bounds__(256) void give_kernel(Args a) {
    __shared__ int part[4];
    int b, e0;
    block_of(a, b, e0);
    const int have = a.w.have[b], left = first_given<COMPACT>(a, b, have);
    int p[ET / 256], n = 0;
#pragma unroll
    for (int i = 0; i < ET / 256; ++i) {
        p[i] = given_back<COMPACT>(a, b, e0 + (ET / 256) * (int)threadIdx.x + i, left, have);
        n += p[i] >= 0;
    }
    int all;
    const int upto = wg_incl_scan<256>(n, part, &all);
    if constexpr (!PUSH) {
        if (threadIdx.x == 0) a.w.block[blockIdx.x] = all;
    } else {
        const int top = a.w.head[0] - (COMPACT ? a.w.head[1] : 0);
        long long at = (long long)top + a.w.block[blockIdx.x] + upto - n;
#pragma unroll
        for (int i = 0; i < ET / 256; ++i)
            if (p[i] >= 0) {
                if (at < a.n_pages) a.pool_out[at] = p[i];
                ++at;
            }
        if (threadIdx.x == 0) {
            if (e0 == 0) a.len_out[b] = a.w.stay[b];
            if (blockIdx.x == 0) a.pool_n_out[0] = (int)min((long long)top + a.w.block[(size_t)a.B * a.segs], (long long)a.n_pages);
        }
    }
}
// Exclusive prefix sums of n numbers, and their sum behind them.
__global__ __launch_bounds__(1024) void scan_kernel(int32_t *x, int n) {
    __shared__ int part[16];
    int sum = 0;
    for (int i0 = 0; i0 < n; i0 += 1024) {
        const int i = i0 + threadIdx.x, v = i < n ? x[i] : 0;
        int all;
        const int upto = wg_incl_scan<1024>(v, part, &all);
        if (i < n) x[i] = sum + upto - v;
        sum += all;
    }
    if (threadIdx.x == 0) x[n] = sum;
}

// Of no requests: the free pages as they are.
__global__ __launch_bounds__(256) void nothing_kernel(Args a) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (a.pool_out != a.pool && i < (size_t)a.n_pages) a.pool_out[i] = a.pool[i];
    if (i == 0) a.pool_n_out[0] = clipped(a.pool_n[0], a.n_pages);
}

// ---- thinning out -----------------------------------------------------------------------------------------------

// A workgroup per request goes through its mask: where every token goes, which pages stay whole, which of the new ones are fresh.
// It keeps the old table row, as the new one may be written over it.
__global__ __launch_bounds__(1024) void mask_kernel(Args a) {
    __shared__ int part[16];
    const int b = blockIdx.x, tid = threadIdx.x, P = 1 << a.pshift;
    const int L = tokens_of(a, b), have = (L + P - 1) >> a.pshift;
    const size_t row = (size_t)b * a.max_pages;
    int32_t *token = a.w.token + (row << a.pshift);
    const u32x4 *mask = (const u32x4 *)(a.mask + (row << a.pshift));
    for (int e = tid; e < have; e += 1024) {
        const int p = a.table[row + e];
        a.w.old[row + e] = p;
        a.w.link[row + e] = -1;
        a.w.from[row + e] = -1;
        if ((unsigned)p < (unsigned)a.n_pages) atomicAdd(&a.w.hold[p], 1);
    }
    __syncthreads();
    const int per = P / 16;   // threads that look at a page: 1, 2 or 4 neighbours
    int kept = 0;
    for (int i0 = 0; i0 * 16 < L; i0 += 1024) {
        const int u = i0 + tid, t0 = 16 * u;   // 16 tokens of one page
        unsigned bits = 0, there = 0;
        if (t0 < L) {
            const u32x4 x = mask[u];
            there = t0 + 16 <= L ? 0xFFFFu : (1u << (L - t0)) - 1u;
            if ((unsigned)a.w.old[row + (t0 >> a.pshift)] < (unsigned)a.n_pages)
#pragma unroll
                for (int i = 0; i < 16; ++i) bits |= (x[i / 4] >> (8 * (i % 4)) & 0xFFu) ? 1u << i : 0u;
            bits &= there;
        }
        const int n = __builtin_popcount(bits);
        int all;
        const int rank = kept + wg_incl_scan<1024>(n, part, &all) - n;
        int at = rank;
        for (unsigned m = bits; m; m &= m - 1) token[at++] = t0 + __builtin_ctz(m);
        // the whole of a page, at a page's beginning, and to its end unless the request ends there too
        unsigned lost = bits != there;
        if (per >= 2) lost |= (unsigned)__shfl_xor((int)lost, 1, 64);
        if (per >= 4) lost |= (unsigned)__shfl_xor((int)lost, 2, 64);
        if (t0 < L && !lost && !(u & (per - 1)) && !(rank & (P - 1))) {
            const int s = t0 >> a.pshift, j = rank >> a.pshift;
            a.w.link[row + s] = j;
            a.w.from[row + j] = s;
        }
        kept += all;
    }
    __syncthreads();
    const int pages = (kept + P - 1) >> a.pshift;
    int fresh = 0;
    for (int j0 = 0; j0 < pages; j0 += 1024) {
        const int j = j0 + tid, n = j < pages && a.w.from[row + j] < 0;
        int all;
        const int upto = wg_incl_scan<1024>(n, part, &all);
        if (n) a.w.from[row + j] = ~(fresh + upto - 1);
        fresh += all;
    }
    if (tid == 0) {
        a.w.have[b] = have;
        a.w.stay[b] = kept;
        a.w.need[b] = fresh;
    }
}

// Which requests are refused, and where the fresh pages of the others begin.
__global__ __launch_bounds__(1024) void admit_kernel(Args a) {
    __shared__ int part[16];
    __shared__ int s_taken;
    const int free0 = clipped(a.pool_n[0], a.n_pages);
    if (threadIdx.x == 0) s_taken = 0;
    long long asked = 0;   // need is at most max_pages, and B * max_pages below 2^31
    for (int b0 = 0; b0 < a.B; b0 += 1024) {
        const int b = b0 + threadIdx.x, need = b < a.B ? a.w.need[b] : 0;
        int all;
        const long long upto = asked + wg_incl_scan<1024>(need, part, &all);
        if (b < a.B) {
            const bool refused = need > 0 && upto > free0;
            a.w.base[b] = refused ? -1 : (int)min(upto - need, (long long)free0);
            a.status[b] = refused;
            if (refused) a.w.stay[b] = tokens_of(a, b);
            if (!refused && need > 0) atomicMax(&s_taken, (int)upto);
        }
        asked += all;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        a.w.head[0] = free0;
        a.w.head[1] = s_taken;
    }
}

// New table rows, the list of fresh pages, the old pages that are given up, and the pool as it was.
__global__ __launch_bounds__(256) void relink_kernel(Args a) {
    int b, e0;
    block_of(a, b, e0);
    const int base = a.w.base[b], have = a.w.have[b], stay = a.w.stay[b], free0 = a.w.head[0];
    const int pages = (stay + (1 << a.pshift) - 1) >> a.pshift;
    const size_t row = (size_t)b * a.max_pages;
    for (int e = e0 + threadIdx.x; e < min(e0 + ET, a.max_pages); e += 256) {
        if (base < 0) {
            if (a.table_out != a.table) a.table_out[row + e] = a.table[row + e];
            continue;
        }
        int p = -1;
        if (e < pages) {
            const int f = a.w.from[row + e];
            if (f >= 0) p = a.w.old[row + f];
            else {
                const int k = base + ~f;
                p = a.pool[free0 - 1 - k];
                a.w.made[k] = (int)(row + e);
                a.w.page[k] = p;
            }
        }
        a.table_out[row + e] = p;
        if (e < have && a.w.link[row + e] < 0) {
            const int q = a.w.old[row + e];
            if ((unsigned)q < (unsigned)a.n_pages) give_up(a, q, (int)(row + e));
        }
    }
    if (a.pool_out != a.pool)
        for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)a.n_pages; i += (size_t)gridDim.x * 256) a.pool_out[i] = a.pool[i];
}

__device__ __forceinline__ float largest(float a, float b) { return a > b ? a : b; }
// Codes carried over to a scale 1 / ratio times as large; NaN stays.
__device__ __forceinline__ unsigned carried(unsigned w, float ratio) {
    int y = 0;
    y = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * ratio, y, false);
    y = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8((int)w, 2) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * ratio, y, true);
    return (unsigned)y;
}

// A workgroup takes one head of a fresh page after the other: its tokens' places, then the 16 bytes of a token (K) or of a
// coordinate (V) per thread.
__global__ __launch_bounds__(256) void gather_kernel(Args a) {
    __shared__ int s_src[64], s_off[64];
    __shared__ float s_ratio[2][64];
    const int tid = threadIdx.x, P = 1 << a.pshift, d = a.pg.d, Hkv = a.pg.Hkv;
    const long long items = (long long)a.w.head[1] * Hkv;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int k = (int)(it / Hkv), h = (int)(it % Hkv), entry = a.w.made[k], dst = a.w.page[k];
        if ((unsigned)dst >= (unsigned)a.n_pages) continue;   // the caller's pool names no page: nothing is written
        const int b = entry / a.max_pages, j = entry % a.max_pages;
        const int n = min(P, a.w.stay[b] - j * P);
        __syncthreads();
        if (tid < 64) {
            float ks = 0.0f, vs = 0.0f;
            int src = 0, off = 0;
            if (tid < n) {
                const int t = a.w.token[(((size_t)b * a.max_pages + j) << a.pshift) + tid];
                src = a.w.old[(size_t)b * a.max_pages + (t >> a.pshift)];
                off = t & (P - 1);
                ks = a.pg.kscale[(size_t)src * Hkv + h];
                vs = a.pg.vscale[(size_t)src * Hkv + h];
            }
            float km = ks, vm = vs;
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                km = largest(km, shfl_xor(km, o));
                vm = largest(vm, shfl_xor(vm, o));
            }
            s_src[tid] = src;
            s_off[tid] = off;
            s_ratio[0][tid] = ks / km;
            s_ratio[1][tid] = vs / vm;
            if (tid == 0) {
                a.pg.kscale[(size_t)dst * Hkv + h] = km;
                a.pg.vscale[(size_t)dst * Hkv + h] = vm;
            }
        }
        __syncthreads();
        const size_t head = (size_t)P * d;
        auto at = [&](uint8_t *x, int page) { return x + ((size_t)page * Hkv + h) * head; };
        for (int u = tid; u < P * d / 16; u += 256) {   // K: cell (tb, db), token o of it
            const int tb = u / d, db = u / 16 % (d / 16), t = tb * 16 + u % 16;
            u32x4 y = {0, 0, 0, 0};
            if (t < n) {
                const int off = s_off[t];
                const float ratio = s_ratio[0][t];
                y = *(const u32x4 *)(at(a.pg.K8, s_src[t]) + ((off >> 4) * (d / 16) + db) * 256 + (off & 15) * 16);
                if (ratio != 1.0f)
#pragma unroll
                    for (int q = 0; q < 4; ++q) y[q] = carried(y[q], ratio);
            }
            ((u32x4 *)at(a.pg.K8, dst))[u] = y;
        }
        for (int u = tid; u < P * d / 16; u += 256) {   // V: cell (tb, db), coordinate c of it
            const int tb = u / d, db = u / 16 % (d / 16), c = u % 16;
            u32x4 y;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                unsigned w = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = tb * 16 + 4 * q + i;
                    if (t >= n) continue;
                    const int off = s_off[t];
                    const float ratio = s_ratio[1][t];
                    unsigned x = at(a.pg.V8, s_src[t])[((off >> 4) * (d / 16) + db) * 256 + c * 16 + (off & 15)];
                    if (ratio != 1.0f) x = carried(x, ratio) & 0xFFu;
                    w |= x << (8 * i);
                }
                y[q] = w;
            }
            ((u32x4 *)at(a.pg.V8, dst))[u] = y;
        }
    }
}

}  // namespace share

size_t pages_ws_bytes(int B, int max_pages, int n_pages, int P) {
    if (B < 0 || max_pages <= 0 || n_pages <= 0 || !page_size_ok(P)) return 0;
    share::Work w;
    return share::lay_out(w, nullptr, B, max_pages, n_pages, P);
}

// What kv_pages_free and kv_pages_compact ask of their arguments alike.
static int share_check(const int32_t *len, const int32_t *table, int B, int max_pages, const int32_t *pool, const int32_t *pool_n, int n_pages,
                       int P, const int32_t *len_out, const int32_t *pool_n_out, const int32_t *status, const void *ws, size_t ws_bytes) {
    if (B < 0 || max_pages <= 0 || n_pages <= 0) return FASTAR_ERR_INVALID_ARG;
    if (!pool || !pool_n || !pool_n_out) return FASTAR_ERR_INVALID_ARG;
    if (B > 0 && (!len || !table || !len_out || !status)) return FASTAR_ERR_INVALID_ARG;
    if (!page_size_ok(P)) return FASTAR_ERR_UNSUPPORTED;
    if ((int64_t)max_pages * P > INT32_MAX || (int64_t)n_pages * P > INT32_MAX || (int64_t)B * max_pages > INT32_MAX) return FASTAR_ERR_UNSUPPORTED;
    if (!launch_ok((int64_t)B * ((max_pages + share::ET - 1) / share::ET), 1024)) return FASTAR_ERR_UNSUPPORTED;
    if (!ws || ((uintptr_t)ws & 255)) return FASTAR_ERR_INVALID_ARG;
    if (ws_bytes < pages_ws_bytes(B, max_pages, n_pages, P)) return FASTAR_ERR_WORKSPACE;
    return FASTAR_OK;
}
static share::Args share_args(const int32_t *len, const int32_t *table, int B, int max_pages, const int32_t *pool, const int32_t *pool_n,
                              int n_pages, int P, int32_t *len_out, int32_t *pool_out, int32_t *pool_n_out, int32_t *status, void *ws) {
    share::Args a{};
    a.len = len, a.table = table, a.pool = pool, a.pool_n = pool_n;
    a.len_out = len_out, a.pool_out = pool_out, a.pool_n_out = pool_n_out, a.status = status;
    a.B = B, a.max_pages = max_pages, a.n_pages = n_pages, a.pshift = __builtin_ctz((unsigned)P);
    a.segs = (max_pages + share::ET - 1) / share::ET;
    share::lay_out(a.w, (int32_t *)ws, B, max_pages, n_pages, P);
    return a;
}
static int nothing(const share::Args &a, hipStream_t s) {
    hipLaunchKernelGGL(share::nothing_kernel, dim3((unsigned)((a.n_pages + 255) / 256)), dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}
// Pages given back by the blocks of entries: counted, summed up, pushed.
template <bool COMPACT>
static int give_back(const share::Args &a, hipStream_t s) {
    const dim3 grid((unsigned)(a.B * a.segs));
    hipLaunchKernelGGL((share::give_kernel<COMPACT, false>), grid, dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(share::scan_kernel, dim3(1), dim3(1024), 0, s, a.w.block, a.B * a.segs);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL((share::give_kernel<COMPACT, true>), grid, dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}

}  // namespace fastar

extern "C" int kv_pages_fork(const fastar_pages *pages, const int32_t *parent, const int32_t *child, const int32_t *keep, int n,
                             const int32_t *len, int32_t *table, int B, int max_pages, const int32_t *pool, const int32_t *pool_n,
                             int32_t *len_out, int32_t *pool_n_out, int32_t *status, void *stream) {
    using namespace fastar;
    if (const int rc = pages_check(pages); rc != FASTAR_OK) return rc;
    if (n < 0 || B < 0 || max_pages <= 0) return FASTAR_ERR_INVALID_ARG;
    if (!pool || !pool_n || !pool_n_out) return FASTAR_ERR_INVALID_ARG;
    if (B > 0 && (!len || !table || !len_out)) return FASTAR_ERR_INVALID_ARG;
    if (n > 0 && (!parent || !child || !status)) return FASTAR_ERR_INVALID_ARG;
    if ((int64_t)max_pages * pages->P > INT32_MAX || (int64_t)B * max_pages > INT32_MAX || n > share::FORKS) return FASTAR_ERR_UNSUPPORTED;
    share::ForkArgs a{};
    a.pg = *pages;
    a.parent = parent, a.child = child, a.keep = keep, a.len = len, a.pool = pool, a.pool_n = pool_n;
    a.table = table, a.len_out = len_out, a.pool_n_out = pool_n_out, a.status = status;
    a.n = n, a.B = B, a.max_pages = max_pages, a.pshift = __builtin_ctz((unsigned)pages->P);
    const int64_t units = 2 * (int64_t)pages->Hkv * pages->P * pages->d / 16, per = share::FT * share::COPY;
    a.parts = (int)(1 + (units + per - 1) / per);
    if (!launch_ok((int64_t)n * a.parts, share::FT)) return FASTAR_ERR_UNSUPPORTED;
    const hipStream_t s = (hipStream_t)stream;
    const bool in_place = len_out == len || pool_n_out == pool_n;
    if (n > 0) {
        hipLaunchKernelGGL(share::fork_kernel<false>, dim3((unsigned)(n * a.parts)), dim3(share::FT), 0, s, a, !in_place);
        FASTAR_LAUNCH_CHECK();
    }
    if (in_place || n == 0) {
        hipLaunchKernelGGL(share::fork_kernel<true>, dim3(1), dim3(share::FT), 0, s, a, true);
        FASTAR_LAUNCH_CHECK();
    }
    return FASTAR_OK;
}

extern "C" int kv_pages_free(const int32_t *keep, const int32_t *len, const int32_t *table, int B, int max_pages, int32_t *pool,
                             const int32_t *pool_n, int n_pages, int P, int32_t *len_out, int32_t *pool_n_out, int32_t *status, void *ws,
                             size_t ws_bytes, void *stream) {
    using namespace fastar;
    if (const int rc = share_check(len, table, B, max_pages, pool, pool_n, n_pages, P, len_out, pool_n_out, status, ws, ws_bytes); rc != FASTAR_OK) return rc;
    if (B > 0 && !keep) return FASTAR_ERR_INVALID_ARG;
    share::Args a = share_args(len, table, B, max_pages, pool, pool_n, n_pages, P, len_out, pool, pool_n_out, status, ws);
    if (B == 0) return nothing(a, (hipStream_t)stream);
    a.keep = keep;
    const hipStream_t s = (hipStream_t)stream;
    const dim3 grid((unsigned)(B * a.segs));
    hipLaunchKernelGGL(share::clear_kernel, dim3((unsigned)((n_pages + 255) / 256)), dim3(256), 0, s, a.w, n_pages);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(share::hold_kernel, grid, dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(share::cut_kernel, grid, dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    return give_back<false>(a, s);
}

extern "C" int kv_pages_compact(const fastar_pages *pages, const uint8_t *keep, const int32_t *len, const int32_t *table, int B, int max_pages,
                                const int32_t *pool, const int32_t *pool_n, int32_t *len_out, int32_t *table_out, int32_t *pool_out,
                                int32_t *pool_n_out, int32_t *status, void *ws, size_t ws_bytes, void *stream) {
    using namespace fastar;
    if (const int rc = pages_check(pages); rc != FASTAR_OK) return rc;
    if (const int rc = share_check(len, table, B, max_pages, pool, pool_n, pages->n_pages, pages->P, len_out, pool_n_out, status, ws, ws_bytes);
        rc != FASTAR_OK)
        return rc;
    if (!pool_out || (B > 0 && (!keep || ((uintptr_t)keep & 15) || !table_out))) return FASTAR_ERR_INVALID_ARG;
    share::Args a = share_args(len, table, B, max_pages, pool, pool_n, pages->n_pages, pages->P, len_out, pool_out, pool_n_out, status, ws);
    if (B == 0) return nothing(a, (hipStream_t)stream);
    a.pg = *pages;
    a.mask = keep;
    a.table_out = table_out;
    const hipStream_t s = (hipStream_t)stream;
    hipLaunchKernelGGL(share::clear_kernel, dim3((unsigned)((a.n_pages + 255) / 256)), dim3(256), 0, s, a.w, a.n_pages);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(share::mask_kernel, dim3((unsigned)B), dim3(1024), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(share::admit_kernel, dim3(1), dim3(1024), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(share::relink_kernel, dim3((unsigned)(B * a.segs)), dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(share::gather_kernel, dim3(2048), dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    return give_back<true>(a, s);
}
