// Pages that requests share: forking (kv_pages_fork), giving pages up (kv_pages_free) and thinning out (kv_pages_compact).
#include <algorithm>
#include <type_traits>

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
// or, where those are written in place, a workgroup of a second launch (FINISH), so that nobody reads them changed.  Bound by the trips to memory before the
// copies (forks -> lengths -> tables -> pool), which a launch of its own would only put in front of another one's: 4 forks 4.8 us, 128 forks with 33 MB of last pages
// 8.6 (3.8 TB/s).
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

// Who holds a page is counted from the tables, by atomics whose order does not show: holders (hold_kernel), who is refused and who gives up (cut_kernel), how many pages
// each block gives back (count_kernel), where they go (push_kernel).  Bound by trips to memory and by the launches: 192 requests on 8000 entries 2.4 + 2.8 + 3.5 + 3.7 + 4.8 us,
// 96 on 102000 3.0 + 5.8 + 7.0 + 4.0 + 5.8.
// Table entries are looked at in blocks of ET, each within a request's row: entry e of request b has number b * max_pages + e.
constexpr int ET = 256;

// A page in the call: its holders before it, those that give it up, and the last of them.  Together, so that an entry meets one line of memory.
struct PageState {
    int32_t hold, gone, last, unused;
};
// 16 tokens of a request in its mask: which are kept, and how many before them.
struct Group {
    int32_t rank;
    uint32_t bits;
};
// A fresh page: its number, its request and how many groups that has, the group of its first token, which of the request's new tokens that is,
// and how many it holds.
struct Fresh {
    int32_t page, b, groups, start, first, n, unused[2];
};
// What a call needs in memory between its launches, cut out of the workspace.
struct Work {
    PageState *state;                        // [n_pages]
    Group *group;                            // [B, max_pages * P / 16]
    int32_t *have, *stay, *need, *base;      // [B] pages and tokens before and after, fresh pages needed and where they begin (-1: refused)
    int32_t *head;                           // [4] free pages before, fresh pages in all
    int32_t *block;                          // pages that a block gives back
    int32_t *old, *link, *from, *start;      // [B, max_pages] table before the call; new page of an old one; old page of a new one, or ~(which fresh one), and the group of its first token
    Fresh *made;                             // [n_pages]
};
inline size_t lay_out(Work &w, char *p, int64_t B, int64_t max_pages, int64_t n_pages, int64_t P) {
    size_t at = 0;
    auto take = [&](auto *&x, size_t n) {
        using T = std::remove_reference_t<decltype(*x)>;
        x = p ? (T *)(p + at) : nullptr;
        at += (n * sizeof(T) + 255) / 256 * 256;
    };
    take(w.head, 4);
    take(w.state, n_pages);
    take(w.have, B);
    take(w.stay, B);
    take(w.need, B);
    take(w.base, B);
    take(w.block, B * ((max_pages + ET - 1) / ET) + 1);
    take(w.old, B * max_pages);
    take(w.link, B * max_pages);
    take(w.from, B * max_pages);
    take(w.start, B * max_pages);
    take(w.made, n_pages);
    take(w.group, (size_t)(B * max_pages) * P / 16);
    return at;
}

struct Args {
    fastar_pages pg;   // thinning out only
    const uint8_t *mask;
    const int32_t *keep, *len, *table, *pool, *pool_n;
    int32_t *len_out, *table_out, *pool_out, *pool_n_out, *status;
    int32_t B, max_pages, n_pages, pshift, segs;   // segs: blocks of entries per row
    bool one_pushes;                               // a workgroup pushes for all blocks
    bool copies;                                   // relink_kernel copies the pool
    bool summed, admitted;                         // block, and base and status, have been worked out by a launch of their own
    Work w;
};

__device__ __forceinline__ void clear_states(const Args &a) {
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < (size_t)a.n_pages; i += (size_t)gridDim.x * blockDim.x)
        *(i32x4 *)&a.w.state[i] = i32x4{0, 0, -1, 0};
}
__global__ __launch_bounds__(256) void clear_kernel(Args a) { clear_states(a); }

// A block of entries: request, and the thread's entry.
__device__ __forceinline__ void entry_of(const Args &a, int block, int &b, int &e) {
    b = block / a.segs;
    e = block % a.segs * ET + threadIdx.x;
}
__device__ __forceinline__ int tokens_of(const Args &a, int b) {
    return (int)min((long long)max(a.len[b], 0), (long long)a.max_pages << a.pshift);
}
__device__ __forceinline__ bool is_page(const Args &a, int p) { return (unsigned)p < (unsigned)a.n_pages; }

__global__ __launch_bounds__(ET) void hold_kernel(Args a) {
    int b, e;
    entry_of(a, blockIdx.x, b, e);
    if (e >= (tokens_of(a, b) + (1 << a.pshift) - 1) >> a.pshift) return;
    const int p = a.table[(size_t)b * a.max_pages + e];
    if (is_page(a, p)) atomicAdd(&a.w.state[p].hold, 1);
}

__device__ __forceinline__ void give_up(const Args &a, int p, int number) {
    atomicAdd(&a.w.state[p].gone, 1);
    atomicMax(&a.w.state[p].last, number);
}
// Which requests are refused, and the pages that the others give up.
__global__ __launch_bounds__(ET) void cut_kernel(Args a) {
    int b, e;
    entry_of(a, blockIdx.x, b, e);
    const int P = 1 << a.pshift, L = tokens_of(a, b), have = (L + P - 1) >> a.pshift;
    const int32_t *row = a.table + (size_t)b * a.max_pages;
    const int p = e < have ? row[e] : -1;
    int stay = clipped(a.keep[b], L);
    bool refused = false;
    if (stay < L && (stay & (P - 1))) {
        const int q = row[stay >> a.pshift];
        refused = is_page(a, q) && a.w.state[q].hold > 1;
    }
    if (refused) stay = L;
    if (e == 0) {
        a.w.have[b] = have;
        a.w.stay[b] = stay;
        a.status[b] = refused;
        if (b == 0) a.w.head[0] = clipped(a.pool_n[0], a.n_pages);
    }
    if (e >= (stay + P - 1) >> a.pshift && is_page(a, p)) give_up(a, p, b * a.max_pages + e);
}

// The page of entry e, if the call gives it back to the pool there: all its holders give it up, and this is the last one.
template <bool COMPACT>
__device__ __forceinline__ int given_back(const Args &a, int b, int e) {
    const int have = a.w.have[b];
    if (e >= have) return -1;
    if (COMPACT ? a.w.base[b] < 0 : e < (a.w.stay[b] + (1 << a.pshift) - 1) >> a.pshift) return -1;   // refused;  kept
    const size_t at = (size_t)b * a.max_pages + e;
    const int p = COMPACT ? a.w.old[at] : a.table[at];
    if (!is_page(a, p) || (COMPACT && a.w.link[at] >= 0)) return -1;
    const PageState s = a.w.state[p];
    return s.gone == s.hold && s.last == (int)at ? p : -1;
}
// How many pages a block gives back.
template <bool COMPACT>
__device__ __forceinline__ void count_block(const Args &a, int block) {
    __shared__ int n;
    int b, e;
    entry_of(a, block, b, e);
    if (threadIdx.x == 0) n = 0;
    __syncthreads();
    const int c = __builtin_popcountll(__ballot(given_back<COMPACT>(a, b, e) >= 0));
    if ((threadIdx.x & 63) == 0 && c) atomicAdd(&n, c);
    __syncthreads();
    if (threadIdx.x == 0) a.w.block[block] = n;
}
__global__ __launch_bounds__(ET) void count_kernel(Args a) { count_block<false>(a, blockIdx.x); }

// All of kv_pages_free by one workgroup, where no more than ONE_TABLE entries can be held and pages' states fit its LDS: entries of all requests in
// one sequence, ONE_ENTRIES per thread, whose pages stay in registers from one round of atomics to the next.  Three trips to memory instead of
// five launches: 50 / 640 / 7872 entries 5.0 / 7.7 / 12.6 us, and 8.7 / 10.7 / 11.9 by launches that follow one another at once; a program that
// launches each by itself waits 20 us for five.  (In more rounds, 15360 entries 43 us and 12.)
constexpr int ONE = 1024, ONE_ENTRIES = 8, ONE_TABLE = ONE * ONE_ENTRIES, ONE_PAGES = 16384;   // threads, also requests; pages: 128 KB
__global__ __launch_bounds__(ONE) void free_one_kernel(Args a) {
    extern __shared__ int s_left[];          // holders, less those that give the page up
    int *s_last = s_left + a.n_pages;        // the last of the latter
    __shared__ int part[ONE / 64], s_have[ONE], s_stay[ONE];   // s_have: inclusive sums of the requests' pages
    const int tid = threadIdx.x, P = 1 << a.pshift, free0 = clipped(a.pool_n[0], a.n_pages);
    int L = 0, stay = 0;
    if (tid < a.B) {
        L = tokens_of(a, tid);
        stay = clipped(a.keep[tid], L);
    }
    const int have = (L + P - 1) >> a.pshift;
    const int cut = stay < L && (stay & (P - 1)) ? a.table[(size_t)tid * a.max_pages + (stay >> a.pshift)] : -1;
    for (int i = tid; i < a.n_pages; i += ONE) s_left[i] = 0, s_last[i] = -1;
    int total;
    s_have[tid] = wg_incl_scan<ONE>(have, part, &total);
    __syncthreads();
    int page[ONE_ENTRIES], who[ONE_ENTRIES], at[ONE_ENTRIES];   // neighbours in the sequence, so that sums over threads go by it
#pragma unroll
    for (int i = 0; i < ONE_ENTRIES; ++i) {
        const int x = tid * ONE_ENTRIES + i;
        page[i] = -1;
        if (x >= total) continue;
        int lo = 0, hi = a.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (s_have[mid] > x) hi = mid;
            else lo = mid + 1;
        }
        who[i] = lo;
        at[i] = x - (lo ? s_have[lo - 1] : 0);
        page[i] = a.table[(size_t)lo * a.max_pages + at[i]];
    }
#pragma unroll
    for (int i = 0; i < ONE_ENTRIES; ++i)
        if (is_page(a, page[i])) atomicAdd(&s_left[page[i]], 1);
    __syncthreads();
    const bool refused = is_page(a, cut) && s_left[cut] > 1;
    if (refused) stay = L;
    s_stay[tid] = (stay + P - 1) >> a.pshift;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ONE_ENTRIES; ++i) {
        if (!is_page(a, page[i])) continue;
        if (at[i] < s_stay[who[i]]) page[i] = -1;
        else {
            atomicAdd(&s_left[page[i]], -1);
            atomicMax(&s_last[page[i]], tid * ONE_ENTRIES + i);
        }
    }
    __syncthreads();
    int n = 0;
#pragma unroll
    for (int i = 0; i < ONE_ENTRIES; ++i) {
        if (is_page(a, page[i]) && (s_left[page[i]] != 0 || s_last[page[i]] != tid * ONE_ENTRIES + i)) page[i] = -1;
        n += is_page(a, page[i]);
    }
    int all;
    int to = free0 + wg_incl_scan<ONE>(n, part, &all) - n;
#pragma unroll
    for (int i = 0; i < ONE_ENTRIES; ++i)
        if (is_page(a, page[i])) {
            if (to < a.n_pages) a.pool_out[to] = page[i];
            ++to;
        }
    if (tid < a.B) {
        a.len_out[tid] = stay;
        a.status[tid] = refused;
    }
    if (tid == 0) a.pool_n_out[0] = min(free0 + all, a.n_pages);
}
// They go to the pool, behind those of the blocks before, and what is known only now is written over what may be the call's input.
template <bool COMPACT>
__global__ __launch_bounds__(ET) void push_kernel(Args a) {
    __shared__ int part[ET / 64], s_before;
    int b, e;
    entry_of(a, blockIdx.x, b, e);
    const int p = given_back<COMPACT>(a, b, e), blocks = a.B * a.segs;
    if (threadIdx.x == 0) s_before = a.summed ? a.w.block[blockIdx.x] : 0;
    int all;
    const int upto = wg_incl_scan<ET>(p >= 0, part, &all);
    const bool last = blockIdx.x == blocks - 1;
    if (!a.summed && (all || last)) {
        int sum = 0;
        for (int i = threadIdx.x; i < (int)blockIdx.x; i += ET) sum += a.w.block[i];
        if (sum) atomicAdd(&s_before, sum);
    }
    __syncthreads();
    const int top = a.w.head[0] - (COMPACT ? a.w.head[1] : 0);
    const long long at = (long long)top + s_before + upto - 1;
    if (p >= 0 && at < a.n_pages) a.pool_out[at] = p;
    if (e == 0) a.len_out[b] = a.w.stay[b];
    if (last && threadIdx.x == 0) a.pool_n_out[0] = (int)min((long long)top + s_before + all, (long long)a.n_pages);
}
// Few blocks: a workgroup pushes for all of them, without counts, beside the workgroups that move tokens.  It takes them one after the other, 1 us each, behind
// the codes if those take less, and saves a launch.  This way / by counts and a fourth launch, from a graph: 1 / 4 / 8 / 16 requests of 600 tokens x 4 heads of 64 13.7 / 15.0 /
// 20.5 / 30.2 us and 16.0 / 17.4 / 18.4 / 19.9 (launched one by one 16.6 / 16.2 / 22.2 / 30.7 and 19.4 / 19.3 / 20.3 / 21.7); 3 of up to 37440 x 8 heads of 128 (9 blocks) 76 and 81, 8 of
// 6300 53.4 and 57.5, 12 of 3700 49 and 53, of which few are kept 25 and 22; 16 of 6300 122 and 120, few 37 and 25.
constexpr int PUSH_ALL = 9;
constexpr int PUSH_ROOM = 16;   // (room for nine alone: the kernel's registers are dealt out otherwise, 77.3 us instead of 76.2)
template <bool COMPACT>
__device__ __forceinline__ void push_all(const Args &a, int blocks) {
    __shared__ int s_part[ET / 64];
    int top = a.w.head[0] - (COMPACT ? a.w.head[1] : 0);
    int p[PUSH_ROOM];
#pragma unroll
    for (int i = 0; i < PUSH_ROOM; ++i) {
        int b, e;
        entry_of(a, i, b, e);
        p[i] = i < blocks ? given_back<COMPACT>(a, b, e) : -1;
        if (i < blocks && e == 0) a.len_out[b] = a.w.stay[b];
    }
#pragma unroll
    for (int i = 0; i < PUSH_ROOM; ++i) {
        if (i >= blocks) break;
        int all;
        const long long at = (long long)top + wg_incl_scan<ET>(p[i] >= 0, s_part, &all) - 1;
        if (p[i] >= 0 && at < a.n_pages) a.pool_out[at] = p[i];
        top = (int)min((long long)top + all, (long long)a.n_pages);
    }
    if (threadIdx.x == 0) a.pool_n_out[0] = top;
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

// A workgroup per request goes through its mask, 64 tokens per thread: how many are kept before every group of 16, which pages stay whole,
// which of the new ones are fresh and where their tokens begin.  It keeps the old table row, as the new one may be written over it.  Whoever has a
// new page's first token writes about that page, so that nothing has to be cleared before, and all loads of a round are one trip to memory: three requests of up
// to 37440 tokens 5.3 us.  More workgroups than there are requests help with the pages' states and copy the pool.  (16 tokens per thread and a list of
// every token's place: 15; its stores, four bytes apart by lanes sixteen apart, were most of it.)
__global__ __launch_bounds__(1024) void mask_kernel(Args a) {
    __shared__ int part[16];
    const int b = blockIdx.x, tid = threadIdx.x, P = 1 << a.pshift;
    if (b >= a.B) {
        clear_states(a);
        if (a.pool_out != a.pool)
            for (size_t i = (size_t)(b - a.B) * 1024 + tid; i < (size_t)a.n_pages; i += (size_t)(gridDim.x - a.B) * 1024) a.pool_out[i] = a.pool[i];
        return;
    }
    const int L = tokens_of(a, b), have = (L + P - 1) >> a.pshift;
    const size_t row = (size_t)b * a.max_pages;
    const u32x4 *mask = (const u32x4 *)(a.mask + (row << a.pshift));
    Group *group = a.w.group + (row << a.pshift) / 16;
    clear_states(a);
    const int per = P / 16;   // groups of a page: 1, 2 or 4
    int kept = 0, fresh = 0;
    for (int i0 = 0; i0 < L; i0 += 64 * 1024) {
        const int t0 = i0 + 64 * tid;
        u32x4 x[4];
        int page[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const bool here = t0 + 16 * q < L;   // so that the group's bytes are the row's
            x[q] = here ? mask[t0 / 16 + q] : u32x4{0, 0, 0, 0};
            page[q] = here ? a.table[row + ((t0 + 16 * q) >> a.pshift)] : -1;
        }
        unsigned bits[4], there[4];
        int n = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int left = L - t0 - 16 * q;
            there[q] = left >= 16 ? 0xFFFFu : left > 0 ? (1u << left) - 1u : 0u;
            bits[q] = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) bits[q] |= (x[q][i / 4] >> (8 * (i % 4)) & 0xFFu) ? 1u << i : 0u;
            bits[q] = is_page(a, page[q]) ? bits[q] & there[q] : 0;
            n += __builtin_popcount(bits[q]);
        }
        int all;
        int rank = kept + wg_incl_scan<1024>(n, part, &all) - n;
        kept += all;
        // the new page whose first token is in the group, and the old page that it is, or -1
        int j[4], s[4], n_fresh = 0;
        bool first[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int u = t0 / 16 + q, c = __builtin_popcount(bits[q]), end = rank + c;
            first[q] = c && ((end - 1) >> a.pshift << a.pshift) >= rank;
            j[q] = (end - 1) >> a.pshift;
            // whole: begins at a page's beginning, nothing missing up to the page's or the request's end
            bool whole = there[q] && !(u & (per - 1)) && !(rank & (P - 1));
#pragma unroll
            for (int i = 0; i < 4; ++i) whole = whole && (i < q || i >= q + per || bits[i] == there[i]);
            s[q] = first[q] && whole ? (16 * u) >> a.pshift : -1;
            n_fresh += first[q] && s[q] < 0;
            if (there[q]) {
                group[u] = Group{rank, bits[q]};
                if (!(u & (per - 1))) {
                    const size_t at = row + ((16 * u) >> a.pshift);
                    a.w.old[at] = page[q];
                    a.w.link[at] = whole ? rank >> a.pshift : -1;
                }
            }
            rank = end;
        }
        int f = fresh + wg_incl_scan<1024>(n_fresh, part, &all) - n_fresh;
        fresh += all;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (first[q]) {
                a.w.from[row + j[q]] = s[q] >= 0 ? s[q] : ~f;
                a.w.start[row + j[q]] = t0 / 16 + q;
                f += s[q] < 0;
            }
    }
    if (tid == 0) {
        a.w.have[b] = have;
        a.w.stay[b] = kept;
        a.w.need[b] = fresh;
    }
}

// Which requests are refused, and where the fresh pages of the others begin.  One workgroup, where there are too many requests for each block of entries to do so: 256 /
// 1024 / 2048 / 4096 / 16384 requests of 30 tokens 25.5 / 43.1 / 68.9 / 128 / 444 us with this launch, 24.4 / 42.7 / 68.7 / 136 / 601 without.
constexpr int ADMIT_ALL = 1024;
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

// New table rows, the list of fresh pages, the holders of old pages and those that give them up, and the pool as it was.  A trip to memory after the
// other, 5.5 us.
__global__ __launch_bounds__(ET) void relink_kernel(Args a) {
    __shared__ int part[ET / 64];
    int b, e;
    entry_of(a, blockIdx.x, b, e);
    const size_t at = (size_t)b * a.max_pages + e;
    const int have = a.w.have[b];
    int stay = a.w.stay[b];
    const int old = e < have ? a.w.old[at] : -1, link = e < have ? a.w.link[at] : 0, was = e < a.max_pages ? a.table[at] : -1;
    const bool is_new = e < (stay + (1 << a.pshift) - 1) >> a.pshift;   // unless the request is refused
    const int from = is_new ? a.w.from[at] : 0, start = is_new ? a.w.start[at] : 0;
    const int free0 = clipped(a.pool_n[0], a.n_pages);
    int base;
    if (a.admitted) base = a.w.base[b];
    else {   // the sums up to the request, and for the first workgroup up to the last one that is not refused
        int mine = 0, before = 0, taken = 0;
        for (int i0 = 0; i0 < a.B; i0 += ET) {
            const int i = i0 + threadIdx.x, need = i < a.B ? a.w.need[i] : 0;
            int all;
            const int upto = before + wg_incl_scan<ET>(need, part, &all);
            if (i == b) mine = need > 0 && upto > free0 ? -1 : min(upto - need, free0);
            if (need > 0 && upto <= free0) taken = upto;
            before += all;
        }
        __shared__ int s_base, s_taken;
        if (threadIdx.x == 0) s_taken = 0;
        __syncthreads();
        if (threadIdx.x == b % ET) s_base = mine;
        if (taken) atomicMax(&s_taken, taken);
        __syncthreads();
        base = s_base;
        if (e == 0) {
            a.w.base[b] = base;
            a.status[b] = base < 0;
            if (base < 0) a.w.stay[b] = tokens_of(a, b);
            if (b == 0) a.w.head[0] = free0, a.w.head[1] = s_taken;
        }
    }
    if (is_page(a, old)) atomicAdd(&a.w.state[old].hold, 1);
    if (base < 0) {
        if (e < a.max_pages && a.table_out != a.table) a.table_out[at] = was;
    } else if (e < a.max_pages) {
        int p = -1;
        if (is_new) {
            if (from >= 0) p = a.w.old[(size_t)b * a.max_pages + from];
            else {
                const int k = base + ~from;
                p = a.pool[free0 - 1 - k];
                a.w.made[k] = Fresh{p, b, (tokens_of(a, b) + 15) / 16, start, e << a.pshift, min(1 << a.pshift, stay - (e << a.pshift)), {0, 0}};
            }
        }
        a.table_out[at] = p;
        if (link < 0 && is_page(a, old)) give_up(a, old, (int)at);
    }
    if (a.copies)
        for (size_t i = (size_t)blockIdx.x * ET + threadIdx.x; i < (size_t)a.n_pages; i += (size_t)gridDim.x * ET) a.pool_out[i] = a.pool[i];
}

// Codes carried over to a scale 1 / ratio times as large; NaN stays.
__device__ __forceinline__ unsigned carried(unsigned w, float ratio) {
    int y = 0;
    y = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * ratio, y, false);
    y = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8((int)w, 2) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * ratio, y, true);
    return (unsigned)y;
}
__device__ __forceinline__ u32x4 carried(u32x4 w, float ratio) {
    return u32x4{carried(w[0], ratio), carried(w[1], ratio), carried(w[2], ratio), carried(w[3], ratio)};
}

// A mask of the bytes below n of eight.
__device__ __forceinline__ uint64_t bytes_below(int n) { return n >= 8 ? ~0ull : n > 0 ? (1ull << (8 * n)) - 1ull : 0ull; }
struct __attribute__((packed, aligned(1))) Bytes16 {
    u32x4 w;
};

// The first workgroups count the pages that blocks of entries give back; the others fill fresh pages, `heads` heads of one after the other, PIECES
// times 16 bytes per thread: of a token (K) and of a coordinate (V).  Bound by the trips to memory of an item: what it is -> groups of tokens -> old pages ->
// codes and, beside them, scales;  so codes are asked for before the scales are there, all of an item's K and the first two runs of its V.
// 112 MB of codes of three windows 52 us (4.1 TB/s read and written), 98 MB in runs of 14 tokens 58 (whole cells of V are read: 4.2 TB/s) on the same pages again and again, of
// which some are in the last-level cache; 64 and 70 (3.5 TB/s) from memory.  (An item's heads one after the other, scales first: 54 and 75;  a branch between the loads, so that each is
// waited for: 65 and 75;  three wavefronts per SIMD 55 and 65, five spill: 93.)
constexpr int PIECES = 4, MAX_HEADS = 16;   // 1024 pieces of a page are 2 heads of 64 x 128, 16 of 16 x 64
__global__ __launch_bounds__(256, 4) void gather_kernel(Args a, int blocks, int heads) {
    if (a.one_pushes) {
        if (blockIdx.x == 0) {
            push_all<true>(a, blocks);
            return;
        }
        blocks = 1;   // the workgroups before those that move tokens
    } else if ((int)blockIdx.x < blocks) {
        count_block<true>(a, blockIdx.x);
        return;
    }
    __shared__ int s_token[64];
    __shared__ size_t s_head[64];                  // of a token's page: number * Hkv
    __shared__ float s_ratio[2][MAX_HEADS][64];
    __shared__ int s_edges;                        // whether some are of the first or the last page
    __shared__ unsigned s_runs[4];                 // bit i of word t: token 16 t + i begins a run of neighbours in one cell
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int P = 1 << a.pshift, dshift = a.pg.d == 128 ? 7 : 6, ushift = a.pshift + dshift - 4, Hkv = a.pg.Hkv, parts = (Hkv + heads - 1) / heads;
    const size_t head_bytes = (size_t)P << dshift;
    const long long items = (long long)a.w.head[1] * parts;
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    for (long long it = blockIdx.x - blocks; it < items; it += gridDim.x - blocks) {
        const int h0 = (int)(it % parts) * heads, mine = min(heads, Hkv - h0);
        const Fresh f = a.w.made[it / parts];
        const int dst = uniform(f.page), n = uniform(f.n);
        if (!is_page(a, dst)) continue;   // the caller's pool names no page: nothing is written
        const size_t row = (size_t)f.b * a.max_pages;
        __syncthreads();   // what the last item had in LDS has been read
        if (wave == 0) {
            const Group *group = a.w.group + (row << a.pshift) / 16;
            int u = f.start;
            bool more = true;
            while (more) {   // 64 groups a round, until the page's last token
                const Group g = u + lane < f.groups ? group[u + lane] : Group{0, 0};
                int o = g.rank - f.first;
                for (unsigned m = g.bits; m; m &= m - 1, ++o)
                    if (o >= 0 && o < n) s_token[o] = 16 * (u + lane) + __builtin_ctz(m);
                u += 64;
                more = u < f.groups && __builtin_amdgcn_readlane(o, 63) < n;
            }
            __builtin_amdgcn_wave_barrier();
            const int t = lane < n ? s_token[lane] : -2, before = __shfl_up(t, 1, 64);
            const unsigned long long runs = __ballot(lane < n && ((lane & 15) == 0 || (t & 15) == 0 || t != before + 1));
            if (lane < 4) s_runs[lane] = (unsigned)(runs >> (16 * lane)) & 0xFFFFu;
            const int src = lane < n ? a.w.old[row + (t >> a.pshift)] : -1;
            s_head[lane] = (size_t)max(src, 0) * Hkv;
            const bool edge = __any(src == 0 || src == a.n_pages - 1);
            if (lane == 0) s_edges = edge;
        }
        __syncthreads();
        const bool edges = uniform(s_edges);
        float ks[MAX_HEADS / 4], vs[MAX_HEADS / 4];   // a token per lane, every fourth head
#pragma unroll
        for (int i = 0; i < MAX_HEADS / 4; ++i)
            if (wave + 4 * i < mine) {
                const size_t at = s_head[lane] + h0 + wave + 4 * i;
                ks[i] = lane < n ? a.pg.kscale[at] : 0.0f;
                vs[i] = lane < n ? a.pg.vscale[at] : 0.0f;
            }
        // pieces tid + 256 r of the item's: head, cell (tb, db), token or coordinate of it.  A wavefront's are of the same 16 tokens.
        u32x4 k[PIECES], v[PIECES][2];
        int hh[PIECES], tb[PIECES], c[PIECES], first[PIECES], behind[PIECES], last[PIECES];
        unsigned m[PIECES];
        auto run_of = [&](int r, int &o, int &e) __attribute__((always_inline)) {   // the next run: [o, e) of the 16 tokens
            o = __builtin_ctz(m[r]);
            m[r] &= m[r] - 1;
            e = m[r] ? __builtin_ctz(m[r]) : min(n - 16 * tb[r], 16);
        };
        // A run's bytes are brought to their places by the address that they are loaded from, some bytes in front of or behind their coordinate's.
        // In the array's first and last page those may lie outside of it: such runs are brought there by shifts, when they are put.
        auto place_of = [&](int r, int o, int &s) __attribute__((always_inline)) {
            const int t = 16 * tb[r] + o, off = uniform(s_token[t]) & (P - 1);
            s = o - (off & 15);
            return a.pg.V8 + (s_head[t] + h0 + hh[r]) * head_bytes + ((off >> 4) << (dshift + 4)) + c[r];
        };
        auto ask = [&](int r, int o) __attribute__((always_inline)) {
            int s;
            const uint8_t *p = place_of(r, o, s);
            const uint8_t *q = p - s;   // without a branch, behind which loads would be waited for one by one
            if (edges) q = p;
            return ((const Bytes16 *)q)->w;
        };
        auto shifted = [&](int r, int o, u32x4 x) __attribute__((always_inline)) {
            int s;
            place_of(r, o, s);
            __uint128_t y = ((__uint128_t)((uint64_t)x[3] << 32 | x[2]) << 64) | ((uint64_t)x[1] << 32 | x[0]);
            y = s >= 0 ? y << (8 * s) : y >> (-8 * s);
            return u32x4{(unsigned)y, (unsigned)(y >> 32), (unsigned)(y >> 64), (unsigned)(y >> 96)};
        };
#pragma unroll
        for (int r = 0; r < PIECES; ++r) {
            const int x = tid + 256 * r, u = x & ((1 << ushift) - 1), t = (u >> dshift) * 16 + u % 16;
            hh[r] = uniform(x >> ushift);
            tb[r] = uniform(u >> dshift);
            c[r] = (u >> 4 & ((1 << dshift) / 16 - 1)) * 256 + u % 16 * 16;
            k[r] = u32x4{0, 0, 0, 0};
            if (hh[r] < mine && t < n) {
                const int off = s_token[t] & (P - 1);
                k[r] = *(const u32x4 *)(a.pg.K8 + (s_head[t] + h0 + hh[r]) * head_bytes + ((off >> 4) << (dshift + 4)) + (c[r] & ~255) + (off & 15) * 16);
            }
        }
#pragma unroll
        for (int r = 0; r < PIECES; ++r) {
            m[r] = hh[r] < mine ? uniform(s_runs[tb[r]]) : 0;
            first[r] = behind[r] = last[r] = 0;
            if (m[r]) {
                int o;
                run_of(r, o, behind[r]);
                v[r][0] = ask(r, o);
                if (m[r]) {
                    run_of(r, first[r], last[r]);
                    v[r][1] = ask(r, first[r]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < MAX_HEADS / 4; ++i)
            if (wave + 4 * i < mine) {
                const int h = wave + 4 * i;
                float km = fmaxf(ks[i], 0.0f), vm = fmaxf(vs[i], 0.0f);   // of those that are numbers: the same in all lanes
#pragma unroll
                for (int o = 1; o < 64; o *= 2) {
                    km = fmaxf(km, shfl_xor(km, o));
                    vm = fmaxf(vm, shfl_xor(vm, o));
                }
                s_ratio[0][h][lane] = ks[i] == km ? 1.0f : ks[i] / km;   // both may be 0: of a page that nothing has been written to
                s_ratio[1][h][lane] = vs[i] == vm ? 1.0f : vs[i] / vm;
                if (lane == 0) {
                    a.pg.kscale[(size_t)dst * Hkv + h0 + h] = km;
                    a.pg.vscale[(size_t)dst * Hkv + h0 + h] = vm;
                }
            }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < PIECES; ++r) {
            if (hh[r] >= mine) continue;
            const int x = tid + 256 * r, u = x & ((1 << ushift) - 1), t = tb[r] * 16 + u % 16;
            const float ratio = s_ratio[0][hh[r]][min(t, n - 1)];
            if (ratio != 1.0f) k[r] = carried(k[r], ratio);
            const size_t to = ((size_t)dst * Hkv + h0 + hh[r]) * head_bytes + (size_t)u * 16;
            *(u32x4 *)(a.pg.K8 + to) = k[r];
            u32x4 y = {0, 0, 0, 0};
            auto put = [&](u32x4 w, int o, int e) __attribute__((always_inline)) {
                if (edges) w = shifted(r, o, w);
                const float by = s_ratio[1][hh[r]][16 * tb[r] + o];
                if (by != 1.0f) w = carried(w, by);
                const uint64_t lo = bytes_below(e) & ~bytes_below(o), hi = bytes_below(e - 8) & ~bytes_below(o - 8);
                y[0] |= w[0] & (unsigned)lo, y[1] |= w[1] & (unsigned)(lo >> 32), y[2] |= w[2] & (unsigned)hi, y[3] |= w[3] & (unsigned)(hi >> 32);
            };
            if (behind[r]) put(v[r][0], 0, behind[r]);   // the first run begins a cell
            if (last[r]) put(v[r][1], first[r], last[r]);
            while (m[r]) {
                int o, e;
                run_of(r, o, e);
                put(ask(r, o), o, e);
            }
            *(u32x4 *)(a.pg.V8 + to) = y;
        }
    }
}

}  // namespace share

// Lets kv_pages_free use as much LDS as its pages' states need.
int share_setup() {
    static DeviceOnce once;
    return once.run([](int) {
        return hipFuncSetAttribute((const void *)share::free_one_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * sizeof(int) * share::ONE_PAGES) == hipSuccess
                   ? FASTAR_OK
                   : FASTAR_ERR_HIP;
    });
}
size_t pages_ws_bytes(int B, int max_pages, int n_pages, int P) {
    if (B < 0 || max_pages <= 0 || n_pages <= 0 || !page_size_ok(P)) return 0;
    share::Work w;
    return share::lay_out(w, nullptr, B, max_pages, n_pages, P);
}

// Blocks of entries up to which each sums up the counts of those before it; beyond, a launch does so for all.  512 / 1024 / 2048 / 4096 requests of 100 tokens freed: each by
// itself 14.5 / 16.8 / 20.7 / 28.7 us from a graph, 21.4 / 18.6 / 21.6 / 30.0 launched one by one; by a launch 14.1 / 15.8 / 18.4 / 24.5 and 25.0 / 24.8 / 24.7 / 27.6.  Thinned out, 17 /
// 64 / 512 / 4096: 20.9 / 24.7 / 38.3 / 214 and 22.5 / 24.8 / 38.0 / 208 from a graph.
constexpr int SUM_ALL = 2048;

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
    a.one_pushes = B * a.segs <= share::PUSH_ALL;
    a.summed = B * a.segs > SUM_ALL;
    a.admitted = B > share::ADMIT_ALL;
    share::lay_out(a.w, (char *)ws, B, max_pages, n_pages, P);
    return a;
}
static int nothing(const share::Args &a, hipStream_t s) {
    hipLaunchKernelGGL(share::nothing_kernel, dim3((unsigned)((a.n_pages + 255) / 256)), dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}
// The blocks' counts summed up, if there are too many for every block to do so, and the pages pushed.
template <bool COMPACT>
static int push(const share::Args &a, hipStream_t s) {
    if (a.summed) {
        hipLaunchKernelGGL(share::scan_kernel, dim3(1), dim3(1024), 0, s, a.w.block, a.B * a.segs);
        FASTAR_LAUNCH_CHECK();
    }
    hipLaunchKernelGGL((share::push_kernel<COMPACT>), dim3((unsigned)(a.B * a.segs)), dim3(share::ET), 0, s, a);
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
    if (B <= share::ONE && (int64_t)B * max_pages <= share::ONE_TABLE && n_pages <= share::ONE_PAGES) {
        if (const int rc = share_setup(); rc != FASTAR_OK) return rc;
        hipLaunchKernelGGL(share::free_one_kernel, dim3(1), dim3(share::ONE), 2 * sizeof(int) * (size_t)n_pages, s, a);
        FASTAR_LAUNCH_CHECK();
        return FASTAR_OK;
    }
    const dim3 grid((unsigned)(B * a.segs));
    hipLaunchKernelGGL(share::clear_kernel, dim3((unsigned)((n_pages + 255) / 256)), dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(share::hold_kernel, grid, dim3(share::ET), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(share::cut_kernel, grid, dim3(share::ET), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(share::count_kernel, grid, dim3(share::ET), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    return push<false>(a, s);
}

extern "C" int kv_pages_compact(const fastar_pages *pages, const uint8_t *keep, const int32_t *len, const int32_t *table, int B, int max_pages,
                                const int32_t *pool, const int32_t *pool_n, int32_t *len_out, int32_t *table_out, int32_t *pool_out,
                                int32_t *pool_n_out, int32_t *status, void *ws, size_t ws_bytes, void *stream) {
    using namespace fastar;
    if (const int rc = pages_check(pages); rc != FASTAR_OK) return rc;
    if (const int rc = share_check(len, table, B, max_pages, pool, pool_n, pages->n_pages, pages->P, len_out, pool_n_out, status, ws, ws_bytes);
        rc != FASTAR_OK)
        return rc;
    if ((int64_t)max_pages * pages->P > MAX_KEYS) return FASTAR_ERR_UNSUPPORTED;   // positions a round beyond a request's end are 32-bit
    if (!pool_out || (B > 0 && (!keep || ((uintptr_t)keep & 15) || !table_out))) return FASTAR_ERR_INVALID_ARG;
    share::Args a = share_args(len, table, B, max_pages, pool, pool_n, pages->n_pages, pages->P, len_out, pool_out, pool_n_out, status, ws);
    if (B == 0) return nothing(a, (hipStream_t)stream);
    a.pg = *pages;
    a.mask = keep;
    a.table_out = table_out;
    const hipStream_t s = (hipStream_t)stream;
    const unsigned blocks = (unsigned)(B * a.segs);
    // Workgroups beside those of the requests where the pool is so large that these would go on for it.  One request of 600 tokens, pools of
    // 2000 / 16384 / 131072 / 1048576 pages: 14.7 / 13.5 / 13.8 / 16.0 us, 14.5 / 22.4 / 88 / 1140 with none; 64 requests 27.6 / 31.2 / 32.6 / 35.4 and 27.5 / 31.1 / 32.4 / 48.2.
    const unsigned room = UINT32_MAX / 1024 - (unsigned)B, more = a.n_pages / 4096 > B ? std::min((unsigned)std::min(a.n_pages / 1024, 1024), room) : 0u;
    a.copies = more == 0 && pool_out != pool;
    hipLaunchKernelGGL(share::mask_kernel, dim3((unsigned)B + more), dim3(1024), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    if (a.admitted) {
        hipLaunchKernelGGL(share::admit_kernel, dim3(1), dim3(1024), 0, s, a);
        FASTAR_LAUNCH_CHECK();
    }
    hipLaunchKernelGGL(share::relink_kernel, dim3(blocks), dim3(share::ET), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    const int heads = std::min(pages->Hkv, 256 * share::PIECES * 16 / (pages->P * pages->d));
    const int64_t items = std::min<int64_t>((int64_t)B * max_pages, a.n_pages) * ((pages->Hkv + heads - 1) / heads);   // at most
    hipLaunchKernelGGL(share::gather_kernel, dim3((a.one_pushes ? 1 : blocks) + (unsigned)std::min<int64_t>(items, 2048)), dim3(256), 0, s, a, (int)blocks, heads);
    FASTAR_LAUNCH_CHECK();
    return a.one_pushes ? FASTAR_OK : push<true>(a, s);
}
