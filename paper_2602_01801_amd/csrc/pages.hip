// The paged 8-bit cache: block tables and slot maps from the requests' lengths (kv_pages_plan), and new keys and values into
// its pages (kv_pages_write).
#include "pages_dev.hpp"

namespace fastar {

namespace pages {

constexpr int PT = 1024;   // threads of the planning workgroup

// Inclusive prefix sum over the workgroup's PT threads (64-bit: lengths are the caller's and may be anything); the total in *all.
__device__ __forceinline__ long long wg_incl_scan(long long v, long long *part, long long *all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
    }
    __syncthreads();   // the last call's partial sums have been read
    if (lane == 63) part[wave] = v;
    __syncthreads();
    long long base = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < PT / 64; ++w) {
        const long long x = part[w];
        if (w < wave) base += x;
        sum += x;
    }
    *all = sum;
    return v + base;
}

__device__ __forceinline__ int slot_of(const int32_t *__restrict__ row, long long pos, int pshift, int n_pages) {
    const int page = row[pos >> pshift];
    return (unsigned)page < (unsigned)n_pages ? (page << pshift) + (int)(pos & ((1 << pshift) - 1)) : -1;
}

// Up to PT requests: a thread each, sums in 32 bits (the launch sees to it that they fit).  Everything that is read -- lengths, table
// entries below a request's own pages, the pool below its top -- is left as it is by the call, so that pages which go from one
// request to another by way of the pool are looked up where they come from, and tables, pool and slots are written side by side:
// two rounds of loads in all (one for lengths, one for pages), against six of the kernel for more requests.  With many tokens more
// workgroups repeat the sums and write slots only; that needs the lengths to stay in place, so not if len_out or pool_n_out is an input.
// 192 requests, a token each 14.1 -> 6.0 us, 64 prompts of 90122 tokens 13 -> 4.6; 1024 requests 5.8, 1025 by the other kernel 51, 10000 249.
constexpr int SMALL_LIMIT = 1 << 20;   // PT times this much stays below 2^31
__global__ __launch_bounds__(PT) void plan_small_kernel(const int32_t *__restrict__ n_new, const int32_t *len, int32_t *table, int B,
                                                        int max_pages, int32_t *pool, const int32_t *pool_n, int n_pages, int pshift,
                                                        int n_tok, int32_t *len_out, int32_t *pool_n_out, int32_t *__restrict__ cu,
                                                        int32_t *__restrict__ slot, int32_t *__restrict__ status, int n_slots) {
    __shared__ int part[3][PT / 64];
    __shared__ int s_rows[PT], s_back[PT], s_upto[PT], s_have[PT], s_len[PT];   // the first three: inclusive prefix sums
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int P = 1 << pshift;
    int n = 0, L = 0;
    bool ended = false;
    if (tid < B) {
        n = n_new[tid];
        L = (int)min(max((long long)len[tid], 0ll), (long long)max_pages << pshift);
        ended = n < 0;
        n = max(n, 0);
    }
    const int free0 = min(max(pool_n[0], 0), n_pages);
    const int have = (L + P - 1) >> pshift;
    int rows = (int)wave_incl_scan((unsigned)min(n, n_tok + 1)), back = (int)wave_incl_scan(ended ? (unsigned)have : 0u);
    if (lane == 63) {
        part[0][wave] = rows;
        part[1][wave] = back;
    }
    __syncthreads();
    auto add_before = [&](int which, int &v) {
        int all = 0;
#pragma unroll
        for (int i = 0; i < PT / 64; ++i) {
            const int x = part[which][i];
            if (i < wave) v += x;
            all += x;
        }
        return all;
    };
    const int n_rows = min(add_before(0, rows), n_tok), n_back = add_before(1, back);
    const int free1 = (int)min((long long)free0 + n_back, (long long)n_pages);
    const long long want = ((long long)L + n + P - 1) >> pshift;
    int st = want > max_pages ? 2 : rows > n_tok && n > 0 ? 3 : 0;
    const int ask = ended || st ? 0 : (int)max(want - have, 0ll);
    int upto = (int)wave_incl_scan((unsigned)ask);
    if (lane == 63) part[2][wave] = upto;
    __syncthreads();
    const int n_ask = add_before(2, upto);
    if (ask > 0 && upto > free1) st = 1;
    s_rows[tid] = min(rows, n_tok);
    s_back[tid] = back;
    s_upto[tid] = upto;
    s_have[tid] = have;
    s_len[tid] = st ? -1 : L;
    __syncthreads();
    auto owner = [&](const int *incl, int x) {   // the request whose part of the sums holds x
        int lo = 0, hi = B - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (incl[mid] > x) hi = mid;
            else lo = mid + 1;
        }
        return lo;
    };
    auto given_back = [&](int r) {
        const int i = owner(s_back, r);
        return table[(size_t)i * max_pages + r - (s_back[i] - s_have[i])];
    };
    auto taken = [&](int f) {   // the f-th page that is taken
        const int at = free1 - 1 - f;
        return at < free0 ? pool[at] : given_back(at - free0);
    };
    for (int t = blockIdx.x * PT + tid; t < min(n_rows, n_slots); t += gridDim.x * PT) {
        const int i = owner(s_rows, t);
        int y = -1;
        if (s_len[i] >= 0) {
            const int pos = s_len[i] + t - (i ? s_rows[i - 1] : 0), pg = pos >> pshift;
            const int page = pg < s_have[i] ? table[(size_t)i * max_pages + pg] : taken((i ? s_upto[i - 1] : 0) + pg - s_have[i]);
            if ((unsigned)page < (unsigned)n_pages) y = (page << pshift) + (pos & (P - 1));
        }
        slot[t] = y;
    }
    if (blockIdx.x) return;
    int n_take = n_ask;   // those asked for by requests before the first for which they do not suffice
    if (n_ask > free1) {
        const int i = owner(s_upto, free1);
        n_take = i ? s_upto[i - 1] : 0;
    }
    for (int f = tid; f < n_take; f += PT) {
        const int i = owner(s_upto, f);
        table[(size_t)i * max_pages + s_have[i] + f - (i ? s_upto[i - 1] : 0)] = taken(f);
    }
    for (int r = tid; r < free1 - free0; r += PT) pool[free0 + r] = given_back(r);
    if (tid < B) {
        cu[tid] = tid ? s_rows[tid - 1] : 0;
        len_out[tid] = ended ? 0 : st ? L : L + n;
        status[tid] = st;
    }
    if (tid == 0) {
        cu[B] = n_rows;
        pool_n_out[0] = free1 - n_take;
    }
}

// Any number of requests, 64-bit sums.  One workgroup: requests in rounds of PT.  Tables and the pool are updated by wavefronts, a request each, so that requests
// with many pages are copied 64 entries at a time.
template <bool SLOTS>
__global__ __launch_bounds__(PT) void plan_kernel(const int32_t *__restrict__ n_new, const int32_t *len, int32_t *table, int B,
                                                  int max_pages, int32_t *pool, const int32_t *pool_n, int n_pages, int pshift,
                                                  int n_tok, int32_t *len_out, int32_t *pool_n_out, int32_t *__restrict__ cu,
                                                  int32_t *__restrict__ slot, int32_t *__restrict__ status) {
    __shared__ long long part[PT / 64];
    __shared__ int s_first[PT], s_have[PT], s_n[PT], s_row[PT], s_len[PT];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int P = 1 << pshift;
    const long long cap = (long long)max_pages << pshift;
    const int free0 = min(max(pool_n[0], 0), n_pages);
    auto held = [&](int b) { return (int)min(max((long long)len[b], 0ll), cap); };
    // 1. pages of ended requests go back
    long long back = 0;
    for (int b0 = 0; b0 < B; b0 += PT) {
        const int b = b0 + tid;
        int have = 0;
        if (b < B && n_new[b] < 0) have = (held(b) + P - 1) >> pshift;
        long long all;
        const long long upto = wg_incl_scan(have, part, &all);
        s_have[tid] = have;
        s_first[tid] = (int)min(back + upto - have, (long long)n_pages);
        __syncthreads();
        for (int i = wave; i < min(PT, B - b0); i += PT / 64)
            for (int j = lane; j < s_have[i]; j += 64) {
                const long long at = (long long)free0 + s_first[i] + j;
                if (at < n_pages) pool[at] = table[(size_t)(b0 + i) * max_pages + j];
            }
        back += all;
        __syncthreads();
    }
    const long long free1 = min((long long)free0 + back, (long long)n_pages);
    __syncthreads();   // the pool is complete (and visible to the workgroup)
    // 2. requests take pages, in order
    long long rows = 0, need_sum = 0, taken = 0;
    for (int b0 = 0; b0 < B; b0 += PT) {
        const int b = b0 + tid;
        int n = 0, have = 0, L = 0, st = 0;
        bool ended = false;
        if (b < B) {
            ended = n_new[b] < 0;
            n = max(n_new[b], 0);
            L = held(b);
            have = (L + P - 1) >> pshift;
        }
        long long n_all;
        const long long end = rows + wg_incl_scan(n, part, &n_all);
        const long long want = ((long long)L + n + P - 1) >> pshift;
        if (want > max_pages) st = 2;
        else if (end > n_tok && n > 0) st = 3;
        const int ask = ended || st ? 0 : (int)max(want - have, 0ll);
        long long ask_all;
        const long long upto = need_sum + wg_incl_scan(ask, part, &ask_all);
        if (ask > 0 && upto > free1) st = 1;
        const int take = st ? 0 : ask;
        if (take > 0) taken = upto;   // admitted requests come first among those that ask
        s_first[tid] = (int)min(upto - ask, (long long)n_pages);
        s_have[tid] = have;
        s_n[tid] = take;
        __syncthreads();
        for (int i = wave; i < min(PT, B - b0); i += PT / 64)
            for (int j = lane; j < s_n[i]; j += 64)
                table[(size_t)(b0 + i) * max_pages + s_have[i] + j] = pool[free1 - 1 - s_first[i] - j];
        if (b < B) {
            cu[b] = (int)min(end - n, (long long)n_tok);
            if (b == B - 1) cu[B] = (int)min(end, (long long)n_tok);
            len_out[b] = ended ? 0 : st ? L : L + n;
            status[b] = st;
        }
        if constexpr (SLOTS) {
            __syncthreads();   // table entries are visible; s_n is free
            s_n[tid] = b < B ? (int)(min(end, (long long)n_tok) - min(end - n, (long long)n_tok)) : 0;
            s_row[tid] = (int)min(end - n, (long long)n_tok);
            s_len[tid] = st ? -1 : L;
            __syncthreads();
            for (int i = wave; i < min(PT, B - b0); i += PT / 64)
                for (int j = lane; j < s_n[i]; j += 64)
                    slot[s_row[i] + j] = s_len[i] < 0 ? -1 : slot_of(table + (size_t)(b0 + i) * max_pages, (long long)s_len[i] + j, pshift, n_pages);
        }
        rows += n_all;
        need_sum += ask_all;
        __syncthreads();
    }
    // the largest number taken by any thread's requests
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) taken = max(taken, (long long)__shfl_xor(taken, o, 64));
    if (lane == 0) part[wave] = taken;
    __syncthreads();
    if (tid == 0) {
        for (int w = 0; w < PT / 64; ++w) taken = max(taken, part[w]);
        pool_n_out[0] = (int)(free1 - taken);
        if (B == 0) cu[0] = 0;
    }
}

// Slots of many tokens: a thread each, its request by bisection of cu.
__global__ __launch_bounds__(256) void slots_kernel(const int32_t *__restrict__ table, int B, int max_pages, int n_pages, int pshift,
                                                    int n_tok, const int32_t *__restrict__ len_out, const int32_t *__restrict__ cu,
                                                    int32_t *__restrict__ slot, const int32_t *__restrict__ status) {
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= n_tok || t >= cu[B]) return;
    int lo = 0, hi = B;   // cu[lo] <= t < cu[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int n = cu[lo + 1] - cu[lo];
    slot[t] = status[lo] ? -1 : slot_of(table + (size_t)lo * max_pages, (long long)len_out[lo] - n + (t - cu[lo]), pshift, n_pages);
}

// ---- writing ----------------------------------------------------------------------------------------------------

// A workgroup looks at `chunk` rows of one head of K or V and writes the runs that begin there, a wavefront for every 16 tokens of
// a page, whose rows stay in registers between the run's maximum and the codes.  Bound by memory: every row is read once and every
// code written once, in whole lines: K by rows, whose halves of a cell's 16 bytes neighbouring lanes exchange; V two coordinates of
// every row per lane, whose codes over the rows are the lane's 32 consecutive bytes of the page (d = 64: twice 8), exchanged within
// the lane.  (A wavefront per page and tensor with 64 registers of data, K in pieces of 64 bytes, V of 16: 76 us where this takes
// 43 for 34612 tokens x 8 heads; a third of the wavefronts were resident, and they read and wrote in turn.)
template <bool BF16, int D, int PSHIFT>
__global__ __launch_bounds__(4 << PSHIFT) void write_kernel(View Kn, View Vn, const int32_t *__restrict__ slot, int n_tok, int chunk,
                                                            fastar_pages pg) {
    constexpr int P = 1 << PSHIFT, NW = P / 16;
    __shared__ unsigned s_top[2][NW];
    const int h = blockIdx.x % pg.Hkv, rest = blockIdx.x / pg.Hkv;
    const bool is_v = rest & 1;
    const View x = is_v ? Vn : Kn;
    uint8_t *codes = is_v ? pg.V8 : pg.K8;
    float *scales = is_v ? pg.vscale : pg.kscale;
    for_runs<PSHIFT>(slot, n_tok, (rest >> 1) * chunk, chunk, (unsigned)pg.n_pages << PSHIFT, 0, n_tok, [&](int t0, int sl, int n, int turn) __attribute__((always_inline)) {
        const int o = sl & (P - 1);
        const size_t ph = (size_t)(sl >> PSHIFT) * pg.Hkv + h;
        const Run run{x.p + h * x.head + (int64_t)(t0 - o) * x.row, x.row, o, o + n, codes + ph * (size_t)(D * P), scales + ph, o > 0 ? scales[ph] : 0.0f};
        if (is_v) v_run<BF16, D, PSHIFT>(run, s_top, turn);
        else k_run<BF16, D, PSHIFT>(run, s_top, turn);
    });
}

}  // namespace pages

}  // namespace fastar

extern "C" int kv_pages_plan(const int32_t *n_new, const int32_t *len, int32_t *table, int B, int max_pages, int32_t *pool,
                             const int32_t *pool_n, int n_pages, int P, int n_tok, int32_t *len_out, int32_t *pool_n_out,
                             int32_t *cu, int32_t *slot, int32_t *status, void *stream) {
    using namespace fastar;
    if (B < 0 || n_tok < 0 || max_pages <= 0 || n_pages <= 0) return FASTAR_ERR_INVALID_ARG;
    if (!pool || !pool_n || !pool_n_out || !cu || (n_tok > 0 && !slot)) return FASTAR_ERR_INVALID_ARG;
    if (B > 0 && (!n_new || !len || !table || !len_out || !status)) return FASTAR_ERR_INVALID_ARG;
    if (!page_size_ok(P)) return FASTAR_ERR_UNSUPPORTED;
    if ((int64_t)max_pages * P > INT32_MAX || (int64_t)n_pages * P > INT32_MAX) return FASTAR_ERR_UNSUPPORTED;
    const int pshift = __builtin_ctz((unsigned)P);
    const hipStream_t s = (hipStream_t)stream;
    if (B <= pages::PT && n_tok < pages::SMALL_LIMIT && max_pages < pages::SMALL_LIMIT) {
        // One workgroup writes ONE_SLOTS slots beside the rest; beyond that there are more workgroups, or a launch of their own where the
        // call works in place.  64 prompts of 2048 / 3840 / 6400 / 16000 slots in all: one workgroup 5.6 / 6.8 / 8.7 / 14.5 us, more of them 4.9
        // each; in place one 4.5 / 5.7 / 7.6 / 13.8, a second launch 6.2 / 6.7 / 6.5 / 6.7.
        constexpr int ONE_SLOTS = 4096;
        const bool alone = len_out == len || pool_n_out == pool_n;
        const int wgs = n_tok <= ONE_SLOTS || alone ? 1 : (n_tok + pages::PT - 1) / pages::PT;
        const bool later = n_tok > ONE_SLOTS && alone;
        hipLaunchKernelGGL(pages::plan_small_kernel, dim3((unsigned)wgs), dim3(pages::PT), 0, s, n_new, len, table, B, max_pages, pool,
                           pool_n, n_pages, pshift, n_tok, len_out, pool_n_out, cu, slot, status, later ? 0 : n_tok);
        FASTAR_LAUNCH_CHECK();
        if (later) {
            hipLaunchKernelGGL(pages::slots_kernel, dim3((unsigned)((n_tok + 255) / 256)), dim3(256), 0, s, table, B, max_pages, n_pages,
                               pshift, n_tok, len_out, cu, slot, status);
            FASTAR_LAUNCH_CHECK();
        }
        return FASTAR_OK;
    }
    if (n_tok <= 4096) {
        hipLaunchKernelGGL(pages::plan_kernel<true>, dim3(1), dim3(pages::PT), 0, s, n_new, len, table, B, max_pages, pool, pool_n,
                           n_pages, pshift, n_tok, len_out, pool_n_out, cu, slot, status);
        FASTAR_LAUNCH_CHECK();
        return FASTAR_OK;
    }
    hipLaunchKernelGGL(pages::plan_kernel<false>, dim3(1), dim3(pages::PT), 0, s, n_new, len, table, B, max_pages, pool, pool_n,
                       n_pages, pshift, n_tok, len_out, pool_n_out, cu, slot, status);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(pages::slots_kernel, dim3((unsigned)((n_tok + 255) / 256)), dim3(256), 0, s, table, B, max_pages, n_pages,
                       pshift, n_tok, len_out, cu, slot, status);
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}

namespace fastar {
int pages_check(const fastar_pages *pg) {
    if (!pg || !pg->K8 || !pg->V8 || !pg->kscale || !pg->vscale) return FASTAR_ERR_INVALID_ARG;
    if (((uintptr_t)pg->K8 & 15) || ((uintptr_t)pg->V8 & 15)) return FASTAR_ERR_INVALID_ARG;
    if (pg->n_pages <= 0 || pg->Hkv <= 0) return FASTAR_ERR_INVALID_ARG;
    if (!page_size_ok(pg->P) || (pg->d != 64 && pg->d != 128)) return FASTAR_ERR_UNSUPPORTED;
    if ((int64_t)pg->n_pages * pg->P > INT32_MAX || (int64_t)pg->Hkv * pg->P * pg->d > INT32_MAX) return FASTAR_ERR_UNSUPPORTED;
    return FASTAR_OK;
}
}  // namespace fastar

extern "C" int kv_pages_write(const fastar_pages *pages, const fastar_rows *K_new, const fastar_rows *V_new, int dtype,
                              const int32_t *slot, int n_tok, void *stream) {
    using namespace fastar;
    if (dtype != FASTAR_F32 && dtype != FASTAR_BF16) return FASTAR_ERR_INVALID_ARG;
    const int elt = dtype == FASTAR_BF16 ? 2 : 4;
    if (n_tok < 0) return FASTAR_ERR_INVALID_ARG;
    if (const int rc = pages_check(pages); rc != FASTAR_OK) return rc;
    if (n_tok == 0) return FASTAR_OK;
    if (!slot || !view_ok(K_new, pages->Hkv, n_tok, elt) || !view_ok(V_new, pages->Hkv, n_tok, elt)) return FASTAR_ERR_INVALID_ARG;
    const View k = view_of(K_new, pages->Hkv, n_tok, elt), v = view_of(V_new, pages->Hkv, n_tok, elt);
    if (k.row > MAX_PITCH || v.row > MAX_PITCH) return FASTAR_ERR_UNSUPPORTED;
    const int chunk = pages::rows_per_workgroup(n_tok, pages->Hkv, pages->P);
    const int64_t units = (int64_t)((n_tok + chunk - 1) / chunk) * pages->Hkv * 2;
    if (!launch_ok(units, 4 * pages->P)) return FASTAR_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)units);
#define FASTAR_WRITE(BF16, D, PSHIFT) \
    hipLaunchKernelGGL((pages::write_kernel<BF16, D, PSHIFT>), grid, dim3(4 << PSHIFT), 0, (hipStream_t)stream, k, v, slot, n_tok, chunk, *pages)
#define FASTAR_WRITE_P(BF16, D)                      \
    do {                                             \
        if (pages->P == 64) FASTAR_WRITE(BF16, D, 6); \
        else if (pages->P == 32) FASTAR_WRITE(BF16, D, 5); \
        else FASTAR_WRITE(BF16, D, 4);               \
    } while (0)
    if (dtype == FASTAR_BF16) {
        if (pages->d == 128) FASTAR_WRITE_P(true, 128);
        else FASTAR_WRITE_P(true, 64);
    } else {
        if (pages->d == 128) FASTAR_WRITE_P(false, 128);
        else FASTAR_WRITE_P(false, 64);
    }
#undef FASTAR_WRITE_P
#undef FASTAR_WRITE
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}
