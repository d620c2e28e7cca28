// The paged 8-bit cache: block tables and slot maps from the requests' lengths (kv_pages_plan), and new keys and values into
// its pages (kv_pages_write).
#include "packed.hpp"

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

// One workgroup: requests in rounds of PT.  Tables and the pool are updated by wavefronts, a request each, so that requests
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

constexpr float F8_MAX = 448.0f;

__device__ __forceinline__ float f8_in_range(float x) { return x != x ? x : fminf(fmaxf(x, -F8_MAX), F8_MAX); }
__device__ __forceinline__ unsigned f8_of(float a, float b, float c, float d) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f8_in_range(a), f8_in_range(b), w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f8_in_range(c), f8_in_range(d), w, true);
    return (unsigned)w;
}
__device__ __forceinline__ float finite_abs(float x) {
    x = fabsf(x);
    return x < INFINITY ? x : 0.0f;
}
// Exponent of the least power of two, 2^-100 at least, whose 448-fold is not below amax.
__device__ __forceinline__ int scale_exp(float amax) {
    int e;
    const float m = frexpf(amax, &e);   // 448 = 0.875 * 2^9
    return max(-100, amax == 0.0f ? -100 : m <= 0.875f ? e - 9 : e - 8);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

template <bool BF16>
__device__ __forceinline__ void load16(const char *p, float (&x)[16]) {
    if constexpr (BF16) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const u32x4 a = ((const u32x4 *)p)[q];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[8 * q + 2 * e] = bf16_lo(a[e]);
                x[8 * q + 2 * e + 1] = bf16_hi(a[e]);
            }
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 a = ((const f32x4 *)p)[q];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * q + e] = a[e];
        }
    }
}

// A wavefront looks at `chunk` rows of one head of K or V and writes the runs that begin there.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void write_kernel(View Kn, View Vn, const int32_t *__restrict__ slot, int n_tok, int chunk,
                                                    fastar_pages pg, int pshift) {
    constexpr int LR = D / 16;   // lanes of a row
    const int lane = threadIdx.x & 63;
    const int unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = unit % pg.Hkv, rest = unit / pg.Hkv;
    const bool is_v = rest & 1;
    const int first = (rest >> 1) * chunk, last = min(first + chunk, n_tok);
    if (first >= n_tok) return;
    const View x = is_v ? Vn : Kn;
    const char *xh = x.p + h * x.head;
    uint8_t *codes = is_v ? pg.V8 : pg.K8;
    float *scales = is_v ? pg.vscale : pg.kscale;
    const int P = 1 << pshift, n_slots = pg.n_pages << pshift;
    const int lr = lane / LR, lc = lane % LR;
    auto at = [&](int t) { return t >= 0 && t < n_tok && (unsigned)slot[t] < (unsigned)n_slots ? slot[t] : -1; };
    for (int t = first; t < last; ++t) {   // uniform
        const int s0 = at(t);
        if (s0 < 0) continue;
        const int page = s0 >> pshift, o = s0 & (P - 1);
        const int before = at(t - 1);
        if (before >= 0 && before == s0 - 1 && o > 0) continue;   // inside a run
        int n = 1;
        while (o + n < P && at(t + n) == s0 + n) ++n;
        float amax = 0.0f;
        for (int r = lr; r < n; r += 64 / LR) {
            float v[16];
            load16<BF16>(xh + (int64_t)(t + r) * x.row + lc * 16 * (BF16 ? 2 : 4), v);
#pragma unroll
            for (int e = 0; e < 16; ++e) amax = fmaxf(amax, finite_abs(v[e]));
        }
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) amax = fmaxf(amax, __shfl_xor(amax, m, 64));
        const int e_new = scale_exp(amax);
        const size_t ph = (size_t)page * pg.Hkv + h;
        uint8_t *cell0 = codes + ph * ((size_t)D << pshift);
        float scale = pow2(e_new);
        if (o > 0) {
            const float old = scales[ph];
            if (old >= scale) {
                scale = old;
            } else {   // the page's codes move to the larger scale, those of the run's rows before they are written
                const float ratio = old / scale;
                for (int i = lane; i < (D << pshift) / 4; i += 64) {
                    const unsigned w = ((unsigned *)cell0)[i];
                    ((unsigned *)cell0)[i] =
                        f8_of(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * ratio,
                              __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * ratio);
                }
                __threadfence();   // before other lanes' new codes go to the same words
            }
        }
        const float inv = 1.0f / scale;
        for (int r = lr; r < n; r += 64 / LR) {
            float v[16];
            load16<BF16>(xh + (int64_t)(t + r) * x.row + lc * 16 * (BF16 ? 2 : 4), v);
            u32x4 w;
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = f8_of(v[4 * q] * inv, v[4 * q + 1] * inv, v[4 * q + 2] * inv, v[4 * q + 3] * inv);
            uint8_t *cell = cell0 + (((o + r) >> 4) * LR + lc) * 256;
            if (!is_v) {
                *(u32x4 *)(cell + ((o + r) & 15) * 16) = w;
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) cell[e * 16 + ((o + r) & 15)] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
            }
        }
        if (lane == 0) scales[ph] = scale;
    }
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
    if ((int64_t)pg->n_pages * pg->P > INT32_MAX) return FASTAR_ERR_UNSUPPORTED;
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
    if (!slot || !view_ok(K_new, elt) || !view_ok(V_new, elt)) return FASTAR_ERR_INVALID_ARG;
    const int chunk = 16;
    const int64_t units = (int64_t)((n_tok + chunk - 1) / chunk) * pages->Hkv * 2;
    if (units > INT32_MAX - 4) return FASTAR_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((units + 3) / 4));
    const int pshift = __builtin_ctz((unsigned)pages->P);
    const View k = view_of(K_new, elt), v = view_of(V_new, elt);
#define FASTAR_WRITE(BF16, D) \
    hipLaunchKernelGGL((pages::write_kernel<BF16, D>), grid, dim3(256), 0, (hipStream_t)stream, k, v, slot, n_tok, chunk, *pages, pshift)
    if (dtype == FASTAR_BF16) {
        if (pages->d == 128) FASTAR_WRITE(true, 128);
        else FASTAR_WRITE(true, 64);
    } else {
        if (pages->d == 128) FASTAR_WRITE(false, 128);
        else FASTAR_WRITE(false, 64);
    }
#undef FASTAR_WRITE
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}
