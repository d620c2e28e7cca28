// What the calls over packed sequences share: argument checks on the host, and a sequence's rows on the device.
#pragma once

#include <cmath>

#include "common.hpp"

namespace fastar {

// Views as the kernels take them: strides in bytes.
struct View {
    char *p;
    int64_t head, row;
};
inline View view_of(const fastar_rows *r, int elt) { return View{(char *)r->p, r->head * elt, r->row * elt}; }

inline bool view_ok(const fastar_rows *r, int elt) {
    return r && r->p && !((uintptr_t)r->p & 15) && r->head >= 0 && r->row >= 0 && !((r->head * elt) & 15) && !((r->row * elt) & 15);
}
// Rows of an output lie apart: the smaller stride clears a row, the larger one all that the smaller one spans.
inline bool rows_apart(const fastar_rows *r, int H, int64_t n, int d) {
    if (H == 1 && n == 1) return true;
    if (H == 1) return r->row >= d;
    if (n == 1) return r->head >= d;
    return (r->head >= d && r->row >= (H - 1) * r->head + d) || (r->row >= d && r->head >= (n - 1) * r->row + d);
}
constexpr int64_t MAX_PITCH = 1 << 24;   // bytes between rows of keys and values: offsets within a tile of 64 are 32-bit
constexpr int MAX_KEYS = 1 << 30;        // of a sequence: positions some tiles further than its end are 32-bit too
inline bool scale_ok(float scale) { return scale > 0.0f && std::isfinite(scale * 1.4426950408889634f); }
inline bool page_size_ok(int P) { return P == 16 || P == 32 || P == 64; }

// Rows [first, first + n) of a sequence, inside the array.
struct Rows {
    int first, n;
};

// 16 bytes per lane from global memory straight into LDS, lane after lane from dst on (uniform, as `base` is): from one base
// address, each lane at an offset of its own, which costs no vector instruction; or from an address per lane.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // m0 is named as clobbered
__device__ __forceinline__ void to_lds(const char *base, unsigned off, unsigned dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(dst), "v"(off), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void to_lds(const char *src, unsigned char *dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src, (__attribute__((address_space(3))) void *)dst, 16, 0, 0);
}
__device__ __forceinline__ unsigned lds_address(const void *p) {
    return (unsigned)(size_t)(__attribute__((address_space(3))) const unsigned char *)p;
}

// Maximum and sum over the four lanes of a row (lane % 16).
__device__ __forceinline__ float max_of_quarters(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_of_quarters(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Item u of a launch whose sequences have ceil(rows * group / R) * Hkv items each, in their order.  Every wavefront looks for
// itself, four sequences per lane, so that a launch of up to 256 sequences waits for one round of loads and for no barrier.
struct Item {
    int b, local, n;   // sequence, item within it, items that it has
    Rows q, k;
};
template <int R>
__device__ __forceinline__ bool find_item(const int32_t *__restrict__ cu_q, const int32_t *__restrict__ cu_k, int B, int n_tok_q, int n_tok_k,
                                          int group, int Hkv, int u, Item &out) {
    const int lane = lane_id();
    int before = 0;
    for (int b0 = 0; b0 < B; b0 += 256) {   // uniform
        int cq[5], ck[5];
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            const int b = min(b0 + 4 * lane + i, B);
            cq[i] = min(max(cu_q[b], 0), n_tok_q);
            ck[i] = min(max(cu_k[b], 0), n_tok_k);
        }
        int n[4], all = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            n[i] = (max(cq[i + 1] - cq[i], 0) * group + R - 1) / R * Hkv;
            all += n[i];
        }
        const int upto = before + (int)wave_incl_scan((unsigned)all);
        const unsigned long long hit = __ballot(u >= upto - all && u < upto);
        if (hit) {
            const int src = __builtin_ctzll(hit);
            int start = upto - all, i = 0;
            for (; i < 3; ++i) {
                if (u < start + n[i]) break;
                start += n[i];
            }
            auto pick = [&](const int *x) { return i == 0 ? x[0] : i == 1 ? x[1] : i == 2 ? x[2] : x[3]; };
            auto bcast = [&](int x) { return __builtin_amdgcn_readlane(x, src); };
            out.b = bcast(b0 + 4 * lane + i);
            out.local = u - bcast(start);
            out.n = bcast(pick(n));
            const int q0 = bcast(pick(cq)), q1 = bcast(pick(cq + 1)), k0 = bcast(pick(ck)), k1 = bcast(pick(ck + 1));
            out.q = Rows{q0, max(q1 - q0, 0)};
            out.k = Rows{k0, max(k1 - k0, 0)};
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// One row key by key over the keys that it sees, a wavefront, lane l coordinates l, l + 64: what tiles whose products brought in
// numbers that are none fall back to.
template <typename T, int D>
__device__ __forceinline__ void row_by_keys(const char *q, const char *K, int64_t k_pitch, const char *V, int64_t v_pitch, int seen,
                                            float scale_log2, float &m, float &l, float (&o)[D / 64]) {
    const int lane = lane_id();
    float qv[D / 64];
    m = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
        o[c] = 0.0f;
        qv[c] = (float)((const T *)q)[64 * c + lane];
    }
    for (int j = 0; j < seen; ++j) {
        const T *kp = (const T *)(K + (int64_t)j * k_pitch), *vp = (const T *)(V + (int64_t)j * v_pitch);
        float x = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 64; ++c) x = fmaf(qv[c], (float)kp[64 * c + lane], x);
#pragma unroll
        for (int i = 32; i > 0; i >>= 1) x += shfl_xor(x, i);
        const float mn = fmaxf(m, x);
        const float al = m == -INFINITY ? 0.0f : exp2f((m - mn) * scale_log2);
        const float p = exp2f((x - (mn == -INFINITY ? 0.0f : mn)) * scale_log2);
        m = mn;
        l = l * al + p;
#pragma unroll
        for (int c = 0; c < D / 64; ++c) o[c] = o[c] * al + p * (float)vp[64 * c + lane];
    }
}

}  // namespace fastar
