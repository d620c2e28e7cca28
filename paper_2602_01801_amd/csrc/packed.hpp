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
// The stride of a dimension of one means nothing and may be anything.
inline View view_of(const fastar_rows *r, int H, int n, int elt) {
    return View{(char *)r->p, H > 1 ? r->head * elt : 0, n > 1 ? r->row * elt : 0};
}
inline bool view_ok(const fastar_rows *r, int H, int n, int elt) {
    auto stride_ok = [&](int64_t s) { return s >= 0 && !((s * elt) & 15); };
    return r && r->p && !((uintptr_t)r->p & 15) && (H <= 1 || stride_ok(r->head)) && (n <= 1 || stride_ok(r->row));
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
// A launch's threads along its first dimension are counted in 32 bits.
inline bool launch_ok(int64_t workgroups, int threads) { return workgroups * threads <= UINT32_MAX; }
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

// The kernel's only argument, read again from where the launch left it: what the rare paths behind a loop need of it is then not held
// in registers over the loop (32760 tokens x 12 heads 2.87 -> 2.79 ms).
template <class Args>
__device__ __forceinline__ Args args_anew() {
    static_assert(sizeof(Args) % 4 == 0);
    struct Words {
        unsigned w[sizeof(Args) / 4];
    } x;
    auto *p = (const __attribute__((address_space(4))) unsigned *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
#pragma unroll
    for (unsigned i = 0; i < sizeof(Args) / 4; ++i) x.w[i] = p[i];
    return __builtin_bit_cast(Args, x);
}

// ln of a row's sum of weights from its reference score and the sum l against it, from log2 but where scaled scores leave its range.
__device__ __forceinline__ float lse_of(float m, float l, float scale_log2) {
    constexpr float LN2 = 0.6931471805599453f;
    const float x = m * scale_log2 + __log2f(l);
    return l == 0.0f ? -INFINITY : fabsf(x) < INFINITY ? x * LN2 : m * (scale_log2 * LN2) + __log2f(l) * LN2;
}
// Whether a row with keys has a sum of weights: the reference score's own weight is one, but m * scale is rounded in the exponent of
// the others, which shows from scaled scores of 2^24 on and takes weights out of the range, up or down, from about 2^31 on.
__device__ __forceinline__ bool sums_up(float m, float l) { return m == -INFINITY || (l >= 0.25f && l < INFINITY); }
// Whether a sum of weights that does not add up is no number because some score is none, which is what the row is then.
__device__ __forceinline__ bool no_number(float m, float l, float scale_log2) { return l != l && fabsf(m * scale_log2) < 0x1p24f; }
// Whether sums of rows that see all n values stand, finite or not: each value is below 2^88, so that 2^30 of them with weights of up
// to 256 stay in the range, or not finite, and then no infinity of the first key if that fills up a tile.  A wavefront, lane l coordinates l, l + 64.
constexpr float VALUES_ADD_UP = 0x1p88f;
template <typename T, int D>
__device__ __forceinline__ bool sums_stand(const char *V, int64_t pitch, int n, bool filled) {
    const int lane = lane_id();
    bool bad = false;
    for (int j = 0; j < n; ++j)
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            const float x = fabsf((float)((const T *)(V + (int64_t)j * pitch))[64 * c + lane]);
            bad |= x < INFINITY ? x >= VALUES_ADD_UP : j == 0 && filled && x == INFINITY;
        }
    return !__any(bad);
}

// One row over the keys first .. seen - 1, a wavefront: what tiles whose sums are not finite fall back to.  The maximum and the sum of
// the weights come first, so that values are taken with weights that add up to one and their sum stays where the values are; a
// key per lane for the scores, then lane l coordinates l, l + 64 for the values.  score(j, q): q.k of key j by this lane, which no
// other lane shares, or -inf; value(j, c): coordinate 64 c + lane of key j; seen_at(j): whether uniform key j has a value.
template <int D, class Score, class Seen, class Value>
__device__ __forceinline__ void row_again(int first, int seen, float scale_log2, Score score, Seen seen_at, Value value, float &m, float &l,
                                          float (&o)[D / 64]) {
    const int lane = lane_id();
    m = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) o[c] = 0.0f;
    auto scored = [&](int j0) __attribute__((always_inline)) {   // all lanes together: they hold the query's coordinates
        const float x = score(min(j0 + lane, seen - 1));
        return j0 + lane < seen ? x : -INFINITY;
    };
    for (int j0 = first; j0 < seen; j0 += 64) {
        const float x = scored(j0);
        float mn = fmaxf(m, x);
#pragma unroll
        for (int i = 32; i > 0; i >>= 1) mn = fmaxf(mn, shfl_xor(mn, i));
        l = l * (m == -INFINITY ? 0.0f : exp2f((m - mn) * scale_log2)) + exp2f((x - (mn == -INFINITY ? 0.0f : mn)) * scale_log2);
        m = mn;
        if (__any(l != l)) break;   // and stays so
    }
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) l += shfl_xor(l, i);
    if (l != l) {
#pragma unroll
        for (int c = 0; c < D / 64; ++c) o[c] = l;
        return;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l, m0 = m == -INFINITY ? 0.0f : m;
    for (int j0 = first; j0 < seen; j0 += 64) {
        const float w = exp2f((scored(j0) - m0) * scale_log2) * inv;
        for (int j = j0; j < min(j0 + 64, seen); ++j) {
            if (!seen_at(j)) continue;
            const float wj = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(w), j - j0));
#pragma unroll
            for (int c = 0; c < D / 64; ++c) o[c] = fmaf(wj, value(j, c), o[c]);
        }
    }
}
// The query's coordinate 64 h + i of lane i's qv[h].
__device__ __forceinline__ float of_lane(float x, int i) { return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(x), i)); }

template <typename T, int D>
__device__ __forceinline__ void row_by_keys(const char *q, const char *K, int64_t k_pitch, const char *V, int64_t v_pitch, int seen,
                                            float scale_log2, float &m, float &l, float (&o)[D / 64]) {
    constexpr int E = 16 / sizeof(T);
    typedef __attribute__((ext_vector_type(E))) T Chunk;
    const int lane = lane_id();
    float qv[D / 64];
#pragma unroll
    for (int c = 0; c < D / 64; ++c) qv[c] = (float)((const T *)q)[64 * c + lane];
    row_again<D>(
        0, seen, scale_log2,
        [&](int j) __attribute__((always_inline)) {
            const Chunk *kp = (const Chunk *)(K + (int64_t)j * k_pitch);
            float x = 0.0f;
#pragma unroll
            for (int h = 0; h < D / 64; ++h)
                for (int i = 0; i < 64; i += E) {
                    const Chunk k = kp[(64 * h + i) / E];
#pragma unroll
                    for (int e = 0; e < E; ++e) x = fmaf(of_lane(qv[h], i + e), (float)k[e], x);
                }
            return x;
        },
        [](int) { return true; }, [&](int j, int c) __attribute__((always_inline)) { return (float)((const T *)(V + (int64_t)j * v_pitch))[64 * c + lane]; }, m, l, o);
}

}  // namespace fastar
