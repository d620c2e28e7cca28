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
inline bool scale_ok(float scale) { return scale > 0.0f && std::isfinite(scale * 1.4426950408889634f); }
inline bool page_size_ok(int P) { return P == 16 || P == 32 || P == 64; }

// Rows [first, first + n) of sequence b, inside [0, n_tok).
struct Rows {
    int first, n;
};
__device__ __forceinline__ Rows rows_of(const int32_t *__restrict__ cu, int b, int n_tok) {
    const int a = min(max(cu[b], 0), n_tok), e = min(max(cu[b + 1], 0), n_tok);
    return Rows{a, max(e - a, 0)};
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
