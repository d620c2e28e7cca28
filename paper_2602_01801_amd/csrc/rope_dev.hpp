// Norm and rotation of a row: what qk_norm_rope and kv_pages_write_rope share, so that both compute the same numbers.
//   y = x (mean x^2 + eps)^-1/2 w;   pair (a, b) of coordinates -> (a cos t - b sin t, a sin t + b cos t), t = pos * freq
// A row is eight coordinates per lane (one 16-byte load in bf16), d / 8 neighbouring lanes.  Every lane of the rotated part
// turns four pairs: interleaved ones lie in its own coordinates; where pairs are rot / 2 apart, the lanes of the lower and the
// upper half swap four coordinates before and after, so that no angle is computed twice within a row.
#pragma once

#include "packed.hpp"

namespace fastar {

// fastar_rope and the positions, as the kernels take them.
struct RopeArgs {
    const double *freq;
    const int32_t *axis, *pos, *cu, *len;
    const float *qw, *kw;
    float eps;
    int32_t norm, rot, interleaved, n_axes, B, n_tok;
};
int rope_check(const fastar_rope *r, const int32_t *pos, const int32_t *cu, const int32_t *len, int B, int n_tok, int d);
RopeArgs rope_args(const fastar_rope *r, const int32_t *pos, const int32_t *cu, const int32_t *len, int B, int n_tok);
int rope_launch(const fastar_rows *Q, const fastar_rows *K, const RopeArgs &r, int Hq, int Hkv, int d, int dtype, const fastar_rows *Qo,
                const fastar_rows *Ko, hipStream_t s);

// Sum over the LPR (8 or 16) neighbouring lanes of a row; every lane has the same bits, as each step adds the same two numbers.
template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
    v += __uint_as_float(lane_of_eight<0>(__float_as_uint(v)));
    v += __uint_as_float(lane_of_eight<1>(__float_as_uint(v)));
    v += __uint_as_float(lane_of_eight<2>(__float_as_uint(v)));
    if constexpr (LPR == 16) v += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x140, 0xF, 0xF, false));   // row_mirror
    return v;
}
template <int LPR>
__device__ __forceinline__ double row_sum(double v) {
#pragma unroll
    for (int o = 1; o < LPR; o *= 2) v += __shfl_xor(v, o, 64);
    return v;
}

// Sequence of row t, cu[0] <= t < cu[B]: the number of the offsets cu[1 ..] that are not beyond t.  A wavefront together, 64 offsets a round.
__device__ __forceinline__ int sequence_of(const int32_t *__restrict__ cu, int B, int t) {
    const int lane = lane_id();
    int lo = 0, n = B;
    while (n > 1) {   // uniform; n falls to ceil(n / 64)
        const int step = (n + 63) / 64;
        const long long j = (long long)(lane + 1) * step;
        const bool passed = j < n && cu[lo + j] <= t;
        const int c = __builtin_popcountll(__ballot(passed));
        lo += c * step;
        n = min(step, n - c * step);
    }
    return lo;
}

// What a lane needs of the rotation: its pairs and their frequencies in turns per position.
struct RopeLane {
    double freq[4];
    int axis[4];
    bool turns, lower;   // takes part; has the first coordinates of its pairs
    int partner;         // the lane it swaps with
};
template <int D>
__device__ __forceinline__ RopeLane rope_lane(const RopeArgs &a) {
    constexpr int LPR = D / 8;
    RopeLane r;
    const int lane = lane_id(), lc = lane % LPR, h = a.rot / 16;
    r.turns = lc < 2 * h;
    r.lower = lc < h;
    r.partner = !r.turns ? lane : r.lower ? lane + h : lane - h;
    const int p0 = a.interleaved ? 4 * lc : r.lower ? 8 * lc : 8 * (lc - h) + 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.freq[i] = r.turns ? a.freq[p0 + i] * 0.15915494309189533577 : 0.0;   // 1 / (2 pi)
        r.axis[i] = r.turns && a.axis && a.pos ? min(max(a.axis[p0 + i], 0), a.n_axes - 1) : 0;
    }
    return r;
}
// The angles of a lane's pairs at a row.  Positions times frequencies in 64 bits, of which the part of a turn is kept: at position
// 200000 a product in 32 bits is off by 0.01.
struct Turn {
    float c[4], s[4];
};
__device__ __forceinline__ Turn turn_of(const RopeLane &r, const double (&pos)[4]) {
    Turn t;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double x = pos[i] * r.freq[i];
        sincospif(2.0f * (float)(x - __builtin_rint(x)), &t.s[i], &t.c[i]);
    }
    return t;
}

// A lane's eight coordinates of a row with their weights: normed and turned.  All lanes of a row together.
template <int D>
__device__ __forceinline__ void norm_and_turn(const RopeArgs &a, const RopeLane &r, const Turn &t, const float (&w)[8], float (&x)[8]) {
    constexpr int LPR = D / 8;
    if (a.norm) {
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
        ss = row_sum<LPR>(ss);
        // squares that leave the range of 32 bits, upwards or, where eps does not rule them, downwards
        const bool odd = !(ss < 0x1p120f) || (ss < 0x1p-80f && a.eps < 0x1p-80f);
        if (__any(odd)) {
            double s2 = 0.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) s2 = fma((double)x[e], (double)x[e], s2);
            s2 = row_sum<LPR>(s2);
            const double inv = 1.0 / sqrt(s2 * (1.0 / D) + (double)a.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = (float)((double)x[e] * inv);
                if (odd) x[e] = y * w[e];
            }
        }
        const float inv = 1.0f / sqrtf(fmaf(ss, 1.0f / D, a.eps));
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!odd) x[e] = x[e] * inv * w[e];
    }
    if (a.rot == 0) return;
    float p[4], q[4];   // pairs (p, q)
    if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = x[2 * i], q[i] = x[2 * i + 1];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float mine = r.lower ? x[i] : x[4 + i], got = __shfl(r.lower ? x[4 + i] : x[i], r.partner, 64);
            p[i] = r.lower ? mine : got;
            q[i] = r.lower ? got : mine;
        }
    }
    float u[4], v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u[i] = fmaf(p[i], t.c[i], -(q[i] * t.s[i]));
        v[i] = fmaf(p[i], t.s[i], q[i] * t.c[i]);
    }
    if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r.turns) x[2 * i] = u[i], x[2 * i + 1] = v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float keep = r.lower ? u[i] : v[i], got = __shfl(r.lower ? v[i] : u[i], r.partner, 64);
            if (r.turns) {
                x[i] = r.lower ? keep : got;
                x[4 + i] = r.lower ? got : keep;
            }
        }
    }
}

// A lane's eight coordinates from memory and back, in one or two 16-byte pieces.
template <bool BF16>
__device__ __forceinline__ void load8(const char *p, float (&x)[8]) {
    if constexpr (BF16) {
        const u32x4 w = *(const u32x4 *)p;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[2 * e] = bf16_lo(w[e]), x[2 * e + 1] = bf16_hi(w[e]);
    } else {
        const f32x4 u = ((const f32x4 *)p)[0], v = ((const f32x4 *)p)[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = u[e], x[4 + e] = v[e];
    }
}
template <bool BF16>
__device__ __forceinline__ void store8(char *p, const float (&x)[8]) {
    if constexpr (BF16) {
        *(u32x4 *)p = u32x4{cvt_bf16x2(x[0], x[1]), cvt_bf16x2(x[2], x[3]), cvt_bf16x2(x[4], x[5]), cvt_bf16x2(x[6], x[7])};
    } else {
        ((f32x4 *)p)[0] = f32x4{x[0], x[1], x[2], x[3]};
        ((f32x4 *)p)[1] = f32x4{x[4], x[5], x[6], x[7]};
    }
}

}  // namespace fastar
