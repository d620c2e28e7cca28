// Norm and rotation of a row: what qk_norm_rope and kv_pages_write_rope share, so that both compute the same numbers.
//   y = x (mean x^2 + eps)^-1/2 w;   pair (a, b) of coordinates -> (a cos t - b sin t, a sin t + b cos t), t = pos * freq
// A row is d / 8 neighbouring lanes with two pieces of four coordinates each, rot / 2 apart where pairs are, so that every lane has both
// coordinates of its four pairs and none are exchanged.  (Eight neighbouring coordinates per lane, swapped with the lane of the other
// half before and after, took 176 vector instructions per lane and row where this takes 75, which was most of the time: 34612 tokens x 40 heads 100 us of 134.)
#pragma once

#include "packed.hpp"

namespace fastar {

// fastar_rope and the positions, as the kernels take them.
struct RopeArgs {
    const double *freq;
    const int32_t *axis, *pos, *cu, *len;
    const float *qw, *kw;
    float eps;
    int32_t norm, rot, n_axes, B, n_tok;
};
int rope_check(const fastar_rope *r, const int32_t *pos, const int32_t *cu, const int32_t *len, int B, int n_tok, int d);
RopeArgs rope_args(const fastar_rope *r, const int32_t *pos, const int32_t *cu, const int32_t *len, int B, int n_tok);
int rope_parts(int n_tok, int Hq, int Hkv, int d);

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
__device__ __forceinline__ float row_max(float v) {   // of numbers that are not negative, by their bits: what is not finite comes out on top
    unsigned u = __float_as_uint(v);
    u = max(u, lane_of_eight<0>(u));
    u = max(u, lane_of_eight<1>(u));
    u = max(u, lane_of_eight<2>(u));
    if constexpr (LPR == 16) u = max(u, (unsigned)__builtin_amdgcn_update_dpp(0, (int)u, 0x140, 0xF, 0xF, false));
    return __uint_as_float(u);
}

// Sequences of a call, a lane each: their offsets and lengths are asked for at once, so that a wavefront waits for one trip to memory while there are
// no more than 64, and for one more for every factor of 64.
struct Places {
    int begin, end, len;
};
// Whether a row t is a sequence's, how far ahead of t its position is where that goes by the sequence's length, and where the sequence ends.
struct Place {
    bool there;
    int ahead, end;
};
// Differences and sums of lengths that are the caller's, whatever they are.
__device__ __forceinline__ int less(int a, int b) { return (int)((unsigned)a - (unsigned)b); }
__device__ __forceinline__ int plus(int a, int b) { return (int)((unsigned)a + (unsigned)b); }
__device__ __forceinline__ Places places_from(const RopeArgs &r, int lo, int n) {
    const int b = lo + min(lane_id(), n - 1);   // lanes beyond the sequences repeat the last one
    return Places{r.cu[b], r.cu[b + 1], r.rot > 0 && !r.pos ? r.len[b] : 0};
}
__device__ __forceinline__ Places places_of(const RopeArgs &r) { return !r.cu || r.B > 64 ? Places{0, 0, 0} : places_from(r, 0, r.B); }
__device__ __forceinline__ Place place_of(const RopeArgs &r, Places p, int t) {
    if (!r.cu) return Place{true, 0, r.n_tok};
    if (r.B > 64) {
        int lo = 0, n = r.B;   // t is a row of sequences lo .. lo + n - 1, if of any
        while (n > 64) {       // uniform; every step leaves a 64th
            const int step = (n + 63) / 64;
            const long long j = (long long)(lane_id() + 1) * step;
            const bool passed = j < n && r.cu[lo + j] <= t;
            const int c = __builtin_popcountll(__ballot(passed));
            lo += c * step;
            n = min(step, n - c * step);
        }
        p = places_from(r, lo, n);
    }
    const unsigned long long here = __ballot(p.begin <= t && t < p.end);
    if (!here) return Place{false, 0, 0};
    const int l = __builtin_ctzll(here), end = min(__builtin_amdgcn_readlane(p.end, l), r.n_tok);
    return Place{true, less(__builtin_amdgcn_readlane(p.len, l), end), end};
}

// What a lane needs of the rotation: its pieces' first coordinates, its pairs' frequencies in turns per position (0: they do not turn).
// INTER: pairs lie side by side.
struct RopeLane {
    int a, b;
    double freq[4];
    int axis[4];
    bool turn_a, turn_b;   // whether the piece's coordinates turn
};
template <int D, bool INTER>
__device__ __forceinline__ RopeLane rope_lane(const RopeArgs &r) {
    constexpr int LPR = D / 8;
    RopeLane l;
    const int i = lane_id() % LPR, half = INTER ? LPR : r.rot / 8;   // lanes with both coordinates of pairs
    l.a = 4 * (i < half ? i : half + i);
    l.b = 4 * (i < half ? i + half : LPR + i);
    l.turn_a = l.a < r.rot;
    l.turn_b = l.b < r.rot;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int pair = INTER ? (j < 2 ? l.a / 2 + j : l.b / 2 + j - 2) : l.a + j;
        const bool turns = INTER && j >= 2 ? l.turn_b : l.turn_a;
        l.freq[j] = turns ? r.freq[pair] * 0.15915494309189533577 : 0.0;   // 1 / (2 pi)
        l.axis[j] = turns && r.axis && r.pos ? min(max(r.axis[pair], 0), r.n_axes - 1) : 0;
    }
    return l;
}
// The angles of a lane's pairs at a row.  Positions times frequencies in 64 bits, of which the part of a turn is kept: at position
// 200000 a product in 32 bits is off by 0.01.  (64-bit arithmetic has the rate of unpacked 32-bit arithmetic here.)  The instructions for sine and
// cosine take turns.  They are within 2^-22.92 of those of their operand (2^26 at random, small sines within 2^-20 of themselves), with the operand's rounding to 32 bits within
// 2^-22.36; the bound of both is 2^-22.1.  That is a choice: quarter turns taken off in 64 bits and polynomials on the rest would make the error of fp32 outputs 6.4e-8 of their
// norm, where it is 7.7 to 8.6e-8 (the plain form's in fp32 7e-8), at no cost to qk_norm_rope in fp32 (28.9 us and 28.8); but keys on their way into pages, whose angles are
// computed for every head, would take 102 us instead of 74 (34612 tokens x 8 heads; rows one after the other, so that none spill, 94), for codes of four bits, and both
// calls write the same bits.
struct Turn {
    float c[4], s[4];
};
struct Fractions {   // of a turn, of a lane's pairs
    float f[4];
    __device__ __forceinline__ Turn turn() const {
        Turn t;
#pragma unroll
        for (int i = 0; i < 4; ++i) t.s[i] = __builtin_amdgcn_sinf(f[i]), t.c[i] = __builtin_amdgcn_cosf(f[i]);
        return t;
    }
};
__device__ __forceinline__ float fraction(const RopeLane &l, int i, int pos) {
    const double x = (double)pos * l.freq[i];
    return (float)(x - __builtin_rint(x));
}
__device__ __forceinline__ Fractions fractions(const RopeLane &l, int pos) {   // one position on every axis
    return Fractions{fraction(l, 0, pos), fraction(l, 1, pos), fraction(l, 2, pos), fraction(l, 3, pos)};
}
__device__ __forceinline__ Fractions fractions(const RopeArgs &r, const RopeLane &l, int t) {   // those of row t
    int p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = r.pos[(size_t)l.axis[i] * r.n_tok + t];
    return Fractions{fraction(l, 0, p[0]), fraction(l, 1, p[1]), fraction(l, 2, p[2]), fraction(l, 3, p[3])};
}
// A lane's weights.
struct Weights {
    float w[8];
    __device__ __forceinline__ void load(const float *p, const RopeLane &l) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = p ? p[l.a + e] : 1.0f, w[4 + e] = p ? p[l.b + e] : 1.0f;
    }
    // Whether some of the row's weights are so large that a normed coordinate times them may leave the range, or are no numbers.  A coordinate that does not
    // turn goes through the turn with c = 1, s = 0 like any other, where its lane's other coordinate times 0 has to be 0; so every row is then done as
    // norm_and_turn_odd does it.  The same in all lanes, as a row is done again as a whole (an output may be its input).
    __device__ __forceinline__ bool wild() const {
        unsigned top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(fabsf(w[e])));
        return __any(top >= __float_as_uint(0x1p100f));
    }
};
template <int D>
__device__ __forceinline__ float squares(const float (&x)[8]) {
    float ss = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
    return row_sum<D / 8>(ss);
}
// 1 / sqrt(mean + eps): one step from the instruction's approximation.
template <int D>
__device__ __forceinline__ float inverse_root(float ss, float eps) {
    const float v = fmaf(ss, 1.0f / D, eps), q = __builtin_amdgcn_rsqf(v);
    return fmaf(0.5f * q, fmaf(-v * q, q, 1.0f), q);
}
// x inv w turned; pairs that do not turn have c = 1, s = 0.
template <bool INTER>
__device__ __forceinline__ void turned(const Turn &t, const Weights &w, float inv, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int ia = INTER ? 2 * i : i, ib = INTER ? 2 * i + 1 : 4 + i;
        const float a = x[ia] * inv * w.w[ia], b = x[ib] * inv * w.w[ib];
        x[ia] = fmaf(a, t.c[i], -(b * t.s[i]));
        x[ib] = fmaf(a, t.s[i], b * t.c[i]);
    }
}
// A lane's eight coordinates of a row: normed and turned, all lanes of a row together.  Not of rows whose squares leave the range (upwards or, where eps does
// not rule them, downwards) or that hold infinities or NaN: those come back true, and are done again by norm_and_turn_odd.
template <int D, bool INTER>
__device__ __forceinline__ bool norm_and_turn(const RopeArgs &r, const Turn &t, const Weights &w, float (&x)[8]) {
    const float ss = squares<D>(x);
    const bool odd = !(ss >= (r.norm && r.eps < 0x1p-80f ? 0x1p-80f : 0.0f) && ss < 0x1p120f);
    turned<INTER>(t, w, r.norm ? inverse_root<D>(ss, r.eps) : 1.0f, x);
    return odd;
}
// The same of any row.  The row and the root of eps are taken times a power of two that brings the larger one near 1, after which the squares add up in 32 bits
// as any row's do; without a finite number but zero to bring there, what the formula gives.  Coordinates that do not turn are kept apart, as 0 times infinity is no number.
template <int D, bool INTER>
__device__ __forceinline__ void norm_and_turn_odd(const RopeArgs &r, const RopeLane &l, const Turn &t, const Weights &w, float (&x)[8]) {
    float inv = 1.0f;
    if (r.norm) {
        unsigned m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(fabsf(x[e])));
        const float most = row_max<D / 8>(__uint_as_float(m)), top = most < INFINITY ? fmaxf(most, sqrtf(r.eps)) : most;
        if (top < INFINITY) {
            const int n = top > 0.0f ? -__builtin_amdgcn_frexp_expf(top) : 0;   // top * 2^n is in [1/2, 1)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_ldexpf(x[e], n);
            inv = inverse_root<D>(squares<D>(x), __builtin_amdgcn_ldexpf(__builtin_amdgcn_ldexpf(r.eps, n), n));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = top == INFINITY && fabsf(x[e]) < INFINITY ? 0.0f : NAN;
        }
    }
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = r.norm ? x[e] * inv * w.w[e] : x[e];
    turned<INTER>(t, w, inv, x);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (!(e < 4 ? l.turn_a : l.turn_b)) x[e] = z[e];
}

// A lane's two pieces as they lie in memory.
template <bool BF16>
struct Raw8 {
    static constexpr int W = BF16 ? 2 : 4;
    typedef __attribute__((ext_vector_type(W))) unsigned Piece;
    Piece a, b;
    __device__ __forceinline__ void load(const char *row, const RopeLane &l) {
        a = *(const Piece *)(row + l.a * (BF16 ? 2 : 4));
        b = *(const Piece *)(row + l.b * (BF16 ? 2 : 4));
    }
    __device__ __forceinline__ void load(const char *base, unsigned row, const RopeLane &l) {   // from a uniform base
        a = *(const Piece *)(base + (row + (unsigned)l.a * (BF16 ? 2 : 4)));
        b = *(const Piece *)(base + (row + (unsigned)l.b * (BF16 ? 2 : 4)));
    }
    __device__ __forceinline__ void to(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (BF16) {
                x[e] = e & 1 ? bf16_hi(a[e / 2]) : bf16_lo(a[e / 2]);
                x[4 + e] = e & 1 ? bf16_hi(b[e / 2]) : bf16_lo(b[e / 2]);
            } else {
                x[e] = __uint_as_float(a[e]);
                x[4 + e] = __uint_as_float(b[e]);
            }
        }
    }
    static __device__ __forceinline__ void store(char *row, const RopeLane &l, const float (&x)[8]) {
        Piece u, v;
        if constexpr (BF16) {
            u = Piece{cvt_bf16x2(x[0], x[1]), cvt_bf16x2(x[2], x[3])};
            v = Piece{cvt_bf16x2(x[4], x[5]), cvt_bf16x2(x[6], x[7])};
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = __float_as_uint(x[e]), v[e] = __float_as_uint(x[4 + e]);
        }
        *(Piece *)(row + l.a * (BF16 ? 2 : 4)) = u;
        *(Piece *)(row + l.b * (BF16 ? 2 : 4)) = v;
    }
};

// Groups of 64 / (d / 8) heads of one token, first, first + step, .. of those of queries and then keys.  A wavefront together: the token's angles
// are computed once for all of them, and AHEAD groups are asked for ahead.  At most ROPE_GROUPS groups.
constexpr int ROPE_GROUPS = 32;
struct RopeViews {
    View q, k, qo, ko;
    int Hq, Hkv;
};
template <int D>
__host__ __device__ __forceinline__ int rope_groups(int H) { return (int)(((long long)H + 512 / D - 1) / (512 / D)); }
template <bool BF16, int D, bool INTER, int AHEAD>
__device__ __forceinline__ void rope_token(const RopeArgs &r, const RopeViews &a, int t, int first, int step) {
    constexpr int LPR = D / 8, RPW = 64 / LPR;
    const int lr = lane_id() / LPR;
    const int gq = rope_groups<D>(a.Hq), n = gq + rope_groups<D>(a.Hkv);
    const Places places = places_of(r);
    const RopeLane rl = rope_lane<D, INTER>(r);
    Fractions at{};
    if (r.rot > 0 && r.pos) at = fractions(r, rl, t);
    auto weights_of = [&](bool is_k) __attribute__((always_inline)) {
        Weights w;
        w.load(r.norm ? is_k ? r.kw : r.qw : nullptr, rl);
        return w;
    };
    const bool first_k = first >= gq;
    Weights w = weights_of(first_k);
    Raw8<BF16> raw[AHEAD];
    auto ask = [&](int g, Raw8<BF16> &x) __attribute__((always_inline)) {
        const bool is_k = g >= gq;
        const int h = (is_k ? g - gq : g) * RPW + lr;
        const char *p = (is_k ? a.k.p : a.q.p) + t * (is_k ? a.k.row : a.q.row);
        if (h < (is_k ? a.Hkv : a.Hq)) x.load(p + h * (is_k ? a.k.head : a.q.head), rl);
        else x.a = 0, x.b = 0;
    };
    auto put = [&](int g, bool mine, const float (&x)[8]) __attribute__((always_inline)) {
        const bool is_k = g >= gq;
        const int h = (is_k ? g - gq : g) * RPW + lr;
        char *p = (is_k ? a.ko.p : a.qo.p) + t * (is_k ? a.ko.row : a.qo.row);
        if (mine && h < (is_k ? a.Hkv : a.Hq)) Raw8<BF16>::store(p + h * (is_k ? a.ko.head : a.qo.head), rl, x);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (first + i * step < n) ask(first + i * step, raw[i]);
    const Place place = place_of(r, places, t);
    if (!place.there) return;
    bool wild = w.wild();
    if (r.rot > 0 && !r.pos) at = fractions(rl, plus(place.ahead, t));
    const Turn turn = at.turn();
    bool keys = first_k;
    unsigned odds = 0;   // bit i: the lane's row of the wavefront's i-th group is to be done again
    int i0 = 0;
    for (int g0 = first; g0 < n; g0 += AHEAD * step, i0 += AHEAD)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int g = g0 + i * step;
            if (g >= n) break;   // uniform
            if (g >= gq && !keys) {
                keys = true;
                w = weights_of(true);
                wild = w.wild();
            }
            float x[8];
            raw[i].to(x);
            if (g + AHEAD * step < n) ask(g + AHEAD * step, raw[i]);
            const bool odd = norm_and_turn<D, INTER>(r, turn, w, x) || wild;
            put(g, !odd, x);
            odds |= odd ? 1u << (i0 + i) : 0u;
        }
    if (!__any(odds)) return;
#pragma unroll 1
    for (int i = 0, g = first; g < n; ++i, g += step) {   // the others' rows are left out: an output may be its input
        if (!__any(odds >> i & 1)) continue;
        float x[8];
        ask(g, raw[0]);
        raw[0].to(x);
        w = weights_of(g >= gq);
        norm_and_turn_odd<D, INTER>(r, rl, turn, w, x);
        put(g, odds >> i & 1, x);
    }
}

// qk_norm_rope's launch (rope.hip).
int rope_launch(const RopeArgs &r, const RopeViews &v, int d, int dtype, int interleaved, hipStream_t s);

}  // namespace fastar
