// What the calls that write new keys and values into pages share (kv_pages_write, kv_pages_write_rope).
#pragma once

#include "rope_dev.hpp"

namespace fastar {

int pages_check(const fastar_pages *pg);

namespace pages {

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

typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
typedef __attribute__((ext_vector_type(2))) short s16x2;

// EPL consecutive elements of a row as they lie in memory.
template <bool BF16, int EPL>
struct Piece {
    static constexpr int W = EPL * (BF16 ? 2 : 4) / 4;
    unsigned w[W];
    __device__ __forceinline__ void load(const char *p) {
        if constexpr (W == 1) {
            w[0] = *(const unsigned *)p;
        } else if constexpr (W == 2) {
            const u32x2 x = *(const u32x2 *)p;
            w[0] = x[0], w[1] = x[1];
        } else {
#pragma unroll
            for (int q = 0; q < W / 4; ++q) {
                const u32x4 x = ((const u32x4 *)p)[q];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[4 * q + e] = x[e];
            }
        }
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (BF16) return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
        else return __uint_as_float(w[i]);
    }
    // Largest |x| by its bits, with what `top` holds (two 16-bit maxima for bf16): numbers that are not finite come out on top.
    __device__ __forceinline__ unsigned top(unsigned top) const {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (BF16) top = __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu)));
            else top = max(top, w[i] & 0x7FFFFFFFu);
        }
        return top;
    }
    // Codes of elements i, i + 1, in the lower or the upper half of r: the conversion instructions divide by a power of two and round
    // to nearest, ties to even (what goes beyond 464 becomes no number; here nothing goes beyond 448).
    template <bool UPPER>
    __device__ __forceinline__ void codes(int i, float scale, unsigned &r) const {
        const s16x2 old = __builtin_bit_cast(s16x2, r);
        if constexpr (BF16) r = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, __builtin_bit_cast(bf16x2, w[i / 2]), scale, UPPER));
        else r = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(old, (*this)[i], (*this)[i + 1], scale, UPPER));
    }
};
// Codes carried over to a scale 1 / ratio times as large.
__device__ __forceinline__ unsigned rescaled(unsigned w, float ratio) {
    return f8_of(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * ratio,
                 __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * ratio);
}
__device__ __forceinline__ float wave_max(float x) {   // of numbers that are not negative
    return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)wave_max_last(__float_as_uint(x)), 63));
}
// Rows o .. e - 1 of a page where some number is not finite, one after the other.
template <bool BF16, int D>
__device__ __forceinline__ void write_odd_run(const char *row0, int64_t pitch, int o, int e, bool is_v, uint8_t *cell0, int page_bytes,
                                              float old_scale, float *scale_out) {
    const int lane = threadIdx.x & 63;
    auto at = [&](int r, int c) {
        const char *p = row0 + r * pitch;
        if constexpr (BF16) return bf16_bits_to_f32(((const unsigned short *)p)[c]);
        else return ((const float *)p)[c];
    };
    float amax = 0.0f;
    for (int r = o; r < e; ++r)
        for (int c = lane; c < D; c += 64) amax = fmaxf(amax, finite_abs(at(r, c)));
    const float scale = fmaxf(pow2(scale_exp(wave_max(amax))), old_scale), inv = 1.0f / scale, ratio = old_scale * inv;
    if (o > 0 && ratio < 1.0f) {
        for (int i = lane; i < page_bytes / 4; i += 64) ((unsigned *)cell0)[i] = rescaled(((unsigned *)cell0)[i], ratio);
        __threadfence();   // before other lanes' new codes go to the same words
    }
    for (int r = o; r < e; ++r)
        for (int c = lane; c < D; c += 64) {
            const float x = at(r, c) * inv;
            cell0[((r >> 4) * (D / 16) + (c >> 4)) * 256 + (is_v ? (c & 15) * 16 + (r & 15) : (r & 15) * 16 + (c & 15))] = (uint8_t)f8_of(x, x, x, x);
        }
    if (lane == 0) *scale_out = scale;
}

// Rows per workgroup: a page's where that makes enough of them; fewer, down to one, so that the runs of single tokens are not
// done one after the other.  At least 1024 / 4096 / 16384 workgroups, pages of 64, 8 heads: 512 single tokens 17.5 / 19.4 / 21.7 us, 16 runs
// of 16 4.5 / 6.0 / 6.0, 8 of 200 6.3 / 9.2 / 18.6, 8 of 4680 38.6 / 37.4 / 52; 30000 tokens of one head 9.5 / 23 / 49: for runs fewer would do
// (`least` says so where that is known).
inline int rows_per_workgroup(int n_tok, int Hkv, int P, int least = 4096) {
    int chunk = P;
    while (chunk > 1 && (int64_t)n_tok * Hkv * 2 / chunk < least) chunk /= 2;
    return chunk;
}

// Rows of one page that follow one another in the order of their slots.
struct Run {
    const char *row0;    // where a row of offset 0 would be
    int64_t pitch;
    int o, e;            // offsets of the first row and behind the last
    uint8_t *page0;      // the page's codes of this head
    float *scale;        // its scale, and what that was (0 where the page is begun anew)
    float old_scale;
};
// The runs that begin among rows first .. first + chunk - 1 (at most 64), one after the other, for a workgroup together: f(row, slot, rows, turn).
// Rows outside of [t_lo, t_hi) have no slot.
template <int PSHIFT, class F>
__device__ __forceinline__ void for_runs(const int32_t *__restrict__ slot, int n_tok, int first, int chunk, unsigned n_slots, int t_lo, int t_hi, F f) {
    constexpr int P = 1 << PSHIFT;
    const int lane = threadIdx.x & 63;
    // rows first - 1 .. first + 127: which are valid, and which go on where the row before them ended
    auto at = [&](int t) {
        const int s = t >= 0 && t < n_tok ? slot[t] : -1;
        return t >= t_lo && t < t_hi ? s : -1;
    };
    const int s0 = at(first + lane), s1 = at(first + 64 + lane);
    const int s_before = at(first - 1);
    const bool ok0 = (unsigned)s0 < n_slots, ok1 = (unsigned)s1 < n_slots;
    int p0 = __shfl_up(s0, 1, 64), p1 = __shfl_up(s1, 1, 64);   // all lanes together: a lane that is not there gives nothing
    if (lane == 0) {
        p0 = s_before;
        p1 = __builtin_amdgcn_readlane(s0, 63);
    }
    const unsigned long long valid = __ballot(ok0);
    const unsigned long long go0 = __ballot(ok0 && (s0 & (P - 1)) && p0 == s0 - 1), go1 = __ballot(ok1 && (s1 & (P - 1)) && p1 == s1 - 1);
    unsigned long long begin = valid & ~go0;
    if (chunk < 64) begin &= (1ull << chunk) - 1ull;
    for (int turn = 0; begin; begin &= begin - 1ull, turn ^= 1) {   // uniform over the workgroup
        const int pos = __builtin_ctzll(begin);
        const unsigned long long after = pos == 63 ? go1 : (go0 >> (pos + 1)) | (go1 << (63 - pos));   // bit i: row pos + 1 + i goes on
        const int n = 1 + (~after ? __builtin_ctzll(~after) : 63);   // at most P: a run ends with its page
        f(first + pos, __builtin_amdgcn_readlane(s0, pos), n, turn);
    }
}
// The largest of the workgroup's NW wavefronts' maxima; the other half of `s_top` is free by the next call.
template <int NW>
__device__ __forceinline__ unsigned top_of(unsigned top, unsigned (*s_top)[NW], int turn) {
    top = (unsigned)__builtin_amdgcn_readlane((int)wave_max_last(top), 63);
    if constexpr (NW > 1) {
        if ((threadIdx.x & 63) == 0) s_top[turn][threadIdx.x >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NW; ++i) top = max(top, s_top[turn][i]);
    }
    return top;
}
constexpr unsigned NOT_FINITE = 0x7F800000u;   // maxima from here on are of rows that hold a number that is not finite

// K, a wavefront for 16 rows: 16 bytes of bf16 per lane and row, whose codes are half of a cell's 16 bytes, exchanged between neighbouring lanes.
template <bool BF16, int D, int PSHIFT>
__device__ __forceinline__ void k_run(const Run &run, unsigned (*s_top)[1 << PSHIFT >> 4], int turn) {
    constexpr int P = 1 << PSHIFT, ELT = BF16 ? 2 : 4, NW = P / 16;
    constexpr int LPR = D / 8, RPI = 64 / LPR, IT = 16 / RPI;   // row i RPI + lr, coordinates 8 lc ..
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane / LPR, lc = lane % LPR;
    const int r0 = 16 * wave, o = run.o, e = run.e;
    const bool touches = r0 < e && r0 + 16 > o;   // rows of the run among the wavefront's 16
    uint8_t *blk = run.page0 + wave * (16 * D);
    auto row_of = [&](int r) { return run.row0 + (unsigned)min(max(r0 + r, o), e - 1) * (unsigned)run.pitch; };   // rows beside the run: one of its own again
    Piece<BF16, 8> k[IT];
    unsigned top = 0;
    if (touches) {
#pragma unroll
        for (int i = 0; i < IT; ++i) k[i].load(row_of(i * RPI + lr) + lc * 8 * ELT);
#pragma unroll
        for (int i = 0; i < IT; ++i) top = k[i].top(top);
    }
    if constexpr (BF16) top = max(top & 0xFFFFu, top >> 16) << 16;
    top = top_of<NW>(top, s_top, turn);
    if (top >= NOT_FINITE) {
        if (wave == 0) write_odd_run<BF16, D>(run.row0, run.pitch, o, e, false, run.page0, D * P, run.old_scale, run.scale);
        return;
    }
    const float scale = fmaxf(pow2(scale_exp(__uint_as_float(top))), run.old_scale), ratio = run.old_scale / scale;
    const bool grows = o > 0 && ratio < 1.0f;
    if (lane == 0 && wave == 0) *run.scale = scale;
    if (!touches && !grows) return;
    u32x2 c[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        unsigned w0 = 0, w1 = 0;
        k[i].template codes<false>(0, scale, w0);
        k[i].template codes<true>(2, scale, w0);
        k[i].template codes<false>(4, scale, w1);
        k[i].template codes<true>(6, scale, w1);
        c[i] = u32x2{w0, w1};
    }
#pragma unroll
    for (int i = 0; i < IT; i += 2) {   // even lanes take row i of the pair's cell, odd ones row i + 1
        const bool odd = lane & 1;
        const u32x2 give = odd ? c[i] : c[i + 1], keep = odd ? c[i + 1] : c[i];
        const u32x2 got = {lane_of_eight<0>(give[0]), lane_of_eight<0>(give[1])};
        const int r = (i + (odd ? 1 : 0)) * RPI + lr;
        u32x4 y = odd ? u32x4{got[0], got[1], keep[0], keep[1]} : u32x4{keep[0], keep[1], got[0], got[1]};
        u32x4 *p = (u32x4 *)(blk + (lc >> 1) * 256 + r * 16);
        const bool mine = r0 + r >= o && r0 + r < e;
        if (!mine && grows) {
            y = *p;
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = rescaled(y[q], ratio);
        }
        if (mine || grows) *p = y;
    }
}

// V, a wavefront for 16 rows: two coordinates of every row per lane, whose codes over the rows are 32 consecutive bytes of the page (d = 64: twice 8).
template <bool BF16, int D, int PSHIFT>
__device__ __forceinline__ void v_run(const Run &run, unsigned (*s_top)[1 << PSHIFT >> 4], int turn) {
    constexpr int P = 1 << PSHIFT, ELT = BF16 ? 2 : 4, NW = P / 16;
    constexpr int VL = D / 2, VR = 16 * VL / 64;   // rows VR g .., coordinates 2 c
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), vc = lane % VL, vg = lane / VL;
    const int r0 = 16 * wave, o = run.o, e = run.e;
    const bool touches = r0 < e && r0 + 16 > o, all = r0 >= o && r0 + 16 <= e;   // rows of the run among the wavefront's 16
    uint8_t *blk = run.page0 + wave * (16 * D);
    auto row_of = [&](int r) { return run.row0 + (unsigned)min(max(r0 + r, o), e - 1) * (unsigned)run.pitch; };
    Piece<BF16, 2> v[VR];
    u32x2 old[4];   // what is there of a block that the run covers in part
    u32x2 *vp = (u32x2 *)(blk + vc * 32 + vg * VR);   // a coordinate's VR bytes; the next one's are 16 bytes on
    auto vword = [&](int i) -> u32x2 & { return D == 128 ? vp[i] : vp[2 * i]; };   // 8 bytes: D = 128: two per coordinate
    constexpr int VW = VR / 4;   // such words: 4 or 2
    unsigned top = 0;
    if (touches) {
#pragma unroll
        for (int i = 0; i < VR; ++i) v[i].load(row_of(vg * VR + i) + vc * 2 * ELT);
        if (!all) {
#pragma unroll
            for (int i = 0; i < VW; ++i) old[i] = vword(i);
        }
#pragma unroll
        for (int i = 0; i < VR; ++i) top = v[i].top(top);
    }
    if constexpr (BF16) top = max(top & 0xFFFFu, top >> 16) << 16;
    top = top_of<NW>(top, s_top, turn);
    if (top >= NOT_FINITE) {
        if (wave == 0) write_odd_run<BF16, D>(run.row0, run.pitch, o, e, true, run.page0, D * P, run.old_scale, run.scale);
        return;
    }
    const float scale = fmaxf(pow2(scale_exp(__uint_as_float(top))), run.old_scale), ratio = run.old_scale / scale;
    const bool grows = o > 0 && ratio < 1.0f;
    if (lane == 0 && wave == 0) *run.scale = scale;
    if (!touches && !grows) return;
    unsigned c[VR / 2];   // of rows 2 i, 2 i + 1: codes of the two coordinates
#pragma unroll
    for (int i = 0; i < VR / 2; ++i) {
        c[i] = 0;
        v[2 * i].template codes<false>(0, scale, c[i]);
        v[2 * i + 1].template codes<true>(0, scale, c[i]);
    }
    u32x2 y[VW];   // coordinate by coordinate, four rows a word
#pragma unroll
    for (int co = 0; co < 2; ++co)
#pragma unroll
        for (int q = 0; q < VR / 4; ++q)
            y[(co * (VR / 4) + q) / 2][(co * (VR / 4) + q) % 2] = __builtin_amdgcn_perm(c[2 * q + 1], c[2 * q], co ? 0x07050301u : 0x06040200u);
    if (!all) {
#pragma unroll
        for (int i = 0; i < VW; ++i) {
            u32x2 w = touches ? old[i] : vword(i);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (grows) w[j] = rescaled(w[j], ratio);
                const int row = r0 + vg * VR + ((2 * i + j) % (VR / 4)) * 4;   // of the word's first byte
                unsigned mask = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) mask |= row + b >= o && row + b < e ? 0xFFu << (8 * b) : 0u;
                w[j] = touches ? (y[i][j] & mask) | (w[j] & ~mask) : w[j];
            }
            y[i] = w;
        }
    }
    if constexpr (D == 128) {
        ((u32x4 *)vp)[0] = u32x4{y[0][0], y[0][1], y[1][0], y[1][1]};
        ((u32x4 *)vp)[1] = u32x4{y[2][0], y[2][1], y[3][0], y[3][1]};
    } else {
#pragma unroll
        for (int i = 0; i < VW; ++i) vword(i) = y[i];
    }
}

}  // namespace pages

}  // namespace fastar
