// What the two kernels of attention over a paged cache share (paged_attn.hip, paged_chunk.hip): the call's arguments, and how the
// device deals out the work.
//
// The lengths are on the device, so the device deals out the work.  An item is a tile of R rows of one sequence and key head, a
// row being a (token, query head of the group) pair; heads that share keys share their loads.  The items' tiles of 64 keys, one
// item after the other, are cut into equal shares, a workgroup each.  A share that holds a part of an item leaves a fragment
// (sums, reference maxima, row sums) in the workspace, and a second launch puts the fragments of an item together.
#pragma once

#include "packed.hpp"

namespace fastar {

namespace paged {

constexpr int TK = 64;              // keys per tile
constexpr int MAX_SHARES = 512;
// Units of work of an item in front of its tiles: what its ends cost (queries, page numbers, first codes, sums put together), in tiles.
// Without them shares of many short sequences end last.  1 / 6 / 9 / 14 of them, tokens of 48 requests of 100 to 37440 keys 210 / 183 /
// 185 / 185 us, of 100 of 30 to 4000 57 / 38 / 39 / 39, of 20 of 10 to 20000 60 / 38.8 / 36.8 / 35.6, of 16 of 2100 24.2 / 22.6 / 21.1 / 22.9.
constexpr int ENDS = 9;

struct Desc {   // an item that was cut: its first share writes this
    int b, h, qt, last;   // last share that holds a part of it; -1: none
};
struct Args {
    View Q, O;
    const int32_t *cu_q, *len, *table;
    int B, max_pages, n_tok, group, causal, pshift;
    fastar_pages pg;
    float scale_log2;
    float *lse;
    Desc *desc;
    float *frag;
};
struct Seq {
    int q0, n_q, L, n_qt, n_tiles;
};
template <int R>
__device__ __forceinline__ Seq seq_from(const Args &a, int q0, int q1, int len) {
    Seq s;
    s.q0 = min(max(q0, 0), a.n_tok);
    s.n_q = max(min(max(q1, 0), a.n_tok) - s.q0, 0);
    s.L = min(max(len, 0), a.max_pages << a.pshift);
    s.n_qt = (s.n_q * a.group + R - 1) / R;
    s.n_tiles = max((s.L + TK - 1) / TK, 1);
    return s;
}
template <int R>
__device__ __forceinline__ Seq seq_of(const Args &a, int b) { return seq_from<R>(a, a.cu_q[b], a.cu_q[b + 1], a.len[b]); }
__device__ __forceinline__ bool page_exists(const Args &a, int id) { return (unsigned)id < (unsigned)a.pg.n_pages; }

__device__ __forceinline__ long long wave_incl_scan64(long long v) {
    const int lane = lane_id();
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
    }
    return v;
}
__device__ __forceinline__ long long readlane64(long long v, int lane) {
    return (long long)(unsigned)__builtin_amdgcn_readlane((int)v, lane) | ((long long)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32);
}

// Four sequences per lane from b0 on: every wavefront looks for itself, without a barrier.
template <int R, bool SPLIT>
struct Chunk {
    int cu[5], len[4], b0;
    long long n[4], all, upto;   // units of each (items if not SPLIT), their sum, and the inclusive sum over the lanes
    __device__ __forceinline__ void load(const Args &a, int first) {
        b0 = first + 4 * lane_id();
#pragma unroll
        for (int i = 0; i < 5; ++i) cu[i] = a.cu_q[min(b0 + i, a.B)];
#pragma unroll
        for (int i = 0; i < 4; ++i) len[i] = a.len[min(b0 + i, a.B - 1)];
        all = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Seq s = seq_from<R>(a, cu[i], cu[i + 1], len[i]);
            n[i] = (long long)s.n_qt * a.pg.Hkv * (SPLIT ? s.n_tiles + ENDS : 1);   // none beyond the last sequence: no rows
            all += n[i];
        }
        upto = wave_incl_scan64(all);
    }
    __device__ __forceinline__ long long total() const { return readlane64(upto, 63); }
    // The sequence that holds unit u of this chunk (counted from its first), if any: its number, its first unit, itself.
    __device__ __forceinline__ bool find(const Args &a, long long u, int &b, long long &base, Seq &s) const {
        const unsigned long long hit = __ballot(u >= upto - all && u < upto);
        if (!hit) return false;
        const int src = __builtin_ctzll(hit);
        long long start = upto - all;
        int i = 0;
        for (; i < 3; ++i) {
            if (u < start + n[i]) break;
            start += n[i];
        }
        auto pick = [&](const int *x) { return __builtin_amdgcn_readlane(i == 0 ? x[0] : i == 1 ? x[1] : i == 2 ? x[2] : x[3], src); };
        const int q0 = pick(cu), q1 = pick(cu + 1), l = pick(len);
        b = __builtin_amdgcn_readlane(b0 + i, src);
        base = readlane64(start, src);
        s = seq_from<R>(a, q0, q1, l);
        return true;
    }
};
template <int R, bool SPLIT>
__device__ __forceinline__ void find_unit(const Args &a, long long u, int &b, long long &base, Seq &s) {
    Chunk<R, SPLIT> c;
    long long before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 256) {   // uniform
        c.load(a, b0);
        if (c.find(a, u - before, b, base, s)) {
            base += before;
            return;
        }
        before += c.total();
    }
}
// The units in all, this workgroup's range of them and where it begins.  False: nothing to do.
struct Range {
    long long W, u, u_end, base;
    int share, n_shares, b;
};
template <int R, bool SPLIT>
__device__ __forceinline__ bool first_unit(const Args &a, int shares, int least, Range &r, Seq &s) {
    Chunk<R, SPLIT> c;
    c.load(a, 0);
    r.W = c.total();
    for (int b0 = 256; b0 < a.B; b0 += 256) {
        Chunk<R, SPLIT> more;
        more.load(a, b0);
        r.W += more.total();
    }
    if constexpr (SPLIT) {
        // a share holds `least` units at least; when all are used, neighbours go to the same XCD
        const long long n = (r.W + least - 1) / least;
        r.n_shares = (int)(n < shares ? n : shares);
        r.share = r.n_shares == shares ? (int)(blockIdx.x & 7) * (shares / 8) + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
        if (r.share >= r.n_shares) return false;
        r.u = r.W * r.share / r.n_shares;
        r.u_end = r.W * (r.share + 1) / r.n_shares;
    } else {
        r.n_shares = 0;
        r.share = blockIdx.x;
        r.u = r.share;
        r.u_end = r.u + 1;
        if (r.u >= r.W) return false;
    }
    if (!c.find(a, r.u, r.b, r.base, s)) find_unit<R, SPLIT>(a, r.u, r.b, r.base, s);
    return true;
}
// The next piece of an item: its tiles ta .. te - 1 (none if the share ends among the units before them).
struct PieceOf {
    int h, qt, ta, te;
    long long last;   // the item's last unit
};
template <bool SPLIT>
__device__ __forceinline__ PieceOf next_piece(Range &r, const Seq &s) {
    const int units = SPLIT ? s.n_tiles + ENDS : 1;
    const long long local = r.u - r.base;
    const int item = (int)(local / units);
    PieceOf p;
    p.h = item / s.n_qt;
    p.qt = item - p.h * s.n_qt;
    p.last = r.base + (long long)(item + 1) * units - 1;
    if constexpr (SPLIT) {
        const int from = (int)(local - (long long)item * units), to = (int)min((long long)units, from + (r.u_end - r.u));
        p.ta = max(from - ENDS, 0);
        p.te = to - ENDS;
        r.u += to - from;
    } else {
        p.ta = 0;
        p.te = s.n_tiles;
        r.u += 1;
    }
    return p;
}
// The last share that holds a part of an item whose last unit is x.
__device__ __forceinline__ int share_of(const Range &r, long long x) { return (int)(((x + 1) * r.n_shares + r.W - 1) / r.W) - 1; }

// Fragment i of the item that began in share `first`.
template <int FLOATS>
__device__ __forceinline__ float *fragment(const Args &a, int first, int i) {
    return a.frag + (size_t)(i == 0 ? 2 * first + 1 : 2 * (first + i)) * FLOATS;
}

// Weight of sums taken against reference m among those against m_all; a reference of -inf means sums of 0, or of no numbers.
__device__ __forceinline__ float weight_of(float m, float m_all, float scale_log2) {
    return m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - m_all) * scale_log2);
}

__device__ __forceinline__ bool finite(f32x4 x) { return fabsf(x[0]) < INFINITY && fabsf(x[1]) < INFINITY && fabsf(x[2]) < INFINITY && fabsf(x[3]) < INFINITY; }

// Eight codes times a power of two, exactly.
__device__ __forceinline__ bf16x8 widen(unsigned lo, unsigned hi, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    const bf16x8 r = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    return r;
}
// Which bytes of 16 consecutive tokens are among the first `live`.
__device__ __forceinline__ u32x4 first_bytes(int live) {
    u32x4 mask;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int n = min(max(live - 4 * e, 0), 4);
        mask[e] = n == 4 ? ~0u : (1u << (8 * n)) - 1u;
    }
    return mask;
}

// One row over keys first .. seen - 1 of its pages (see row_again).
template <int D>
__device__ __forceinline__ void row_by_paged_keys(const Args &a, const char *q, const int32_t *pages, int h, int first, int seen, float &m,
                                                  float &l, float (&o)[D / 64]) {
    const int lane = lane_id();
    float qv[D / 64];
#pragma unroll
    for (int c = 0; c < D / 64; ++c) qv[c] = (float)((const __bf16 *)q)[64 * c + lane];
    auto cell_of = [&](int page, int off) __attribute__((always_inline)) {   // first byte of the cells of a token's block of 16
        return ((size_t)page * a.pg.Hkv + h) * ((size_t)D << a.pshift) + (off >> 4) * (16 * D);
    };
    const int in_page = (1 << a.pshift) - 1;
    row_again<D>(
        first, seen, a.scale_log2,
        [&](int j) __attribute__((always_inline)) {
            const int id = pages[j >> a.pshift], page = page_exists(a, id) ? id : 0, off = j & in_page;
            const uint8_t *k8 = a.pg.K8 + cell_of(page, off) + (off & 15) * 16;
            float x = 0.0f;
            const float ks = a.pg.kscale[(size_t)page * a.pg.Hkv + h];
#pragma unroll
            for (int hh = 0; hh < D / 64; ++hh)
                for (int i = 0; i < 64; i += 16) {
                    const u32x4 k = *(const u32x4 *)(k8 + (64 * hh + i) * 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x = fmaf(of_lane(qv[hh], i + 4 * e), __builtin_amdgcn_cvt_f32_fp8((int)k[e], 0) * ks, x);
                        x = fmaf(of_lane(qv[hh], i + 4 * e + 1), __builtin_amdgcn_cvt_f32_fp8((int)k[e], 1) * ks, x);
                        x = fmaf(of_lane(qv[hh], i + 4 * e + 2), __builtin_amdgcn_cvt_f32_fp8((int)k[e], 2) * ks, x);
                        x = fmaf(of_lane(qv[hh], i + 4 * e + 3), __builtin_amdgcn_cvt_f32_fp8((int)k[e], 3) * ks, x);
                    }
                }
            return page_exists(a, id) ? x : -INFINITY;
        },
        [&](int j) __attribute__((always_inline)) { return page_exists(a, pages[j >> a.pshift]); },
        [&](int j, int c) __attribute__((always_inline)) {
            const int page = pages[j >> a.pshift], off = j & in_page, co = 64 * c + lane;
            return __builtin_amdgcn_cvt_f32_fp8((int)a.pg.V8[cell_of(page, off) + (co >> 4) * 256 + (co & 15) * 16 + (off & 15)], 0) *
                   a.pg.vscale[(size_t)page * a.pg.Hkv + h];
        },
        m, l, o);
}

// The same of rows that see all keys first .. seen - 1: tiles are filled up with zeros here.
__device__ __forceinline__ bool paged_sums_stand(const Args &a, const int32_t *pages, int h, int first, int seen) {
    bool bad = false;
    for (int i = (first >> a.pshift) + lane_id(); i <= (seen - 1) >> a.pshift; i += 64)
        if (page_exists(a, pages[i])) bad |= !(a.pg.vscale[(size_t)pages[i] * a.pg.Hkv + h] < VALUES_ADD_UP / 512.0f);
    return !__any(bad);
}

// What a fragment's sums count for against the others': its weight; sums of rows that were done again add up to one, which the sign of
// their sum of weights says (theirs is that times its size).
__device__ __forceinline__ float parts_of(float l, float weight) { return l < 0.0f ? -l * weight : weight; }

}  // namespace paged

}  // namespace fastar
