// New keys and values into pages, the keys normed and rotated on the way, and the queries beside them (kv_pages_write_rope).
#include <algorithm>

#include "pages_dev.hpp"

namespace fastar {

namespace pages {

// Rows o .. e - 1 of a page where some row's squares leave the range or some number is not finite, a few at a time: roped(r, x) gives a
// lane's two pieces of row r.  Two passes, for the scale and for the codes.
template <int D, class Roped>
__device__ __forceinline__ void write_odd_roped_run(Roped roped, const RopeLane &l, int o, int e, uint8_t *cell0, int page_bytes, float old_scale,
                                                    float *scale_out) {
    constexpr int LPR = D / 8, RPI = 64 / LPR;
    const int lane = threadIdx.x & 63, lr = lane / LPR;
    float amax = 0.0f, inv = 1.0f;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
        for (int r0 = o; r0 < e; r0 += RPI) {
            const int r = r0 + lr;
            float x[8];
            roped(min(r, e - 1), x);   // rows beyond the last are the last again
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                amax = fmaxf(amax, finite_abs(x[i]));
                x[i] *= inv;
            }
            if (pass == 0 || r >= e) continue;
            uint8_t *p = cell0 + (r >> 4) * (D / 16) * 256 + (r & 15) * 16;
            *(unsigned *)(p + (l.a >> 4) * 256 + (l.a & 15)) = f8_of(x[0], x[1], x[2], x[3]);
            *(unsigned *)(p + (l.b >> 4) * 256 + (l.b & 15)) = f8_of(x[4], x[5], x[6], x[7]);
        }
        if (pass == 1) break;
        const float scale = fmaxf(pow2(scale_exp(wave_max(amax))), old_scale);
        inv = 1.0f / scale;
        if (o > 0 && old_scale * inv < 1.0f) {
            for (int i = lane; i < page_bytes / 4; i += 64) ((unsigned *)cell0)[i] = rescaled(((unsigned *)cell0)[i], old_scale * inv);
            __threadfence();   // before other lanes' new codes go to the same words
        }
        if (lane == 0) *scale_out = scale;
    }
}
// Where four coordinates of a row lie in a wavefront's part of LDS: neighbouring groups of a cell change places with the cell, so that eight
// lanes that read the same group of eight cells meet all banks, as those that write neighbouring groups do.
__device__ __forceinline__ int lds_group(int group) { return group ^ (group >> 3 & 3); }

struct RopeWriteArgs {
    RopeArgs r;
    RopeViews q;          // Hkv = 0: the keys go another way
    View k, v;
    fastar_pages pg;
    const int32_t *slot;
    int chunk, parts;     // rows per workgroup of keys and values; wavefronts per token of queries
    long long kv, all;    // workgroups of keys and values, and in all
};

// K, a wavefront for 16 rows, between the load and the maximum normed and rotated in 32 bits.  The rows wait for the run's maximum in LDS, from which
// 16 coordinates of a row go to a lane, a cell's 16 bytes.  (In registers, exchanged by lanes: 147 of them, and three wavefronts per SIMD.)
template <bool BF16, int D, int PSHIFT, bool INTER>
__device__ __forceinline__ void rope_k_run(const RopeArgs &r, const Run &run, int t0,
                                           unsigned (*s_top)[1 << PSHIFT >> 4], f32x4 *s_rows, int turn) {
    constexpr int P = 1 << PSHIFT, NW = P / 16, LPR = D / 8, RPI = 64 / LPR, IT = 16 / RPI;   // row i RPI + lr
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane / LPR;
    const int r0 = 16 * wave, o = run.o, e = run.e;
    const bool touches = r0 < e && r0 + 16 > o;   // rows of the run among the wavefront's 16
    uint8_t *blk = run.page0 + wave * (16 * D);
    auto row_at = [&](int i) { return min(max(r0 + i, o), e - 1); };   // rows beside the run: one of its own again
    const Places places = places_of(r);
    const RopeLane rl = rope_lane<D, INTER>(r);
    Weights kw;
    kw.load(r.norm ? r.kw : nullptr, rl);
    Raw8<BF16> raw[IT];
    if (touches) {
#pragma unroll
        for (int i = 0; i < IT; ++i) raw[i].load(run.row0, (unsigned)row_at(i * RPI + lr) * (unsigned)run.pitch, rl);
    }
    const Place place = place_of(r, places, t0);
    const bool derived = !r.pos && t0 + e - o <= place.end;   // positions follow one another
    auto turn_at = [&](int row) __attribute__((always_inline)) {   // of offset `row` in the page
        const int t = t0 + row - o;
        if (r.rot == 0) return Fractions{}.turn();
        if (derived) return fractions(rl, plus(place.ahead, t)).turn();
        if (r.pos) return fractions(r, rl, t).turn();
        int b = 0;   // a run of several sequences
        while (b < r.B - 1 && r.cu[b + 1] <= t) ++b;
        return fractions(rl, plus(less(r.len[b], min(r.cu[b + 1], r.n_tok)), t)).turn();
    };
    const bool wild = kw.wild();
    unsigned top = 0;
    if (touches) {
        bool odd = wild;
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            float x[8];
            raw[i].to(x);
            odd |= norm_and_turn<D, INTER>(r, turn_at(row_at(i * RPI + lr)), kw, x);
            f32x4 *row = s_rows + (i * RPI + lr) * (D / 4);
            row[lds_group(rl.a / 4)] = f32x4{x[0], x[1], x[2], x[3]};
            row[lds_group(rl.b / 4)] = f32x4{x[4], x[5], x[6], x[7]};
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(fabsf(x[j])));
        }
        if (odd) top = NOT_FINITE;
    }
    top = top_of<NW>(top, s_top, turn);
    if (top >= NOT_FINITE) {
        if (wave == 0)
            write_odd_roped_run<D>([&](int row, float (&x)[8]) __attribute__((always_inline)) {
                Raw8<BF16> w;
                w.load(run.row0 + row * run.pitch, rl);
                float z[8];
                w.to(x);
                w.to(z);
                const Turn at = turn_at(row);
                const bool odd = norm_and_turn<D, INTER>(r, at, kw, z) || wild;
                norm_and_turn_odd<D, INTER>(r, rl, at, kw, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = odd ? x[j] : z[j];
            }, rl, o, e, run.page0, D * P, run.old_scale, run.scale);
        return;
    }
    const float scale = fmaxf(pow2(scale_exp(__uint_as_float(top))), run.old_scale), ratio = run.old_scale / scale;
    const bool grows = o > 0 && ratio < 1.0f;
    if (lane == 0 && wave == 0) *run.scale = scale;
    if (!touches && !grows) return;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const int u = i * 64 + lane, row = u / (D / 16), cell = u % (D / 16);
        const bool mine = r0 + row >= o && r0 + row < e;
        u32x4 *p = (u32x4 *)(blk + cell * 256 + row * 16), y;
        if (mine) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 x = s_rows[row * (D / 4) + lds_group(4 * cell + q)];
                Piece<false, 4> w;
                unsigned c = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) w.w[j] = __float_as_uint(x[j]);
                w.template codes<false>(0, scale, c);
                w.template codes<true>(2, scale, c);
                y[q] = c;
            }
        } else if (grows) {
            y = *p;
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = rescaled(y[q], ratio);
        }
        if (mine || grows) *p = y;
    }
}

// Workgroups of keys, of values and of queries, evenly mixed over the launch: those of keys compute more than they move, the others the
// other way round, and few tokens save a launch.  34612 tokens, 40 heads on 8, 193 to 198 us (4.7 TB/s), in fp32 339 (5.2), 12 on 12 146 (3.6), in fp32 182 (5.3); 96 single tokens with
// their queries 8.2.  (Queries by a launch of their own, at eight wavefronts per SIMD instead of four: 203, 349, 146 and 199; 96 tokens 13.7 instead of 11.1 a call.)  Without queries
// keys and values of 34612 tokens x 8 heads take 74, where writing them as they are takes 45: 29 are the vector instructions of the keys, at the four wavefronts per SIMD that
// their LDS and registers leave (five spill, 87); of 12 heads 94 (3.4 TB/s), in fp32 120 (4.4).
template <bool BF16, int D, int PSHIFT, bool INTER>
__global__ __launch_bounds__(4 << PSHIFT, 4) void write_rope_kernel(RopeWriteArgs a) {
    constexpr int P = 1 << PSHIFT, NW = P / 16;
    __shared__ unsigned s_top[2][NW];
    __shared__ f32x4 s_rows[NW][16 * D / 4];
    const long long u = blockIdx.x, kv = u * a.kv / a.all;
    if ((u + 1) * a.kv / a.all == kv) {
        const long long unit = (u - kv) * NW + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int t = (int)(unit / a.parts);
        if (t < a.r.n_tok) rope_token<BF16, D, INTER, 8>(a.r, a.q, t, (int)(unit % a.parts), a.parts);
        return;
    }
    const fastar_pages &pg = a.pg;
    const int h = (int)(kv % pg.Hkv), rest = (int)(kv / pg.Hkv), first = (rest >> 1) * a.chunk;
    const bool is_v = rest & 1;
    const unsigned n_slots = (unsigned)pg.n_pages << PSHIFT;
    const int t_lo = a.r.cu ? a.r.cu[0] : 0, t_hi = a.r.cu ? a.r.cu[a.r.B] : a.r.n_tok;
    auto run_of = [&](const View &x, uint8_t *codes, float *scales, int t0, int sl, int n) {
        const int o = sl & (P - 1);
        const size_t ph = (size_t)(sl >> PSHIFT) * pg.Hkv + h;
        return Run{x.p + h * x.head + (int64_t)(t0 - o) * x.row, x.row, o, o + n, codes + ph * (size_t)(D * P), scales + ph, o > 0 ? scales[ph] : 0.0f};
    };
    if (is_v) {
        for_runs<PSHIFT>(a.slot, a.r.n_tok, first, a.chunk, n_slots, t_lo, t_hi, [&](int t0, int sl, int n, int turn) __attribute__((always_inline)) {
            v_run<BF16, D, PSHIFT>(run_of(a.v, pg.V8, pg.vscale, t0, sl, n), s_top, turn);
        });
        return;
    }
    for_runs<PSHIFT>(a.slot, a.r.n_tok, first, a.chunk, n_slots, t_lo, t_hi, [&](int t0, int sl, int n, int turn) __attribute__((always_inline)) {
        rope_k_run<BF16, D, PSHIFT, INTER>(a.r, run_of(a.k, pg.K8, pg.kscale, t0, sl, n), t0, s_top, s_rows[__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)], turn);
    });
}

}  // namespace pages

}  // namespace fastar

extern "C" int kv_pages_write_rope(const fastar_pages *pages, const fastar_rows *Q, const fastar_rows *K_new, const fastar_rows *V_new,
                                   int dtype, const int32_t *slot, const int32_t *pos, const int32_t *cu, const int32_t *len, int B, int n_tok,
                                   int Hq, const fastar_rope *rope, const fastar_rows *Qo, void *stream) {
    using namespace fastar;
    if (dtype != FASTAR_F32 && dtype != FASTAR_BF16) return FASTAR_ERR_INVALID_ARG;
    if (Hq < 0) return FASTAR_ERR_INVALID_ARG;
    if (const int rc = pages_check(pages); rc != FASTAR_OK) return rc;
    if (const int rc = rope_check(rope, pos, cu, len, B, n_tok, pages->d); rc != FASTAR_OK) return rc;
    if (n_tok == 0 || (cu && B == 0)) return FASTAR_OK;
    const int elt = dtype == FASTAR_BF16 ? 2 : 4, d = pages->d, Hkv = pages->Hkv;
    if (!slot || !view_ok(K_new, Hkv, n_tok, elt) || !view_ok(V_new, Hkv, n_tok, elt)) return FASTAR_ERR_INVALID_ARG;
    if (Hq > 0 && !(view_ok(Q, Hq, n_tok, elt) && view_ok(Qo, Hq, n_tok, elt) && rows_apart(Qo, Hq, n_tok, d))) return FASTAR_ERR_INVALID_ARG;
    pages::RopeWriteArgs a{};
    a.r = rope_args(rope, pos, cu, len, B, n_tok);
    a.k = view_of(K_new, Hkv, n_tok, elt);
    a.v = view_of(V_new, Hkv, n_tok, elt);
    if (a.k.row > MAX_PITCH || a.v.row > MAX_PITCH) return FASTAR_ERR_UNSUPPORTED;
    a.pg = *pages;
    a.slot = slot;
    // The runs of a workgroup are done one after the other, 2.8 us each, and one whose rows begin none has been there for nothing.  Of up to four sequences few runs can
    // meet in one, so that a workgroup per compute unit suffices; of more, it depends on their lengths, which the host does not know.  Rows for 256 / for 4096
    // workgroups: a sequence of 64 / 256 / 1024 tokens, 12 heads on 12, pages of 64, 6.3 / 6.8 / 11.0 us and 6.8 / 13.2 / 17.9, four of them 7.8 / 12.6 / 22.4 and
    // 13.5 / 18.3 / 27.2; one, 12 heads on 4, pages of 16, 5.6 / 6.1 / 9.1 and 5.6 / 6.7 / 10.7.  Eight of 256 19 and 23, sixteen 26 and 28; but four of 500 beside 60 single
    // tokens 148 and 41, 96 single tokens 14.8 and 8.3.
    a.chunk = pages::rows_per_workgroup(n_tok, Hkv, pages->P, cu && B <= 4 ? 256 : 4096);
    a.kv = (int64_t)((n_tok + a.chunk - 1) / a.chunk) * Hkv * 2;
    a.all = a.kv;
    const hipStream_t s = (hipStream_t)stream;
    if (Hq > 0) {
        a.q = RopeViews{view_of(Q, Hq, n_tok, elt), View{}, view_of(Qo, Hq, n_tok, elt), View{}, Hq, 0};
        a.parts = rope_parts(n_tok, Hq, 0, d);
        const int waves = pages->P / 16;
        a.all += ((int64_t)n_tok * a.parts + waves - 1) / waves;
        if (!launch_ok(a.all, 4 * pages->P)) {   // more than a launch can have: the queries by themselves
            if (!launch_ok(a.kv, 4 * pages->P)) return FASTAR_ERR_UNSUPPORTED;
            if (const int rc = rope_launch(a.r, a.q, d, dtype, rope->interleaved, s); rc != FASTAR_OK) return rc;
            a.all = a.kv;
        }
    }
    if (!launch_ok(a.all, 4 * pages->P)) return FASTAR_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)a.all);
#define FASTAR_WRITE(BF16, D, PSHIFT) \
    do {                                                                                                                                 \
        if (rope->interleaved) hipLaunchKernelGGL((pages::write_rope_kernel<BF16, D, PSHIFT, true>), grid, dim3(4 << PSHIFT), 0, s, a);  \
        else hipLaunchKernelGGL((pages::write_rope_kernel<BF16, D, PSHIFT, false>), grid, dim3(4 << PSHIFT), 0, s, a);                   \
    } while (0)
#define FASTAR_WRITE_P(BF16, D)                      \
    do {                                             \
        if (pages->P == 64) FASTAR_WRITE(BF16, D, 6); \
        else if (pages->P == 32) FASTAR_WRITE(BF16, D, 5); \
        else FASTAR_WRITE(BF16, D, 4);               \
    } while (0)
    if (dtype == FASTAR_BF16) {
        if (d == 128) FASTAR_WRITE_P(true, 128);
        else FASTAR_WRITE_P(true, 64);
    } else {
        if (d == 128) FASTAR_WRITE_P(false, 128);
        else FASTAR_WRITE_P(false, 64);
    }
#undef FASTAR_WRITE_P
#undef FASTAR_WRITE
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}
