// Norm of queries and keys per head and their rotation by position, in one pass (qk_norm_rope).
#include <algorithm>

#include "rope_dev.hpp"

namespace fastar {

namespace rope {

constexpr int WAVES = 4;

struct Args {
    View q, k, qo, ko;
    RopeArgs r;
    int Hq, Hkv, parts;
};

// A wavefront takes one token, whose angles it computes once, and every parts-th group of 64 / (d / 8) heads of it.
template <bool BF16, int D>
__global__ __launch_bounds__(64 * WAVES) void rope_kernel(Args a) {
    constexpr int LPR = D / 8, RPW = 64 / LPR, ELT = BF16 ? 2 : 4;
    const RopeArgs &r = a.r;
    const int lane = lane_id(), lr = lane / LPR, lc = lane % LPR;
    const long long unit = (long long)blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = (int)(unit / a.parts), part = (int)(unit % a.parts);
    if (t >= r.n_tok) return;
    if (r.cu && (t < r.cu[0] || t >= r.cu[r.B])) return;
    const RopeLane rl = rope_lane<D>(r);
    double pos[4] = {0.0, 0.0, 0.0, 0.0};
    if (r.rot > 0) {
        if (r.pos) {
#pragma unroll
            for (int i = 0; i < 4; ++i) pos[i] = r.pos[(size_t)rl.axis[i] * r.n_tok + t];
        } else {
            const int b = sequence_of(r.cu, r.B, t);
            const double p = (double)((long long)r.len[b] - min(r.cu[b + 1], r.n_tok) + t);
#pragma unroll
            for (int i = 0; i < 4; ++i) pos[i] = p;
        }
    }
    const Turn turn = turn_of(rl, pos);
    float qw[8], kw[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        qw[e] = r.norm && r.qw ? r.qw[8 * lc + e] : 1.0f;
        kw[e] = r.norm && r.kw ? r.kw[8 * lc + e] : 1.0f;
    }
    const int gq = (a.Hq + RPW - 1) / RPW, gk = (a.Hkv + RPW - 1) / RPW;
    for (int g = part; g < gq + gk; g += a.parts) {
        const bool is_k = g >= gq;
        const int h = (is_k ? g - gq : g) * RPW + lr, H = is_k ? a.Hkv : a.Hq;
        const View &in = is_k ? a.k : a.q, &out = is_k ? a.ko : a.qo;
        float x[8], w[8];
        load8<BF16>(in.p + min(h, H - 1) * in.head + t * in.row + lc * 8 * ELT, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = is_k ? kw[e] : qw[e];
        norm_and_turn<D>(r, rl, turn, w, x);
        if (h < H) store8<BF16>(out.p + h * out.head + t * out.row + lc * 8 * ELT, x);
    }
}

}  // namespace rope

int rope_check(const fastar_rope *r, const int32_t *pos, const int32_t *cu, const int32_t *len, int B, int n_tok, int d) {
    if (!r || B < 0 || n_tok < 0) return FASTAR_ERR_INVALID_ARG;
    if ((r->norm != 0 && r->norm != 1) || (r->interleaved != 0 && r->interleaved != 1)) return FASTAR_ERR_INVALID_ARG;
    if (r->norm && !(r->eps >= 0.0f && r->eps < INFINITY)) return FASTAR_ERR_INVALID_ARG;
    if (d != 64 && d != 128) return FASTAR_ERR_UNSUPPORTED;
    if (r->rot < 0 || r->rot > d || r->n_axes < 1) return FASTAR_ERR_INVALID_ARG;
    if (r->rot > 0 && (!r->freq || (!pos && !len))) return FASTAR_ERR_INVALID_ARG;
    if (!cu && (B > 0 || (r->rot > 0 && !pos))) return FASTAR_ERR_INVALID_ARG;
    if (r->rot % 16 || r->n_axes > 4 || n_tok > MAX_KEYS) return FASTAR_ERR_UNSUPPORTED;
    return FASTAR_OK;
}
RopeArgs rope_args(const fastar_rope *r, const int32_t *pos, const int32_t *cu, const int32_t *len, int B, int n_tok) {
    return RopeArgs{r->freq, r->axis, pos, cu, len, r->qw, r->kw, r->eps, r->norm, r->rot, r->interleaved, r->n_axes, B, n_tok};
}

// Checks the views and launches; everything else has been checked.
int rope_launch(const fastar_rows *Q, const fastar_rows *K, const RopeArgs &r, int Hq, int Hkv, int d, int dtype, const fastar_rows *Qo,
                const fastar_rows *Ko, hipStream_t s) {
    const int elt = dtype == FASTAR_BF16 ? 2 : 4, n_tok = r.n_tok;
    auto both_ok = [&](const fastar_rows *in, const fastar_rows *out, int H) {
        return H == 0 || (view_ok(in, H, n_tok, elt) && view_ok(out, H, n_tok, elt) && rows_apart(out, H, n_tok, d));
    };
    if (!both_ok(Q, Qo, Hq) || !both_ok(K, Ko, Hkv)) return FASTAR_ERR_INVALID_ARG;
    rope::Args a{};
    if (Hq) a.q = view_of(Q, Hq, n_tok, elt), a.qo = view_of(Qo, Hq, n_tok, elt);
    if (Hkv) a.k = view_of(K, Hkv, n_tok, elt), a.ko = view_of(Ko, Hkv, n_tok, elt);
    a.r = r;
    a.Hq = Hq;
    a.Hkv = Hkv;
    const int rpw = 512 / d;
    const int64_t groups = ((int64_t)Hq + rpw - 1) / rpw + ((int64_t)Hkv + rpw - 1) / rpw;
    // A token's groups on as many wavefronts as make 8192 of them.
    a.parts = (int)std::min<int64_t>(groups, std::max<int64_t>(1, 8192 / n_tok));
    const int64_t wgs = ((int64_t)n_tok * a.parts + rope::WAVES - 1) / rope::WAVES;
    if (!launch_ok(wgs, 64 * rope::WAVES)) return FASTAR_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)wgs), block(64 * rope::WAVES);
    if (dtype == FASTAR_BF16) {
        if (d == 128) hipLaunchKernelGGL((rope::rope_kernel<true, 128>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((rope::rope_kernel<true, 64>), grid, block, 0, s, a);
    } else {
        if (d == 128) hipLaunchKernelGGL((rope::rope_kernel<false, 128>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((rope::rope_kernel<false, 64>), grid, block, 0, s, a);
    }
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}

}  // namespace fastar

extern "C" int qk_norm_rope(const fastar_rows *Q, const fastar_rows *K, const int32_t *pos, const int32_t *cu, const int32_t *len, int B,
                            int n_tok, int Hq, int Hkv, int d, int dtype, const fastar_rope *rope, const fastar_rows *Qo,
                            const fastar_rows *Ko, void *stream) {
    using namespace fastar;
    if (dtype != FASTAR_F32 && dtype != FASTAR_BF16) return FASTAR_ERR_INVALID_ARG;
    if (Hq < 0 || Hkv < 0) return FASTAR_ERR_INVALID_ARG;
    if (const int rc = rope_check(rope, pos, cu, len, B, n_tok, d); rc != FASTAR_OK) return rc;
    if (n_tok == 0 || (cu && B == 0) || (Hq == 0 && Hkv == 0)) return FASTAR_OK;
    return rope_launch(Q, K, rope_args(rope, pos, cu, len, B, n_tok), Hq, Hkv, d, dtype, Qo, Ko, (hipStream_t)stream);
}
