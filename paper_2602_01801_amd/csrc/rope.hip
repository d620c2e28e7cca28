// Norm of queries and keys per head and their rotation by position, in one pass (qk_norm_rope).
#include <algorithm>

#include "rope_dev.hpp"

namespace fastar {

namespace rope_call {

constexpr int WAVES = 4;

struct Args {
    RopeArgs r;
    RopeViews v;
    int parts;   // wavefronts per token
};

// Bound by memory: every row is read and written once.  A wavefront per token and as many groups of its heads as the rule below leaves it, asked for four
// ahead, so that its angles and its trip to the sequences' offsets are paid once: 13683 tokens x 48 heads 68 us (4.9 TB/s; 120 with four groups per wavefront, each
// with its own), 4680 x 24 in fp32 25.6 (4.5 TB/s; 20 from the last-level cache), one token 2.7.
template <bool BF16, int D, bool INTER>
__global__ __launch_bounds__(64 * WAVES) void rope_kernel(Args a) {
    const long long unit = (long long)blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = (int)(unit / a.parts), part = (int)(unit % a.parts);
    if (t >= a.r.n_tok) return;
    rope_token<BF16, D, INTER, 4>(a.r, a.v, t, part, a.parts);
}

}  // namespace rope_call

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
    return RopeArgs{r->freq, r->axis, pos, cu, len, r->qw, r->kw, r->eps, r->norm, r->rot, r->n_axes, B, n_tok};
}

// A token's groups of heads on as many wavefronts as make 4096 of them, ROPE_GROUPS each at most.  A wavefront's angles are for all of its groups, so
// that more wavefronts compute more: for 4096 / 16384 / 32768 of them 1024 tokens of 48 heads take 8.9 / 12.7 / 12.7 us, 4680 of 24 in fp32 20.2 / 27.1 / 31.5.
int rope_parts(int n_tok, int Hq, int Hkv, int d) {
    const int groups = d == 128 ? rope_groups<128>(Hq) + rope_groups<128>(Hkv) : rope_groups<64>(Hq) + rope_groups<64>(Hkv);
    return std::max((groups + ROPE_GROUPS - 1) / ROPE_GROUPS, std::min(groups, std::max(1, 4096 / n_tok)));
}
int rope_launch(const RopeArgs &r, const RopeViews &v, int d, int dtype, int interleaved, hipStream_t s) {
    const rope_call::Args a{r, v, rope_parts(r.n_tok, v.Hq, v.Hkv, d)};
    const int64_t wgs = ((int64_t)r.n_tok * a.parts + rope_call::WAVES - 1) / rope_call::WAVES;
    if (!launch_ok(wgs, 64 * rope_call::WAVES)) return FASTAR_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)wgs), block(64 * rope_call::WAVES);
#define FASTAR_ROPE(BF16, D)                                                                                              \
    do {                                                                                                                  \
        if (interleaved) hipLaunchKernelGGL((rope_call::rope_kernel<BF16, D, true>), grid, block, 0, s, a);         \
        else hipLaunchKernelGGL((rope_call::rope_kernel<BF16, D, false>), grid, block, 0, s, a);                          \
    } while (0)
    if (dtype == FASTAR_BF16) {
        if (d == 128) FASTAR_ROPE(true, 128);
        else FASTAR_ROPE(true, 64);
    } else {
        if (d == 128) FASTAR_ROPE(false, 128);
        else FASTAR_ROPE(false, 64);
    }
#undef FASTAR_ROPE
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
    const int elt = dtype == FASTAR_BF16 ? 2 : 4;
    auto both_ok = [&](const fastar_rows *in, const fastar_rows *out, int H) {
        return H == 0 || (view_ok(in, H, n_tok, elt) && view_ok(out, H, n_tok, elt) && rows_apart(out, H, n_tok, d));
    };
    if (!both_ok(Q, Qo, Hq) || !both_ok(K, Ko, Hkv)) return FASTAR_ERR_INVALID_ARG;
    RopeViews v{};
    if (Hq) v.q = view_of(Q, Hq, n_tok, elt), v.qo = view_of(Qo, Hq, n_tok, elt);
    if (Hkv) v.k = view_of(K, Hkv, n_tok, elt), v.ko = view_of(Ko, Hkv, n_tok, elt);
    v.Hq = Hq;
    v.Hkv = Hkv;
    return rope_launch(rope_args(rope, pos, cu, len, B, n_tok), v, d, dtype, rope->interleaved, (hipStream_t)stream);
}
