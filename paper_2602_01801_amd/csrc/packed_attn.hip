// Attention over packed sequences, the simple form: a wavefront per (query row, query head), a lane per key of a tile of 64 for
// the scores, a lane per D / 64 coordinates for the values.  fp32 arithmetic throughout.
#include "packed.hpp"

namespace fastar {

int launch_prompt_bf16(const View &Q, const View &K, const View &V, const int32_t *cu_q, const int32_t *cu_k, int B, int n_tok_q,
                       int n_tok_k, int Hq, int Hkv, int d, int causal, float scale_log2, const View &O, float *lse, hipStream_t s);

namespace packed {

constexpr float LN2 = 0.6931471805599453f;

template <bool BF16>
__device__ __forceinline__ float load1(const char *p, int t) {
    if constexpr (BF16) return bf16_bits_to_f32(((const unsigned short *)p)[t]);
    else return ((const float *)p)[t];
}

template <bool BF16, int D, bool PAGED>
__global__ __launch_bounds__(256) void attn_simple_kernel(View Q, View K, View V, const int32_t *__restrict__ cu_q,
                                                          const int32_t *__restrict__ cu_k, const int32_t *__restrict__ len,
                                                          const int32_t *__restrict__ table, int max_pages, fastar_pages pg, int pshift,
                                                          int B, int n_tok_q, int n_tok_k, int Hq, int Hkv, int causal,
                                                          float scale_log2, View O, float *__restrict__ lse) {
    __shared__ float qs[4][D], ps[4][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const long long unit = (long long)blockIdx.x * 4 + wave;
    const int h = (int)(unit / n_tok_q), t = (int)(unit % n_tok_q);
    if (h >= Hq) return;
    if (t < cu_q[0] || t >= cu_q[B]) return;
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu_q[mid] <= t) lo = mid;
        else hi = mid;
    }
    const Rows rq = rows_of(cu_q, lo, n_tok_q);
    int n, k0 = 0;
    if constexpr (PAGED) n = min(max(len[lo], 0), max_pages << pshift);
    else {
        const Rows rk = rows_of(cu_k, lo, n_tok_k);
        n = rk.n;
        k0 = rk.first;
    }
    const int hk = h / (Hq / Hkv);
    const int seen = causal ? min(n, n - rq.n + (t - rq.first) + 1) : n;
    const char *q = Q.p + h * Q.head + t * Q.row;
    for (int c = lane; c < D; c += 64) qs[wave][c] = load1<BF16>(q, c);
    float m = -INFINITY, l = 0.0f, o[D / 64];
    for (int c = 0; c < D / 64; ++c) o[c] = 0.0f;
    for (int j0 = 0; j0 < seen; j0 += 64) {
        const int j = j0 + lane;
        float s = -INFINITY;
        if (j < seen) {
            if constexpr (PAGED) {
                const int page = table[(size_t)lo * max_pages + (j >> pshift)];
                if ((unsigned)page < (unsigned)pg.n_pages) {
                    const size_t ph = (size_t)page * Hkv + hk;
                    const int off = j & ((1 << pshift) - 1);
                    const uint8_t *c = pg.K8 + ph * ((size_t)D << pshift) + (off >> 4) * (16 * D) + (off & 15) * 16;
                    float a = 0.0f;
                    for (int x = 0; x < D; ++x) a = fmaf(__builtin_amdgcn_cvt_f32_fp8((int)c[(x >> 4) * 256 + (x & 15)], 0), qs[wave][x], a);
                    s = a * pg.kscale[ph];
                }
            } else {
                const char *k = K.p + hk * K.head + (int64_t)(k0 + j) * K.row;
                s = 0.0f;
                for (int x = 0; x < D; ++x) s = fmaf(load1<BF16>(k, x), qs[wave][x], s);
            }
        }
        float mt = s;
        for (int x = 32; x > 0; x >>= 1) mt = fmaxf(mt, __shfl_xor(mt, x, 64));
        const float mn = fmaxf(m, mt);
        const float base = mn == -INFINITY ? 0.0f : mn;   // a tile without a key, or whose scores are no numbers
        const float a = exp2f((m - base) * scale_log2), p = exp2f((s - base) * scale_log2);
        m = mn;
        float pt = p;
        for (int x = 32; x > 0; x >>= 1) pt += __shfl_xor(pt, x, 64);
        l = l * a + pt;
        ps[wave][lane] = p;
        for (int c = 0; c < D / 64; ++c) o[c] *= a;
        for (int i = 0; i < min(64, seen - j0); ++i) {
            const float w = ps[wave][i];
            if (w == 0.0f) continue;
            for (int c = 0; c < D / 64; ++c) {
                const int x = 64 * c + lane;
                float v;
                if constexpr (PAGED) {
                    const int jj = j0 + i, page = table[(size_t)lo * max_pages + (jj >> pshift)];
                    const size_t ph = (size_t)page * Hkv + hk;
                    const int off = jj & ((1 << pshift) - 1);
                    v = __builtin_amdgcn_cvt_f32_fp8((int)pg.V8[ph * ((size_t)D << pshift) + (off >> 4) * (16 * D) + (x >> 4) * 256 + (x & 15) * 16 + (off & 15)], 0) *
                        pg.vscale[ph];
                } else {
                    v = load1<BF16>(V.p + hk * V.head + (int64_t)(k0 + j0 + i) * V.row, x);
                }
                o[c] = fmaf(w, v, o[c]);
            }
        }
    }
    char *op = O.p + h * O.head + t * O.row;
    for (int c = 0; c < D / 64; ++c) {
        const float r = l == 0.0f ? 0.0f : o[c] / l;   // a sum that is no number stays one
        if constexpr (BF16) ((__bf16 *)op)[64 * c + lane] = (__bf16)r;
        else ((float *)op)[64 * c + lane] = r;
    }
    if (lse && lane == 0) lse[(size_t)h * n_tok_q + t] = l == 0.0f ? -INFINITY : (m * scale_log2 + __log2f(l)) * LN2;
}

}  // namespace packed

}  // namespace fastar

extern "C" int prompt_attn_fwd(const fastar_rows *Q, const fastar_rows *K, const fastar_rows *V, const int32_t *cu_q,
                               const int32_t *cu_k, int B, int n_tok_q, int n_tok_k, int Hq, int Hkv, int d, int dtype, int causal,
                               float scale, const fastar_rows *O, float *lse, void *stream) {
    using namespace fastar;
    if (dtype != FASTAR_F32 && dtype != FASTAR_BF16) return FASTAR_ERR_INVALID_ARG;
    const int elt = dtype == FASTAR_BF16 ? 2 : 4;
    if (B < 0 || n_tok_q < 0 || n_tok_k < 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv) return FASTAR_ERR_INVALID_ARG;
    if (!scale_ok(scale) || (causal & ~1)) return FASTAR_ERR_INVALID_ARG;
    if (d != 64 && d != 128) return FASTAR_ERR_UNSUPPORTED;
    if ((int64_t)n_tok_q * Hq > INT32_MAX / 2) return FASTAR_ERR_UNSUPPORTED;
    if (n_tok_q == 0 || B == 0) return FASTAR_OK;
    if (!cu_q || !view_ok(Q, elt) || !view_ok(O, elt) || !rows_apart(O, Hq, n_tok_q, d)) return FASTAR_ERR_INVALID_ARG;
    if (n_tok_k > 0 && (!view_ok(K, elt) || !view_ok(V, elt))) return FASTAR_ERR_INVALID_ARG;
    if (n_tok_k > 0 && (K->row * elt > MAX_PITCH || V->row * elt > MAX_PITCH)) return FASTAR_ERR_UNSUPPORTED;
    if (!cu_k) cu_k = cu_q;
    const View none{nullptr, 0, 0};
    const View q = view_of(Q, elt), k = n_tok_k ? view_of(K, elt) : none, v = n_tok_k ? view_of(V, elt) : none, o = view_of(O, elt);
    const dim3 grid((unsigned)(((int64_t)n_tok_q * Hq + 3) / 4));
    const float sl = scale * 1.4426950408889634f;
#define FASTAR_SIMPLE(BF16, D)                                                                                                    \
    hipLaunchKernelGGL((packed::attn_simple_kernel<BF16, D, false>), grid, dim3(256), 0, (hipStream_t)stream, q, k, v, cu_q, cu_k, \
                       nullptr, nullptr, 0, fastar_pages{}, 0, B, n_tok_q, n_tok_k, Hq, Hkv, causal, sl, o, lse)
    if (dtype == FASTAR_BF16)
        return launch_prompt_bf16(q, k, v, cu_q, cu_k, B, n_tok_q, n_tok_k, Hq, Hkv, d, causal, sl, o, lse, (hipStream_t)stream);
    if (d == 128) FASTAR_SIMPLE(false, 128);
    else FASTAR_SIMPLE(false, 64);
#undef FASTAR_SIMPLE
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}
