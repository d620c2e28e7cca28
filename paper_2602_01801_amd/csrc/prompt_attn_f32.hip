// Attention over packed prompts, fp32 (prompt_attn_fwd), on the fp32 matrix instructions, and the entry point for both types.
//
// A workgroup owns 16 RW rows of one sequence and key head ((token, head of the group) pairs); RW wavefronts, a team, take 16
// rows each and walk tiles of 16 HB keys; teams of a workgroup take turns at the tiles of the same rows and put their sums
// together at the end.  Both contractions are transposed (lane l: row l % 16, quarter q = l / 16) on v_mfma_f32_16x16x4_f32,
// whose k order is free as long as both operands agree:
//     S^T = K Q^T    A = K, lane l: key l % 16, coordinates 16 c + 4 q .. + 3 in one 16-byte read, four products
//     O^T = V^T P^T  B = the score registers as they are (product v: key 4 q + v); A = V: block 4 e + x of 16 output rows stands
//                    for coordinates 64 e + 4 (l % 16) + x, so that a lane's 16-byte read feeds four blocks
// Two forms.  Where workgroups fill the chip: four wavefronts over shared tiles of 32 keys, K and V straight from global memory
// into LDS, two stages.  Where they do not: a workgroup per 16 rows, whose four wavefronts take every fourth tile of 16 keys
// without a barrier, K by way of LDS, V from global memory into registers.
// What bounds the first are the matrix instructions (32 cycles each, nothing runs beside them): 12 heads on 4 key heads x 4680
// tokens, causal, 621 us = 108 TFLOP/s of 157; the second the chain of one wavefront's tile (0.7 us of scores, 0.1 of softmax, 0.6 of
// values at one wavefront per SIMD) and 5 us of a launch's ends: 4 sequences of 390 to 780 x 4 heads over prompts of 64 to 512 30 us.
#include "packed.hpp"

#include <type_traits>

namespace fastar {

int launch_prompt_bf16(const View &Q, const View &K, const View &V, const int32_t *cu_q, const int32_t *cu_k, int B, int n_tok_q,
                       int n_tok_k, int Hq, int Hkv, int d, int causal, float scale_log2, const View &O, float *lse, hipStream_t s);

namespace prompt32 {

__device__ __forceinline__ f32x4 mfma_16x16x4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
// LDS reads as assembly: the compiler would wait for the tile loads in flight before each of its own.
__device__ __forceinline__ f32x4 lds_read(unsigned addr) {
    f32x4 r;
    asm volatile("ds_read_b128 %0, %1" : "=v"(r) : "v"(addr));
    return r;
}
template <int N>
__device__ __forceinline__ void wait_vm() {   // until at most N loads are outstanding
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}
// Waits until at most `behind` batches of N reads later than f are outstanding; f has landed then.
template <int N>
__device__ __forceinline__ void wait_for(f32x4 (&f)[N], int behind) {
    if constexpr (N == 2) {
        if (behind == 2) asm volatile("s_waitcnt lgkmcnt(4)" : "+v"(f[0]), "+v"(f[1]));
        else if (behind == 1) asm volatile("s_waitcnt lgkmcnt(2)" : "+v"(f[0]), "+v"(f[1]));
        else asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]), "+v"(f[1]));
    } else {
        if (behind == 2) asm volatile("s_waitcnt lgkmcnt(2)" : "+v"(f[0]));
        else if (behind == 1) asm volatile("s_waitcnt lgkmcnt(1)" : "+v"(f[0]));
        else asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]));
    }
}

// Workgroups of 64 rows from which on 16 rows no longer take a workgroup of their own (two of the former per compute unit).
// 16 rows each against 64, causal, d = 128: 300 workgroups of 64 rows 115 / 142 us, 188 (not causal) 69 / 77; d = 64: 264 42 / 49.
constexpr int FULL = 512;

struct Args {
    View Q, K, V, O;
    const int32_t *cu_q, *cu_k;
    int B, n_tok_q, n_tok_k, Hkv, group, causal;
    float scale_log2;
    float *lse;
};

template <int D, int RW, int TEAMS, int HB, int NS>
__global__ __launch_bounds__(TEAMS * RW * 64, 2) void attn_f32_prompt_kernel(const Args a) {
    constexpr int NW = RW, R = 16 * RW, TK = 16 * HB;
    constexpr int CH = D / 16, ROWB = D * 4, TILEB = TK * ROWB, CPR = ROWB / 16;
    constexpr int RPI = 1024 / ROWB, IPW = TILEB / 1024 / NW;   // rows per direct load of 1 KiB, loads per wavefront, tensor and tile
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];   // [team][stage][K, V]
    __shared__ float s_m[TEAMS][NW][16], s_l[TEAMS][NW][16];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int team = wave / NW, w = wave % NW;
    const int col = lane & 15, quarter = lane >> 4;

    Item it;
    if (!find_item<R>(a.cu_q, a.cu_k, a.B, a.n_tok_q, a.n_tok_k, a.group, a.Hkv, blockIdx.x, it)) return;
    const int h = it.local % a.Hkv, qt = it.n / a.Hkv - 1 - it.local / a.Hkv;
    const Rows rq = it.q, rk = it.k;
    const int n_rows = rq.n * a.group, n = rk.n;
    auto sees = [&](int r) { return a.causal ? min(max(n - rq.n + min(r, n_rows - 1) / a.group + 1, 0), n) : n; };
    const int nt = (sees(qt * R + R - 1) + TK - 1) / TK;
    const int row0 = qt * R + w * 16;
    const int limit_min = sees(row0);
    const int my_row = min(row0 + col, n_rows - 1);
    const int my_tok = my_row / a.group, my_head = h * a.group + my_row - my_tok * a.group;
    const int limit = sees(my_row);
    const float scale_log2 = a.scale_log2;

    f32x4 q[CH], o[CH];
    {
        const char *qp = a.Q.p + my_head * a.Q.head + (int64_t)(rq.first + my_tok) * a.Q.row;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            q[c] = *(const f32x4 *)(qp + (16 * c + 4 * quarter) * 4);
            o[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
    float m = -INFINITY, neg = 0.0f, l = 0.0f;

    const char *Kb = a.K.p + h * a.K.head + (int64_t)rk.first * a.K.row, *Vb = a.V.p + h * a.V.head + (int64_t)rk.first * a.V.row;
    unsigned char *mine = lds + team * NS * (RW == 1 ? 1 : 2) * TILEB;
    // one 16-byte piece per lane; K's pieces are permuted within a row, piece c of row w at c ^ (w & 15)
    unsigned koff[IPW], voff[IPW];
#pragma unroll
    for (int i = 0; i < IPW; ++i) {
        const int r = RPI * (IPW * w + i) + lane / CPR;
        koff[i] = (unsigned)r * (unsigned)a.K.row + 16 * ((lane % CPR) ^ (r & 15));
        voff[i] = (unsigned)r * (unsigned)a.V.row + 16 * (lane % CPR);
    }
    auto issue = [&](const char *base, int64_t pitch, const unsigned (&off)[IPW], unsigned char *dst, int t) __attribute__((always_inline)) {
        if (RW > 1 && t * TK + TK <= n) {   // uniform
            const char *tile = base + (int64_t)t * TK * pitch;
#pragma unroll
            for (int i = 0; i < IPW; ++i) to_lds(tile, off[i], lds_address(dst) + (IPW * w + i) * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < IPW; ++i) {   // rows past the end: key 0, which is seen wherever a key is
                const int r = RPI * (IPW * w + i) + lane / CPR;
                to_lds(base + off[i] + (t * TK + r < n ? (int64_t)t * TK * pitch : -(int64_t)r * pitch), dst + (IPW * w + i) * 1024);
            }
        }
    };
    constexpr bool OWN = RW == 1;                 // a wavefront's tiles are its own
    constexpr int STAGEB = (OWN ? 1 : 2) * TILEB;   // K (and V) of a tile
    auto issue_tile = [&](int t, int stage) __attribute__((always_inline)) {
        if (t >= nt) return;
        issue(Kb, a.K.row, koff, mine + stage * STAGEB, t);
        if constexpr (!OWN) issue(Vb, a.V.row, voff, mine + stage * STAGEB + TILEB, t);
    };
    constexpr int STEPS = 4 * HB;   // of the second product; step i: key 16 (i / 4) + 4 quarter + i % 4
    f32x4 vown[OWN ? STEPS : 1][D / 64];
    auto load_v = [&](int t) __attribute__((always_inline)) {   // 16 lanes read 256 bytes of a row
        if (t >= nt) return;
#pragma unroll
        for (int i = 0; i < (OWN ? STEPS : 0); ++i) {
            const int r = t * TK + (i >> 2) * 16 + 4 * quarter + (i & 3);
            const char *p = Vb + (int64_t)(r < n ? r : 0) * a.V.row + col * 16;
#pragma unroll
            for (int e = 0; e < D / 64; ++e) vown[i][e] = *(const f32x4 *)(p + 256 * e);
        }
    };
    const unsigned mine_lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)mine;
    const unsigned kaddr0 = mine_lds + col * ROWB + ((quarter ^ col) << 4);        // chunk c: exclusive or with 64 c
    const unsigned vaddr0 = mine_lds + TILEB + 4 * quarter * ROWB + col * 16;

    const int turns = (nt + TEAMS - 1) / TEAMS;   // the same for all teams
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) issue_tile(TEAMS * i + team, i);
    load_v(team);
    int stage = 0;
    for (int i = 0; i < turns; ++i) {
        const int t = TEAMS * i + team;
        // tile t is there
        if constexpr (OWN) {
            if (t >= nt) break;
            wait_vm<STEPS * (D / 64)>();   // V was asked for last
            asm volatile("" ::: "memory");
        } else {
            wait_vm<0>();
            asm volatile("s_barrier" ::: "memory");   // for all of the team; nobody reads the stage of the turn before any more
        }
        issue_tile(t + TEAMS * (NS - 1), stage == 0 ? NS - 1 : stage - 1);
        const unsigned kaddr = kaddr0 + stage * STAGEB, vaddr = vaddr0 + stage * STAGEB;
        stage = stage == NS - 1 ? 0 : stage + 1;
        if (t >= nt) continue;   // uniform over the team
        constexpr int NA = 2 / HB;   // two chains of products at least: one waits for its own results
        f32x4 s[HB], sa[NA][HB];
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int hb = 0; hb < HB; ++hb) sa[i][hb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        {
            f32x4 kf[3][HB];   // operands are asked for two chunks ahead
            auto read = [&](int c) __attribute__((always_inline)) {
#pragma unroll
                for (int hb = 0; hb < HB; ++hb) kf[c % 3][hb] = lds_read((kaddr ^ (unsigned)(64 * c)) + 16 * hb * ROWB);
            };
            read(0);
            read(1);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (c + 2 < CH) read(c + 2);
                wait_for(kf[c % 3], min(CH - 1 - c, 2));
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int hb = 0; hb < HB; ++hb) sa[e % NA][hb] = mfma_16x16x4(kf[c % 3][hb][e], q[c][e], sa[e % NA][hb]);
            }
#pragma unroll
            for (int hb = 0; hb < HB; ++hb) s[hb] = NA == 2 ? sa[0][hb] + sa[NA - 1][hb] : sa[0][hb];
        }
        if (t * TK + TK > limit_min) {
#pragma unroll
            for (int hb = 0; hb < HB; ++hb)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (t * TK + 16 * hb + 4 * quarter + v >= limit) s[hb][v] = -INFINITY;
        }
        float mx = s[0][0];
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
#pragma unroll
            for (int v = 0; v < 4; ++v) mx = fmaxf(mx, s[hb][v]);
        mx = max_of_quarters(mx);
        if (__any((mx - m) * scale_log2 > 8.0f)) {   // the reference may lag the maximum by 8 octaves
            const float mn = fmaxf(m, mx);
            const float alpha = m == -INFINITY ? 0.0f : exp2f((m - mn) * scale_log2);
            m = mn;
            neg = mn == -INFINITY ? 0.0f : -mn * scale_log2;
            l *= alpha;
#pragma unroll
            for (int c = 0; c < CH; ++c) o[c] *= alpha;
        }
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                s[hb][v] = exp2f(fmaf(s[hb][v], scale_log2, neg));   // with its subnormal results: values go up to 2^128
                l += s[hb][v];
            }
        {
            f32x4 vf[3][D / 64];
            auto read = [&](int i) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < D / 64; ++e) vf[i % 3][e] = lds_read(vaddr + ((i >> 2) * 16 + (i & 3)) * ROWB + 256 * e);
            };
            if constexpr (!OWN) {
                read(0);
                read(1);
            }
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                if constexpr (!OWN) {
                    if (i + 2 < STEPS) read(i + 2);
                    wait_for(vf[i % 3], min(STEPS - 1 - i, 2));
                }
#pragma unroll
                for (int e = 0; e < D / 64; ++e)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        o[4 * e + x] = mfma_16x16x4(OWN ? vown[OWN ? i : 0][e][x] : vf[i % 3][e][x], s[i >> 2][i & 3], o[4 * e + x]);
            }
            load_v(t + TEAMS);
        }
    }
    l = sum_of_quarters(l);
    if constexpr (TEAMS > 1) {   // the other teams hand their sums to team 0
        __syncthreads();
        static_assert(CH * 1024 <= NS * STAGEB / NW, "a team's sums fit its stages");
        f32x4 *give = (f32x4 *)lds;   // [team - 1][wavefront][block][lane]
        if (team > 0) {
#pragma unroll
            for (int c = 0; c < CH; ++c) give[(((team - 1) * NW + w) * CH + c) * 64 + lane] = o[c];
        }
        if (quarter == 0) {
            s_m[team][w][col] = m;
            s_l[team][w][col] = l;
        }
        __syncthreads();
        if (team > 0) return;
        float m_all = m;
#pragma unroll
        for (int i = 1; i < TEAMS; ++i) m_all = fmaxf(m_all, s_m[i][w][col]);
        auto weight = [&](float mi) { return mi == -INFINITY ? 0.0f : exp2f((mi - m_all) * scale_log2); };
        const float mine_w = weight(m);
        l *= mine_w;
#pragma unroll
        for (int c = 0; c < CH; ++c) o[c] *= mine_w;
#pragma unroll
        for (int i = 1; i < TEAMS; ++i) {
            const float wi = weight(s_m[i][w][col]);
            l += s_l[i][w][col] * wi;
#pragma unroll
            for (int c = 0; c < CH; ++c) o[c] += give[(((i - 1) * NW + w) * CH + c) * 64 + lane] * wi;
        }
        m = m_all;
    }
    bool odd = !sums_up(m, l);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int v = 0; v < 4; ++v) odd |= !(fabsf(o[c][v]) < INFINITY);
    // register v of block 4 e + x: coordinate 64 e + 4 (4 quarter + v) + x: four blocks' registers v are 16 bytes of a row
    if (row0 + col < n_rows) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        char *op = a.O.p + my_head * a.O.head + (int64_t)(rq.first + my_tok) * a.O.row;
#pragma unroll
        for (int e = 0; e < D / 64; ++e)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const f32x4 y = {o[4 * e][v] * inv, o[4 * e + 1][v] * inv, o[4 * e + 2][v] * inv, o[4 * e + 3][v] * inv};
                *(f32x4 *)(op + (64 * e + 16 * quarter + 4 * v) * 4) = y;
            }
        if (a.lse && quarter == 0)
            a.lse[(size_t)my_head * a.n_tok_q + rq.first + my_tok] = lse_of(m, l, scale_log2);
    }
    // as in prompt_attn.hip: rows whose sums are not finite
    if (__builtin_expect(__any(odd), 0)) {
        const Args a = args_anew<Args>();
        const char *K = a.K.p + h * a.K.head + (int64_t)rk.first * a.K.row, *V = a.V.p + h * a.V.head + (int64_t)rk.first * a.V.row;
        if (!a.causal && !__any(!sums_up(m, l) && !no_number(m, l, a.scale_log2)) && sums_stand<float, D>(V, a.V.row, n, n % TK != 0)) return;
        for (int r = 0; r < 16 && row0 + r < n_rows; ++r) {
            const int rr = row0 + r, tok = rr / a.group, head = h * a.group + rr - tok * a.group;
            float mr, lr, acc[D / 64];
            row_by_keys<float, D>(a.Q.p + head * a.Q.head + (int64_t)(rq.first + tok) * a.Q.row, K, a.K.row, V, a.V.row,
                                  a.causal ? min(max(n - rq.n + tok + 1, 0), n) : n, a.scale_log2, mr, lr, acc);
            float *op = (float *)(a.O.p + head * a.O.head + (int64_t)(rq.first + tok) * a.O.row);
#pragma unroll
            for (int c = 0; c < D / 64; ++c) op[64 * c + lane] = acc[c];
            if (lane == 0 && a.lse) a.lse[(size_t)head * a.n_tok_q + rq.first + tok] = lse_of(mr, lr, a.scale_log2);
        }
    }
}

template <int D, int RW, int TEAMS, int HB, int NS>
struct Form {
    static constexpr int R = 16 * RW, LDS = TEAMS * NS * (RW == 1 ? 1 : 2) * 16 * HB * D * 4;
    static int setup() {
        if (LDS <= 65536) return FASTAR_OK;
        return hipFuncSetAttribute((const void *)attn_f32_prompt_kernel<D, RW, TEAMS, HB, NS>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS) == hipSuccess ? FASTAR_OK : FASTAR_ERR_HIP;
    }
    static int launch(const Args &a, hipStream_t s) {
        if (!launch_ok(items(a), TEAMS * RW * 64)) return FASTAR_ERR_UNSUPPORTED;
        if (const int rc = prompt_f32_setup(); rc != FASTAR_OK) return rc;
        hipLaunchKernelGGL((attn_f32_prompt_kernel<D, RW, TEAMS, HB, NS>), dim3((unsigned)items(a)), dim3(TEAMS * RW * 64), LDS, s, a);
        FASTAR_LAUNCH_CHECK();
        return FASTAR_OK;
    }
    static int64_t items(const Args &a) { return (((int64_t)a.n_tok_q * a.group + R - 1) / R + a.B) * a.Hkv; }   // at most
};
template <int D>
int launch(const Args &a, hipStream_t s) {
    if (Form<D, 4, 1, 2, 2>::items(a) > FULL) return Form<D, 4, 1, 2, 2>::launch(a, s);
    return Form<D, 1, 4, 1, 2>::launch(a, s);
}

}  // namespace prompt32

int prompt_f32_setup() {
    using namespace prompt32;
    static DeviceOnce once;
    return once.run([](int) {
        int rc = Form<128, 4, 1, 2, 2>::setup();
        if (rc == FASTAR_OK) rc = Form<64, 4, 1, 2, 2>::setup();
        if (rc == FASTAR_OK) rc = Form<128, 1, 4, 1, 2>::setup();
        if (rc == FASTAR_OK) rc = Form<64, 1, 4, 1, 2>::setup();
        return rc;
    });
}

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
    if ((int64_t)n_tok_q * Hq > INT32_MAX / 2 || n_tok_k > MAX_KEYS) return FASTAR_ERR_UNSUPPORTED;
    if (n_tok_q == 0 || B == 0) return FASTAR_OK;
    if (!cu_q || !view_ok(Q, Hq, n_tok_q, elt) || !view_ok(O, Hq, n_tok_q, elt) || !rows_apart(O, Hq, n_tok_q, d)) return FASTAR_ERR_INVALID_ARG;
    if (n_tok_k > 0 && (!view_ok(K, Hkv, n_tok_k, elt) || !view_ok(V, Hkv, n_tok_k, elt))) return FASTAR_ERR_INVALID_ARG;
    if (!cu_k) cu_k = cu_q;
    const View none{nullptr, 0, 0};
    const View q = view_of(Q, Hq, n_tok_q, elt), o = view_of(O, Hq, n_tok_q, elt);
    const View k = n_tok_k ? view_of(K, Hkv, n_tok_k, elt) : none, v = n_tok_k ? view_of(V, Hkv, n_tok_k, elt) : none;
    if (k.row > MAX_PITCH || v.row > MAX_PITCH) return FASTAR_ERR_UNSUPPORTED;
    const float scale_log2 = scale * 1.4426950408889634f;
    if (dtype == FASTAR_BF16)
        return launch_prompt_bf16(q, k, v, cu_q, cu_k, B, n_tok_q, n_tok_k, Hq, Hkv, d, causal, scale_log2, o, lse, (hipStream_t)stream);
    const prompt32::Args a = {q, k, v, o, cu_q, cu_k, B, n_tok_q, n_tok_k, Hkv, Hq / Hkv, causal, scale_log2, lse};
    return d == 128 ? prompt32::launch<128>(a, (hipStream_t)stream) : prompt32::launch<64>(a, (hipStream_t)stream);
}
