// Attention over packed prompts, fp32 (prompt_attn_fwd), on the fp32 matrix instructions, and the entry point for both types.
//
// A workgroup owns 64 rows of one sequence and key head ((token, head of the group) pairs), a wavefront 16 of them; tiles of 32
// keys go straight from global memory into LDS, one copy for all, two stages.  Both contractions are transposed (lane l: row
// l % 16, quarter q = l / 16) on v_mfma_f32_16x16x4_f32, whose k order is free as long as both operands agree:
//     S^T = K Q^T    A = K, lane l: key l % 16, coordinates 16 c + 4 q .. + 3 in one 16-byte read, four products
//     O^T = V^T P^T  B = the score registers as they are (product v: key 4 q + v); A = V: block 4 e + x of 16 output rows stands
//                    for coordinates 64 e + 4 (l % 16) + x, so that a lane's 16-byte read feeds four blocks
// What bounds it where the chip is full are the matrix instructions (32 cycles each, 128 per tile, nothing runs beside them).
// Launches with fewer workgroups than compute units let two teams of four wavefronts take turns at the tiles (TEAMS = 2).
#include "packed.hpp"

#include <type_traits>

namespace fastar {

int launch_prompt_bf16(const View &Q, const View &K, const View &V, const int32_t *cu_q, const int32_t *cu_k, int B, int n_tok_q,
                       int n_tok_k, int Hq, int Hkv, int d, int causal, float scale_log2, const View &O, float *lse, hipStream_t s);

namespace prompt32 {

constexpr int TK = 32;      // keys per tile
constexpr int NW = 4;       // wavefronts per team
constexpr int R = 16 * NW;  // rows per workgroup
constexpr float LN2 = 0.6931471805599453f;

__device__ __forceinline__ f32x4 mfma_16x16x4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float max_of_quarters(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_of_quarters(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// LDS reads as assembly: the compiler would wait for the tile loads in flight before each of its own.
template <int OFF>
__device__ __forceinline__ f32x4 lds_read(unsigned addr) {
    f32x4 r;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "n"(OFF));
    return r;
}
template <int N>
__device__ __forceinline__ void wait2(f32x4 &a, f32x4 &b) {
    asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(a), "+v"(b) : "n"(N));
}
template <int N>
__device__ __forceinline__ void wait1(f32x4 &a) {
    asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(a) : "n"(N));
}

struct Args {
    View Q, K, V, O;
    const int32_t *cu_q, *cu_k;
    int B, n_tok_q, n_tok_k, Hkv, group, causal;
    float scale_log2;
    float *lse;
};

template <int D, int TEAMS>
__global__ __launch_bounds__(TEAMS * NW * 64, 2) void attn_f32_prompt_kernel(const Args a) {
    constexpr int CH = D / 16, ROWB = D * 4, TILEB = TK * ROWB, CPR = ROWB / 16;
    constexpr int RPI = 1024 / ROWB, IPW = TILEB / 1024 / NW;   // rows per direct load of 1 KiB, loads per wavefront, tensor and tile
    constexpr int NT = TEAMS * NW * 64;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];   // [team][stage][K, V]
    __shared__ int s_part[TEAMS * NW], s_found[3];
    __shared__ float s_m[NW][16], s_l[NW][16];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int team = wave / NW, w = wave % NW;
    const int col = lane & 15, quarter = lane >> 4;

    int b, qt, h;   // as in prompt_attn.hip
    {
        int before = 0, found = 0;
        const int u = blockIdx.x;
        for (int b0 = 0; b0 < a.B && !found; b0 += NT) {   // uniform
            int n = 0;
            if (b0 + tid < a.B) n = (rows_of(a.cu_q, b0 + tid, a.n_tok_q).n * a.group + R - 1) / R * a.Hkv;
            int v = (int)wave_incl_scan((unsigned)n);
            __syncthreads();
            if (tid == 0) s_found[0] = -1;
            if (lane == 63) s_part[wave] = v;
            __syncthreads();
            int base = before;
#pragma unroll
            for (int i = 0; i < TEAMS * NW; ++i) {
                if (i < wave) base += s_part[i];
                before += s_part[i];
            }
            v += base;
            if (u >= v - n && u < v) {
                s_found[0] = b0 + tid;
                s_found[1] = v - n;
                s_found[2] = n;
            }
            __syncthreads();
            found = s_found[0] >= 0;
        }
        if (!found) return;
        b = __builtin_amdgcn_readfirstlane(s_found[0]);
        const int local = u - __builtin_amdgcn_readfirstlane(s_found[1]), n_qt = __builtin_amdgcn_readfirstlane(s_found[2]) / a.Hkv;
        h = local % a.Hkv;
        qt = n_qt - 1 - local / a.Hkv;
    }
    const Rows rq = rows_of(a.cu_q, b, a.n_tok_q), rk = rows_of(a.cu_k, b, a.n_tok_k);
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
    unsigned char *mine = lds + team * 4 * TILEB;
    // one 16-byte piece per lane; K's pieces are permuted within a row, piece c of row w at c ^ (w & 15)
    auto issue = [&](const char *base, int64_t pitch, unsigned char *dst, int t, bool is_k) __attribute__((always_inline)) {
        const char *tile = base + (int64_t)t * TK * pitch;
        const bool all = t * TK + TK <= n;
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const int r = RPI * (IPW * w + i) + lane / CPR;
            const int piece = (lane % CPR) ^ (is_k ? r & 15 : 0);
            const unsigned off = (unsigned)r * (unsigned)pitch + 16 * piece;
            const char *src = all || t * TK + r < n ? tile + off : base + 16 * piece;   // rows past the end: key 0, which is seen wherever a key is
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                             (__attribute__((address_space(3))) void *)(dst + (IPW * w + i) * 1024), 16, 0, 0);
        }
    };
    auto issue_tile = [&](int t, int stage) __attribute__((always_inline)) {
        if (t >= nt) return;
        issue(Kb, a.K.row, mine + stage * 2 * TILEB, t, true);
        issue(Vb, a.V.row, mine + stage * 2 * TILEB + TILEB, t, false);
    };
    const unsigned mine_lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)mine;
    const unsigned kaddr0 = mine_lds + col * ROWB + ((quarter ^ col) << 4);        // chunk c: exclusive or with 64 c
    const unsigned vaddr0 = mine_lds + TILEB + 4 * quarter * ROWB + col * 16;

    const int turns = (nt + TEAMS - 1) / TEAMS;   // the same for both teams
    issue_tile(team, 0);
    for (int i = 0; i < turns; ++i) {
        const int t = TEAMS * i + team, stage = i & 1;
        __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
        asm volatile("s_barrier" ::: "memory");   // the tile is there, and nobody reads the other stage any more
        issue_tile(t + TEAMS, stage ^ 1);
        if (t >= nt) continue;   // uniform over the team
        const unsigned kaddr = kaddr0 + stage * 2 * TILEB, vaddr = vaddr0 + stage * 2 * TILEB;
        f32x4 s[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
        {
            f32x4 kf[3][2];
            auto read = [&](int c, f32x4 (&f)[2]) __attribute__((always_inline)) {
                const unsigned at = kaddr ^ (unsigned)(64 * c);
                f[0] = lds_read<0>(at);
                f[1] = lds_read<16 * ROWB>(at);
            };
            read(0, kf[0]);
            read(1, kf[1]);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (c + 2 < CH) read(c + 2, kf[(c + 2) % 3]);
                if (c + 2 < CH) wait2<4>(kf[c % 3][0], kf[c % 3][1]);
                else if (c + 1 < CH) wait2<2>(kf[c % 3][0], kf[c % 3][1]);
                else wait2<0>(kf[c % 3][0], kf[c % 3][1]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int hb = 0; hb < 2; ++hb) s[hb] = mfma_16x16x4(kf[c % 3][hb][e], q[c][e], s[hb]);
            }
        }
        if (t * TK + TK > limit_min) {
#pragma unroll
            for (int hb = 0; hb < 2; ++hb)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (t * TK + 16 * hb + 4 * quarter + v >= limit) s[hb][v] = -INFINITY;
        }
        float mx = s[0][0];
#pragma unroll
        for (int hb = 0; hb < 2; ++hb)
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
        for (int hb = 0; hb < 2; ++hb)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                s[hb][v] = exp2f(fmaf(s[hb][v], scale_log2, neg));   // with its subnormal results: values go up to 2^128
                l += s[hb][v];
            }
        {
            f32x4 vf[3][D / 64];
            auto read = [&](auto step, f32x4 (&f)[D / 64]) __attribute__((always_inline)) {
                constexpr int row = (decltype(step)::value >> 2) * 16 + (decltype(step)::value & 3);
                f[0] = lds_read<row * ROWB>(vaddr);
                if constexpr (D == 128) f[1] = lds_read<row * ROWB + 256>(vaddr);
            };
            auto product = [&](auto step, auto behind) __attribute__((always_inline)) {
                constexpr int i = decltype(step)::value, n_behind = decltype(behind)::value * (D / 64);
                f32x4 (&f)[D / 64] = vf[i % 3];
                if constexpr (D == 128) wait2<n_behind>(f[0], f[1]);
                else wait1<n_behind>(f[0]);
#pragma unroll
                for (int e = 0; e < D / 64; ++e)
#pragma unroll
                    for (int x = 0; x < 4; ++x) o[4 * e + x] = mfma_16x16x4(f[e][x], s[i >> 2][i & 3], o[4 * e + x]);
            };
#define N(i) std::integral_constant<int, i>{}
            read(N(0), vf[0]);
            read(N(1), vf[1]);
            read(N(2), vf[2]); product(N(0), N(2));
            read(N(3), vf[0]); product(N(1), N(2));
            read(N(4), vf[1]); product(N(2), N(2));
            read(N(5), vf[2]); product(N(3), N(2));
            read(N(6), vf[0]); product(N(4), N(2));
            read(N(7), vf[1]); product(N(5), N(2));
            product(N(6), N(1));
            product(N(7), N(0));
#undef N
        }
    }
    l = sum_of_quarters(l);
    if constexpr (TEAMS == 2) {   // team 1 hands its sums to team 0
        __syncthreads();
        f32x4 *give = (f32x4 *)lds + (size_t)w * CH * 64;
        if (team == 1) {
#pragma unroll
            for (int c = 0; c < CH; ++c) give[c * 64 + lane] = o[c];
            if (quarter == 0) {
                s_m[w][col] = m;
                s_l[w][col] = l;
            }
        }
        __syncthreads();
        if (team == 1) return;
        const float mo = s_m[w][col], lo = s_l[w][col], m_all = fmaxf(m, mo);
        const float w_mine = m == -INFINITY ? 0.0f : exp2f((m - m_all) * scale_log2), w_other = mo == -INFINITY ? 0.0f : exp2f((mo - m_all) * scale_log2);
        m = m_all;
        l = l * w_mine + lo * w_other;
#pragma unroll
        for (int c = 0; c < CH; ++c) o[c] = o[c] * w_mine + give[c * 64 + lane] * w_other;
    }
    bool odd = false;
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
            a.lse[(size_t)my_head * a.n_tok_q + rq.first + my_tok] = l == 0.0f ? -INFINITY : (m * scale_log2 + __log2f(l)) * LN2;
    }
    // as in prompt_attn.hip: rows that a value which they do not see may have spoilt
    if (a.causal && __any(odd)) {
        for (int r = 0; r < 16 && row0 + r < n_rows; ++r) {
            const int rr = row0 + r, tok = rr / a.group, head = h * a.group + rr - tok * a.group;
            float mr, lr, acc[D / 64];
            row_by_keys<float, D>(a.Q.p + head * a.Q.head + (int64_t)(rq.first + tok) * a.Q.row, Kb, a.K.row, Vb, a.V.row, sees(rr), scale_log2, mr, lr, acc);
            float *op = (float *)(a.O.p + head * a.O.head + (int64_t)(rq.first + tok) * a.O.row);
#pragma unroll
            for (int c = 0; c < D / 64; ++c) op[64 * c + lane] = lr == 0.0f ? 0.0f : acc[c] / lr;
            if (lane == 0 && a.lse) a.lse[(size_t)head * a.n_tok_q + rq.first + tok] = lr == 0.0f ? -INFINITY : (mr * scale_log2 + __log2f(lr)) * LN2;
        }
    }
}

template <int D, int TEAMS>
constexpr int lds_bytes() { return TEAMS * 4 * TK * D * 4; }

template <int D>
int launch(const Args &a, int64_t items, hipStream_t s) {
    // Two teams where one leaves compute units without a workgroup; their LDS allows only one workgroup per unit.
    if (items <= 256) hipLaunchKernelGGL((attn_f32_prompt_kernel<D, 2>), dim3((unsigned)items), dim3(2 * NW * 64), (lds_bytes<D, 2>()), s, a);
    else hipLaunchKernelGGL((attn_f32_prompt_kernel<D, 1>), dim3((unsigned)items), dim3(NW * 64), (lds_bytes<D, 1>()), s, a);
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}

}  // namespace prompt32

int prompt_f32_setup() {
    using namespace prompt32;
    static DeviceOnce once;
    return once.run([](int) {
        if (hipFuncSetAttribute((const void *)attn_f32_prompt_kernel<128, 2>, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes<128, 2>()) != hipSuccess ||
            hipFuncSetAttribute((const void *)attn_f32_prompt_kernel<64, 2>, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes<64, 2>()) != hipSuccess ||
            hipFuncSetAttribute((const void *)attn_f32_prompt_kernel<128, 1>, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes<128, 1>()) != hipSuccess)
            return FASTAR_ERR_HIP;
        return FASTAR_OK;
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
    if ((int64_t)n_tok_q * Hq > INT32_MAX / 2) return FASTAR_ERR_UNSUPPORTED;
    if (n_tok_q == 0 || B == 0) return FASTAR_OK;
    if (!cu_q || !view_ok(Q, elt) || !view_ok(O, elt) || !rows_apart(O, Hq, n_tok_q, d)) return FASTAR_ERR_INVALID_ARG;
    if (n_tok_k > 0 && (!view_ok(K, elt) || !view_ok(V, elt))) return FASTAR_ERR_INVALID_ARG;
    if (n_tok_k > 0 && (K->row * elt > MAX_PITCH || V->row * elt > MAX_PITCH)) return FASTAR_ERR_UNSUPPORTED;
    if (!cu_k) cu_k = cu_q;
    const View none{nullptr, 0, 0};
    const View q = view_of(Q, elt), k = n_tok_k ? view_of(K, elt) : none, v = n_tok_k ? view_of(V, elt) : none, o = view_of(O, elt);
    const float scale_log2 = scale * 1.4426950408889634f;
    if (dtype == FASTAR_BF16)
        return launch_prompt_bf16(q, k, v, cu_q, cu_k, B, n_tok_q, n_tok_k, Hq, Hkv, d, causal, scale_log2, o, lse, (hipStream_t)stream);
    if (const int rc = prompt_f32_setup(); rc != FASTAR_OK) return rc;
    const prompt32::Args a = {q, k, v, o, cu_q, cu_k, B, n_tok_q, n_tok_k, Hkv, Hq / Hkv, causal, scale_log2, lse};
    const int64_t items = (((int64_t)n_tok_q * a.group + prompt32::R - 1) / prompt32::R + B) * Hkv;   // at most
    if (items > INT32_MAX) return FASTAR_ERR_UNSUPPORTED;
    return d == 128 ? prompt32::launch<128>(a, items, (hipStream_t)stream) : prompt32::launch<64>(a, items, (hipStream_t)stream);
}
