// Attention over packed prompts, bf16 (prompt_attn_fwd).
//
// A workgroup owns 256 rows of one sequence and key head, a row being a (token, query head of the group) pair: heads that
// share keys share the tiles, and the diagonal of a causal prompt costs the fewer masked tiles the larger the group is.
// Eight wavefronts of 32 rows each walk tiles of 64 keys.  Both contractions are transposed, S^T = K Q^T and O^T = V^T P^T, so
// that a row's softmax stays in two lanes and P^T is a matrix operand as the score registers hold it.  K and V go straight from
// global memory into LDS (one copy for all eight wavefronts; 16-byte chunks permuted within a row so that operand reads meet no
// bank twice), K is read as it is, V through the transposing LDS read.
// Launches of few workgroups (SPLIT): 128 rows each, four wavefronts for either half of their keys, put together at the end.
//
// Schedule: a SIMD runs matrix instructions of one wavefront beside vector instructions of another, so the wavefronts of a SIMD
// are kept half a tile apart.  Wavefronts 0..3 and 4..7 are two groups that take turns, a barrier per half step:
//     X(t): O += P(t-1) V(t-1), then S(t) = K(t) Q^T       (matrix instructions)
//     Y(t): loads of tile t+2, softmax of S(t) -> P(t)      (vector instructions)
// Three stages of K and four of V make room for tiles that one group still reads while the other has asked for the next ones.
// What bounds it: 3200 cycles per tile and pair of wavefronts, 2048 of them matrix instructions, at the 1.6 to 1.7 GHz that the chip
// holds under it (matrix instructions alone reach 1.73 PFLOP/s on such data): 32760 tokens x 12 heads on 4 key heads, causal,
// 2.71 to 2.80 ms = 1.2 PFLOP/s.  Short sequences add 5 us of a workgroup's ends (lengths, queries and first tiles 2.5, output 1.2).
#include "attn_lds.hpp"
#include "packed.hpp"

#include <type_traits>

namespace fastar {

namespace prompt {

using namespace attn_lds;

constexpr int TK = 64;         // keys per tile
constexpr int NWG = 4;         // wavefronts per group
// Stages of K and of V: shared by both groups, or of each group's own.
constexpr int NK = 3, NV = 4, OWN_STAGES = 2;
// Workgroups of 256 rows up to which 128 rows take a workgroup, whose two groups share their tiles: as many of them as compute
// units; causal ones up to twice that, since the first half of the rows has a quarter of the work.  256 / 128 rows, 12 heads of 128:
// 60 workgroups (1000 tokens, causal) 31.8 / 22.2 us, 156 (3000) 73.2 / 49.9, 240 (4680) 111 / 86, not causal 134 / 162; 392 (40 heads on
// 8, 2 x 1200, causal) 47 / 62.
constexpr int SPLIT_ITEMS = 128;

struct Args {
    View Q, K, V, O;
    const int32_t *cu_q, *cu_k;
    int B, n_tok_q, n_tok_k, Hkv, group, causal;
    float scale_log2;
    float *lse;
};

template <int D, bool SPLIT>
__global__ __launch_bounds__(2 * NWG * 64, 1) void attn_bf16_kernel(const Args a) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];   // [K stages][V stages]
    constexpr int KF = D / 16, DB = D / 32, ROWB = D * 2, TILEB = TK * ROWB;
    constexpr int OS_SPLIT = NWG * (DB * 4 + 1) * 1024;   // behind the sums that group 1 hands over
    constexpr int R = SPLIT ? 128 : 256, NK = SPLIT ? OWN_STAGES : prompt::NK, NV = SPLIT ? OWN_STAGES : prompt::NV;
    constexpr int IPW = TILEB / 1024 / (SPLIT ? NWG : 2 * NWG);   // direct loads of 1 KiB per wavefront, tensor and tile
    constexpr int RPI = 1024 / ROWB;                // rows that one of them brings
    constexpr int CPR = ROWB / 16;                  // 16-byte chunks per row
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = wave / NWG, part = SPLIT ? wave % NWG : wave;   // part: of the rows and of a tile's loads
    const int col = lane & 31, g = lane >> 5;

    // workgroup -> (sequence, tile of rows, head): sequences in order, of each the last rows first (they have the most keys),
    // heads next to each other
    Item it;
    if (!find_item<R>(a.cu_q, a.cu_k, a.B, a.n_tok_q, a.n_tok_k, a.group, a.Hkv, blockIdx.x, it)) return;
    const int h = it.local % a.Hkv, qt = it.n / a.Hkv - 1 - it.local / a.Hkv;
    const Rows rq = it.q, rk = it.k;
    const int n_rows = rq.n * a.group, n = rk.n;
    // keys that row r sees; rising with r
    auto sees = [&](int r) { return a.causal ? min(max(n - rq.n + min(r, n_rows - 1) / a.group + 1, 0), n) : n; };
    const int nt_all = (sees(qt * R + R - 1) + TK - 1) / TK;   // tiles of the workgroup; of this group: nt from t0 on
    const int nt0 = SPLIT ? (nt_all + 1) / 2 : nt_all, nt1 = SPLIT ? nt_all - nt0 : nt_all;
    const int nt = grp == 0 ? nt0 : nt1, t0 = SPLIT && grp == 1 ? nt0 : 0;
    const int row0 = qt * R + part * 32;                       // rows of the wavefront
    const int limit_min = sees(row0);   // what its first row sees
    const int my_row = min(row0 + col, n_rows - 1);
    const int my_tok = my_row / a.group, my_head = h * a.group + my_row - my_tok * a.group;
    const int limit = sees(my_row);

    bf16x8 qf[KF];
    {
        const char *qp = a.Q.p + my_head * a.Q.head + (int64_t)(rq.first + my_tok) * a.Q.row;
#pragma unroll
        for (int s = 0; s < KF; ++s) qf[s] = *(const bf16x8 *)(qp + (16 * s + 8 * g) * 2);
    }
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[db][v] = 0.0f;
    float m = -INFINITY, neg = 0.0f, l0 = 0.0f, l1 = 0.0f;
    const float scale_log2 = a.scale_log2;

    // ---- tile loads: instruction i of this wavefront brings tile rows RPI (IPW wave + i) .., lane l row + l / CPR, chunk l % CPR
    // of LDS; which chunk of the row that is in global memory is permuted by the row
    unsigned char *kbuf = lds + (SPLIT ? grp * 2 * OWN_STAGES * TILEB : 0), *vbuf = kbuf + NK * TILEB;
    const char *Kb = a.K.p + h * a.K.head + (int64_t)rk.first * a.K.row, *Vb = a.V.p + h * a.V.head + (int64_t)rk.first * a.V.row;
    auto swz_k = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
    // a transposing read takes 64 bytes of four rows at a time: a quarter of the banks each
    auto swz_v = [](int row) { return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; };
    unsigned koff[IPW], voff[IPW];
#pragma unroll
    for (int i = 0; i < IPW; ++i) {
        const int r = RPI * (IPW * part + i) + lane / CPR;
        koff[i] = (unsigned)r * (unsigned)a.K.row + 16 * ((lane % CPR) ^ swz_k(r));
        voff[i] = (unsigned)r * (unsigned)a.V.row + 16 * ((lane % CPR) ^ swz_v(r));
    }
    auto issue = [&](const char *base, int64_t pitch, const unsigned (&off)[IPW], unsigned char *dst, int t) __attribute__((always_inline)) {
        if (t * TK + TK <= n) {   // uniform
            const char *tile = base + (int64_t)t * TK * pitch;
#pragma unroll
            for (int i = 0; i < IPW; ++i) to_lds(tile, off[i], lds_address(dst) + (IPW * part + i) * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < IPW; ++i) {   // rows past the end: key 0, which is seen wherever a key is
                const int r = RPI * (IPW * part + i) + lane / CPR;
                to_lds(base + off[i] + (t * TK + r < n ? (int64_t)t * TK * pitch : -(int64_t)r * pitch), dst + (IPW * part + i) * 1024);
            }
        }
    };
    auto issue_k = [&](int t) __attribute__((always_inline)) { if (t < nt) issue(Kb, a.K.row, koff, kbuf + (t % NK) * TILEB, t0 + t); };
    auto issue_v = [&](int t) __attribute__((always_inline)) { if (t < nt) issue(Vb, a.V.row, voff, vbuf + (t % NV) * TILEB, t0 + t); };

    // per-lane LDS addresses of the operands
    const unsigned kbuf_lds = lds_address(kbuf), vbuf_lds = lds_address(vbuf);
    const int s16 = lane & 15, l16 = lane >> 4;
    const int vrow = 4 * (l16 >> 1) + (s16 >> 2);
    // K's first 16 coordinates (the s-th: exclusive or with 32 s), V's first 32 (the db-th: with 64 db)
    unsigned kaddr = kbuf_lds + col * ROWB + ((g ^ swz_k(col)) << 4);
    unsigned vaddr = vbuf_lds + vrow * ROWB + (((2 * (l16 & 1) + ((s16 & 3) >> 1)) ^ swz_v(vrow)) << 4) + (s16 & 1) * 8;
    int ks = 0, vs = 0;   // stages that kaddr and vaddr point into

    f32x16 s_acc[2];
    bf16x8 pf[2][2];
    s16x4 va[2][DB][2];
    float mx_tile = -INFINITY;
    auto phase_x = [&](int t, auto pv_c, auto qk_c) __attribute__((always_inline)) {
        constexpr bool PV = decltype(pv_c)::value, QK = decltype(qk_c)::value;
        __builtin_amdgcn_s_setprio(2);
        s16x4 vb[2][DB][2];
        bf16x8 ka[KF], kb[KF];
        if constexpr (PV) read_vt<32 * ROWB, ROWB>(vb, vaddr);
        if constexpr (QK) read_k<0>(ka, kaddr);
        if constexpr (PV) {
            pv_mfma(o, va, pf[0]);
            wait_v<QK ? KF : 0>(vb);
            pv_mfma(o, vb, pf[1]);
            vaddr += vs == NV - 1 ? -(NV - 1) * TILEB : TILEB;
            vs = vs == NV - 1 ? 0 : vs + 1;
        }
        if constexpr (QK) {
            read_k<32 * ROWB>(kb, kaddr);
            wait_k<KF>(ka);
#pragma unroll
            for (int v = 0; v < 16; ++v) s_acc[0][v] = s_acc[1][v] = 0.0f;
#pragma unroll
            for (int s = 0; s < KF; ++s) s_acc[0] = mfma_bf16_32x32x16(ka[s], qf[s], s_acc[0]);
            wait_k<0>(kb);
            __builtin_amdgcn_sched_barrier(0);
            kaddr += ks == NK - 1 ? -(NK - 1) * TILEB : TILEB;
            ks = ks == NK - 1 ? 0 : ks + 1;
#pragma unroll
            for (int s = 0; s < KF; ++s) s_acc[1] = mfma_bf16_32x32x16(kb[s], qf[s], s_acc[1]);
            __builtin_amdgcn_sched_barrier(0);
            const int key0 = (t0 + t) * TK;
            if (key0 + TK > limit_min) {   // uniform: some row of the wavefront does not see some key of the tile
#pragma unroll
                for (int hb = 0; hb < 2; ++hb)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (key0 + 32 * hb + 8 * (v >> 2) + 4 * g + (v & 3) >= limit) s_acc[hb][v] = -INFINITY;
            }
            float mx = s_acc[0][0];
#pragma unroll
            for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s_acc[0][v]);
#pragma unroll
            for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s_acc[1][v]);
            mx_tile = max_across_halves(mx);
            asm volatile("" : "+v"(s_acc[0]), "+v"(s_acc[1]), "+v"(mx_tile));
        }
        __builtin_amdgcn_s_setprio(0);
    };
    auto phase_y = [&](int t) __attribute__((always_inline)) {
        issue_k(t + 2);
        issue_v(SPLIT ? t + 1 : t + 2);
        // The reference may lag the maximum by 8 octaves.  The maximum itself (error of the output 0.0018 to 0.0020 instead of 0.0020 to
        // 0.0022 on the same inputs, 0.0016 of either its rounding) rescales sums in most tiles: 14 ragged prompts 357 us instead of 337, 32760 tokens 2.90 ms instead of 2.79; a lag of 3
        // octaves 346 and 2.80.  Sums of the rounded weights beside those that lse needs, for a row's own key to have weight 1: 349 and 2.91.
        if (__any((mx_tile - m) * scale_log2 > 8.0f)) {
            const float mn = fmaxf(m, mx_tile);
            const float alpha = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - mn) * scale_log2);
            m = mn;
            neg = mn == -INFINITY ? 0.0f : -mn * scale_log2;
            l0 *= alpha;
            l1 *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
        }
#pragma unroll
        for (int hb = 0; hb < 2; ++hb)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                bf16x2 pr[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p0 = __builtin_amdgcn_exp2f(fmaf(s_acc[hb][8 * hh + 2 * j], scale_log2, neg));
                    const float p1 = __builtin_amdgcn_exp2f(fmaf(s_acc[hb][8 * hh + 2 * j + 1], scale_log2, neg));
                    l0 += p0;
                    l1 += p1;
                    pr[j][0] = (__bf16)p0;
                    pr[j][1] = (__bf16)p1;
                }
                __builtin_memcpy(&pf[hb][hh], pr, 16);
            }
        asm volatile("" : "+v"(pf[0][0]), "+v"(pf[0][1]), "+v"(pf[1][0]), "+v"(pf[1][1]), "+v"(l0), "+v"(l1));
        read_vt<0, ROWB>(va, vaddr);
        wait_v<0>(va);
    };
    auto landed = [&]() __attribute__((always_inline)) {   // this wavefront's loads are there before the barrier that publishes them
        __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
        wg_barrier();
    };

    // Half steps: group 0 runs X(t) in half step 2t and Y(t) in 2t+1, group 1 one later.  K(t) is read in half steps 2t and 2t+1,
    // V(t) in 2t+1 .. 2t+3; Y(t) asks for K(t+2) (stage of K(t-1)) and V(t+2) (stage of V(t-2)), and what it asked for is
    // waited for before the barrier into Y(t+1): group 1's at the start of half step 2t+4, when K(t+2) is first read.
    // SPLIT: a group reads only what it has asked for itself; Y(t) asks for K(t+2) (stage of K(t)) and V(t+1) (of V(t-1)), both of
    // which X(t) was the last to read.
    const int n_bar = max(nt0 > 0 ? 2 * nt0 + 1 : 0, nt1 > 0 ? 2 * nt1 + 2 : 1) + 1;   // barriers that every wavefront passes
    int done = 0;
    if (nt > 0) {
        issue_k(0);
        issue_v(0);
        issue_k(1);
        if constexpr (!SPLIT) issue_v(1);
    }
    landed();
    if (grp == 1) {
        wg_barrier();
        ++done;
    }
    if (nt > 0) {
        phase_x(0, std::false_type{}, std::true_type{});
        for (int t = 0; t < nt - 1; ++t) {
            landed();
            phase_y(t);
            wg_barrier();
            phase_x(t + 1, std::true_type{}, std::true_type{});
        }
        landed();
        phase_y(nt - 1);
        wg_barrier();
        phase_x(nt, std::true_type{}, std::false_type{});
        done += 2 * nt;
    }
    for (++done; done < n_bar; ++done) wg_barrier();

    const float l_lane = l0 + l1;
    float l = l_lane + shfl_xor(l_lane, 32);
    if constexpr (SPLIT) {   // group 1 hands its sums to group 0
        __syncthreads();   // the tiles are dead
        f32x4 *give = (f32x4 *)lds + (size_t)part * (DB * 4 + 1) * 64;
        if (grp == 1) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) give[(db * 4 + q4) * 64 + lane] = f32x4{o[db][4 * q4], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]};
            give[DB * 4 * 64 + lane] = f32x4{m, l, 0.0f, 0.0f};
        }
        __syncthreads();
        if (grp == 1) return;
        const f32x4 ml = give[DB * 4 * 64 + lane];
        const float m_all = fmaxf(m, ml[0]);
        const float w_mine = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - m_all) * scale_log2);
        const float w_other = ml[0] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((ml[0] - m_all) * scale_log2);
        m = m_all;
        l = l * w_mine + ml[1] * w_other;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const f32x4 x = give[(db * 4 + q4) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[db][4 * q4 + e] = o[db][4 * q4 + e] * w_mine + x[e] * w_other;
            }
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    bool odd = !sums_up(m, l);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) odd |= !(fabsf(o[db][v]) < INFINITY);
    // LDS takes the rows of the output, a wavefront's own each, so that they are stored whole
    constexpr int OSTR = D + 8;
    unsigned short *Os = (unsigned short *)(lds + (SPLIT ? OS_SPLIT : 0)) + (size_t)part * 32 * OSTR;
    if constexpr (!SPLIT) __syncthreads();   // the tiles are dead
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            const bf16x4 w = {(__bf16)(o[db][4 * q4] * inv), (__bf16)(o[db][4 * q4 + 1] * inv), (__bf16)(o[db][4 * q4 + 2] * inv),
                              (__bf16)(o[db][4 * q4 + 3] * inv)};
            *(bf16x4 *)(Os + col * OSTR + 32 * db + 8 * q4 + 4 * g) = w;
        }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < 32 * CPR / 64; ++i) {
        const int r = i * (64 / CPR) + lane / CPR, rr = row0 + r;
        if (rr < n_rows) {
            const int tok = rr / a.group, head = h * a.group + rr - tok * a.group;
            *(u32x4 *)(a.O.p + head * a.O.head + (int64_t)(rq.first + tok) * a.O.row + (lane % CPR) * 16) = *(const u32x4 *)(Os + r * OSTR + (lane % CPR) * 8);
        }
    }
    if (a.lse && g == 0 && row0 + col < n_rows)
        a.lse[(size_t)my_head * a.n_tok_q + rq.first + my_tok] = lse_of(m, l, scale_log2);
    // Sums that are not finite, or none: a value that a row does not see, or key 0's, which fills up the last tile, may have come in as 0 * x
    // (a product of tiles has no other way), or weights, or weights times values, have left the range.  Those rows are done again one by one, over
    // the keys that they see and with weights that add up to one; where all rows see all keys, only if the sums may be wrong.
    if (__builtin_expect(__any(odd), 0)) {
        const Args a = args_anew<Args>();
        const char *K = a.K.p + h * a.K.head + (int64_t)rk.first * a.K.row, *V = a.V.p + h * a.V.head + (int64_t)rk.first * a.V.row;
        if (!a.causal && !__any(!sums_up(m, l) && !no_number(m, l, a.scale_log2)) && sums_stand<__bf16, D>(V, a.V.row, n, n % TK != 0)) return;
        for (int r = 0; r < 32 && row0 + r < n_rows; ++r) {
            const int rr = row0 + r, tok = rr / a.group, head = h * a.group + rr - tok * a.group;
            float mr, lr, acc[D / 64];
            row_by_keys<__bf16, D>(a.Q.p + head * a.Q.head + (int64_t)(rq.first + tok) * a.Q.row, K, a.K.row, V, a.V.row,
                                   a.causal ? min(max(n - rq.n + tok + 1, 0), n) : n, a.scale_log2, mr, lr, acc);
            __bf16 *op = (__bf16 *)(a.O.p + head * a.O.head + (int64_t)(rq.first + tok) * a.O.row);
#pragma unroll
            for (int c = 0; c < D / 64; ++c) op[64 * c + lane] = (__bf16)acc[c];
            if (lane == 0 && a.lse) a.lse[(size_t)head * a.n_tok_q + rq.first + tok] = lse_of(mr, lr, a.scale_log2);
        }
    }
}

template <int D, bool SPLIT>
constexpr int lds_bytes() { return (SPLIT ? 4 * OWN_STAGES : NK + NV) * TK * D * 2; }
static_assert(NWG * (4 * 4 + 1) * 1024 + NWG * 32 * (128 + 8) * 2 <= lds_bytes<128, true>() && NWG * (2 * 4 + 1) * 1024 + NWG * 32 * (64 + 8) * 2 <= lds_bytes<64, true>(),
              "sums and rows fit");

template <int D, bool SPLIT>
int setup() {
    return hipFuncSetAttribute((const void *)attn_bf16_kernel<D, SPLIT>, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes<D, SPLIT>()) == hipSuccess ? FASTAR_OK : FASTAR_ERR_HIP;
}
template <int D, bool SPLIT>
int launch(const Args &a, int64_t items, hipStream_t s) {
    hipLaunchKernelGGL((attn_bf16_kernel<D, SPLIT>), dim3((unsigned)items), dim3(2 * NWG * 64), (lds_bytes<D, SPLIT>()), s, a);
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}

}  // namespace prompt

int prompt_setup() {
    static DeviceOnce once;
    return once.run([](int) {
        const int rc = prompt::setup<128, false>();
        return rc == FASTAR_OK ? prompt::setup<128, true>() : rc;
    });
}

int launch_prompt_bf16(const View &Q, const View &K, const View &V, const int32_t *cu_q, const int32_t *cu_k, int B, int n_tok_q,
                       int n_tok_k, int Hq, int Hkv, int d, int causal, float scale_log2, const View &O, float *lse, hipStream_t s) {
    using namespace prompt;
    const Args a = {Q, K, V, O, cu_q, cu_k, B, n_tok_q, n_tok_k, Hkv, Hq / Hkv, causal, scale_log2, lse};
    auto items = [&](int rows) { return (((int64_t)n_tok_q * a.group + rows - 1) / rows + B) * Hkv; };   // at most
    if (!launch_ok(items(256), 2 * NWG * 64)) return FASTAR_ERR_UNSUPPORTED;
    if (const int rc = prompt_setup(); rc != FASTAR_OK) return rc;
    const bool split = items(256) <= (causal ? 2 : 1) * SPLIT_ITEMS;
    if (d == 128) return split ? launch<128, true>(a, items(128), s) : launch<128, false>(a, items(256), s);
    return split ? launch<64, true>(a, items(128), s) : launch<64, false>(a, items(256), s);
}

}  // namespace fastar
