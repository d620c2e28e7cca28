// Attention of packed queries over a paged cache of E4M3 codes (paged_attn_fwd): the kernel for chunks of many rows.
//
// prompt_attn.hip's schedule -- 256 rows per workgroup, two groups of four wavefronts half a tile apart -- over tiles that come
// from pages.  A wavefront of paged_attn.hip widens every code it multiplies with; here a tile's codes are widened once for all
// eight wavefronts: each takes an eighth of the tile, 16 bytes of K and of V per lane, into registers, and writes it to LDS as bf16 a
// tile later, in the matrix phase (in the vector phase, which is the longer one, 505 us where this takes 460).  V's cells hold a
// coordinate's 16 tokens, so V lies transposed in LDS and is read as it is; within 16 tokens the order is 0-3, 8-11, 4-7, 12-15,
// which is the order that half a wavefront holds P in.  The items' tiles are dealt out as in paged_dev.hpp, a workgroup per compute
// unit.  What bounds it: the two phases' instructions, 4000 cycles per tile and pair of wavefronts, 2048 of them matrix instructions;
// rows that no token fills (8 % of five chunks of 201 to 780 tokens x 3 heads); 14 us of fragments.  Those chunks over caches of 4680
// to 37440 keys x 4 key heads: 430 to 460 us from box to box, 840 to 900 TFLOP/s (paged_attn.hip's way with 64 rows per wavefront took 790).
#include "attn_lds.hpp"
#include "paged_dev.hpp"

#include <type_traits>

namespace fastar {

namespace paged {

namespace chunk {

using namespace attn_lds;

constexpr int NWG = 4;         // wavefronts per group
constexpr int R = 256;         // rows per item
constexpr int NK = 2, NV = 3;  // stages
constexpr int SHARES = 256;
// Units of a share at least (tiles, and the ENDS in front of an item's): a fragment costs as much as some tiles.  4 / 8 / 16 / 32: 100 tokens x
// 12 heads on 4 x 2000 keys 27 / 31 / 43 / 67 us, 300 on 9000 68 / 68 / 52 / 76, 130 x 4 heads on one x 100000 94 / 95 / 95 / 99.
constexpr int LEAST = 8;
constexpr int FEW_KEYS = 512;  // longer tables are cut while items leave compute units idle (100 tokens x 12 heads on 4 x 2000 keys 72 us whole, 31 cut)
constexpr int FRAG_FLOATS = R * 128 + 2 * R;
static_assert(SHARES <= MAX_SHARES, "descriptors");

template <int D>
constexpr int lds_bytes() { return (NK + NV) * TK * D * 2; }

template <int D, bool SPLIT>
__global__ __launch_bounds__(2 * NWG * 64, 1) void attn_chunk_kernel(const Args a) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];   // [K stages: a row per key][V stages: a row per coordinate]
    constexpr int KF = D / 16, DB = D / 32, ROWB = D * 2, TILEB = TK * ROWB, VROWB = TK * 2, CPR = ROWB / 16;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = wave / NWG;
    const int col = lane & 31, g = lane >> 5;
    const int Hkv = a.pg.Hkv;
    const float scale_log2 = a.scale_log2;
    unsigned char *kbuf = lds, *vbuf = lds + NK * TILEB;
    const unsigned kbuf_lds = lds_address(kbuf), vbuf_lds = lds_address(vbuf);
    auto swz_k = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
    auto swz_v = [](int row) { return (row >> 1) & 7; };

    // this lane's piece of a tile: token block and coordinate block of its cell, row of the cell.  d = 128: of K and of V; d = 64:
    // wavefronts 0..3 bring K, 4..7 V
    const int tb = D == 128 ? wave >> 1 : wave & 3, cb = D == 128 ? (wave & 1) * 4 + (lane >> 4) : lane >> 4, cr = lane & 15;
    const bool has_k = D == 128 || wave < 4, has_v = D == 128 || wave >= 4;
    const int blk_mask = (1 << (a.pshift - 4)) - 1;
    const size_t page_bytes = (size_t)D << a.pshift;
    const unsigned piece = (unsigned)(((tb & blk_mask) * (D / 16) + cb) * 256 + cr * 16);
    const unsigned kw = (unsigned)((16 * tb + cr) * ROWB + (((2 * cb) ^ swz_k(16 * tb + cr)) << 4));   // where it goes: 16 coordinates of a key
    const unsigned vw = (unsigned)((16 * cb + cr) * VROWB + (((2 * tb) ^ swz_v(16 * cb + cr)) << 4));  // 16 tokens of a coordinate

    Range r;
    Seq sq;
    if (!first_unit<R, SPLIT>(a, SHARES, LEAST, r, sq)) {
        if (SPLIT && tid == 0) a.desc[r.share].last = -1;
        return;
    }
    Desc d = {0, 0, 0, -1};
    while (r.u < r.u_end) {   // uniform: one piece of one item per turn
        if (SPLIT && r.u >= r.base + (long long)sq.n_qt * Hkv * (sq.n_tiles + ENDS)) find_unit<R, SPLIT>(a, r.u, r.b, r.base, sq);
        const PieceOf its = next_piece<SPLIT>(r, sq);
        if (its.te <= its.ta) continue;
        const int h = its.h, qt = its.qt, ta = its.ta, te = its.te;
        const bool begins = ta == 0, ends = te == sq.n_tiles, whole = !SPLIT || (begins && ends);

        const int n_rows = sq.n_q * a.group;
        auto sees = [&](int x) {
            return a.causal ? min(max(sq.L - sq.n_q + min(x, n_rows - 1) / a.group + 1, 0), sq.L) : sq.L;
        };
        const int limit_max = sees(qt * R + R - 1);
        const int t_end = min(te, (limit_max + TK - 1) / TK);   // tiles ta .. t_end - 1
        const int row0 = qt * R + wave * 32;
        const int limit_min = sees(row0);   // what the wavefront's first row sees
        const int my_row = min(row0 + col, n_rows - 1);
        const int my_tok = my_row / a.group, my_head = h * a.group + my_row - my_tok * a.group;
        const int limit = sees(my_row);
        const int32_t *pages = a.table + (size_t)r.b * a.max_pages;
        const int last_page = max((limit_max - 1) >> a.pshift, 0);

        bf16x8 qf[KF];
        {
            const char *qp = a.Q.p + my_head * a.Q.head + (int64_t)(sq.q0 + my_tok) * a.Q.row;
#pragma unroll
            for (int s = 0; s < KF; ++s) qf[s] = *(const bf16x8 *)(qp + (16 * s + 8 * g) * 2);
        }
        f32x16 o[DB];
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[db][v] = 0.0f;
        float m = -INFINITY, neg = 0.0f, l0 = 0.0f, l1 = 0.0f;

        // ---- tiles: page numbers of their four blocks of 16 tokens (lane % 4), then this lane's codes, then LDS ----
        auto ids_of = [&](int t) __attribute__((always_inline)) { return pages[min((t * TK + 16 * (lane & 3)) >> a.pshift, last_page)]; };
        u32x4 kr, vr;
        float ks, vs;
        bool ok;
        int kput = 0, vput = 0;   // stages that the next tile goes to, in bytes
        const unsigned page_stride = (unsigned)(Hkv * page_bytes);   // of all heads
        const uint8_t *K8 = a.pg.K8 + h * page_bytes, *V8 = a.pg.V8 + h * page_bytes;
        const float *kscale = a.pg.kscale + h, *vscale = a.pg.vscale + h;
        auto fetch = [&](int ids) __attribute__((always_inline)) {   // returns which blocks' pages exist
            int id = __builtin_amdgcn_readlane(ids, tb);
            ok = page_exists(a, id);
            id = ok ? id : 0;
            const size_t at = (size_t)(unsigned)id * page_stride;
            if (has_k) {
                kr = *(const u32x4 *)(K8 + at + piece);
                ks = kscale[(size_t)(unsigned)id * (unsigned)Hkv];
            }
            if (has_v) {
                vr = *(const u32x4 *)(V8 + at + piece);
                vs = vscale[(size_t)(unsigned)id * (unsigned)Hkv];
            }
            return (int)(__ballot(page_exists(a, ids)) & 15);
        };
        auto put = [&](int t) __attribute__((always_inline)) {
            if (has_k) {
                unsigned char *p = kbuf + kput;
                *(bf16x8 *)(p + kw) = widen(kr[0], kr[1], ks);
                *(bf16x8 *)(p + (kw ^ 16)) = widen(kr[2], kr[3], ks);
            }
            if (has_v) {
                const int live = ok ? limit_max - (t * TK + 16 * tb) : 0;
                if (live < 16) {   // uniform; values that no row sees need not be numbers, nor page 0's scale
                    vr &= first_bytes(live);
                    if (!ok) vs = 1.0f;
                }
                unsigned char *p = vbuf + vput;
                *(bf16x8 *)(p + vw) = widen(vr[0], vr[2], vs);
                *(bf16x8 *)(p + (vw ^ 16)) = widen(vr[1], vr[3], vs);
            }
            kput = kput == (NK - 1) * TILEB ? 0 : kput + TILEB;
            vput = vput == (NV - 1) * TILEB ? 0 : vput + TILEB;
        };

        // per-lane LDS addresses of the operands: of K's first 16 coordinates (the s-th: exclusive or with 32 s), of V's first 16 tokens
        // (the i-th: with 32 i)
        unsigned kaddr = kbuf_lds + col * ROWB + ((g ^ swz_k(col)) << 4), vaddr = vbuf_lds + col * VROWB + ((g ^ swz_v(col)) << 4);
        int kst = 0, vst = 0;   // stages that they point into

        f32x16 s_acc[2];
        bf16x8 pf[2][2], va[2][DB];
        float mx_tile = -INFINITY;
        auto read_v = [&](int hb, bf16x8 (&f)[2][DB]) __attribute__((always_inline)) {
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const unsigned at = vaddr ^ (32 * (2 * hb + st));
                f[st][0] = lds_read_b128<0>(at);
                f[st][1] = lds_read_b128<32 * VROWB>(at);
                if constexpr (DB == 4) {
                    f[st][2] = lds_read_b128<64 * VROWB>(at);
                    f[st][3] = lds_read_b128<96 * VROWB>(at);
                }
            }
        };
        auto pv = [&](const bf16x8 (&f)[2][DB], const bf16x8 (&p)[2]) __attribute__((always_inline)) {
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int db = 0; db < DB; ++db) o[db] = mfma_bf16_32x32x16(f[st][db], p[st], o[db]);
        };
        // on their way: page numbers of tile t + 2 (ids), codes of tile t + 1 (registers); which pages of tiles t and t + 1 exist
        int ids = 0, e1 = 15, e2 = 15;
        auto phase_x = [&](int t, auto pv_c, auto qk_c) __attribute__((always_inline)) {
            constexpr bool PV = decltype(pv_c)::value, QK = decltype(qk_c)::value;
            __builtin_amdgcn_s_setprio(2);
            bf16x8 vb[2][DB], ka[KF], kb[KF];
            if constexpr (PV) read_v(1, vb);
            if constexpr (QK) read_k<0>(ka, kaddr);
            const int exist = e1;
            if constexpr (PV) {
                pv(va, pf[0]);
                if constexpr (QK) {
                    if (t + 1 < t_end) put(t + 1);
                    e1 = e2;
                    if (t + 2 < t_end) e2 = fetch(ids);
                    if (t + 3 < t_end) ids = ids_of(t + 3);
                }
                wait_b<QK ? KF : 0>(vb);
                pv(vb, pf[1]);
                vaddr += vst == NV - 1 ? -(NV - 1) * TILEB : TILEB;
                vst = vst == NV - 1 ? 0 : vst + 1;
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
                kaddr += kst == NK - 1 ? -(NK - 1) * TILEB : TILEB;
                kst = kst == NK - 1 ? 0 : kst + 1;
#pragma unroll
                for (int s = 0; s < KF; ++s) s_acc[1] = mfma_bf16_32x32x16(kb[s], qf[s], s_acc[1]);
                __builtin_amdgcn_sched_barrier(0);
                if (t * TK + TK > limit_min || exist != 15) {   // uniform: some row of the wavefront does not see some key of the tile
#pragma unroll
                    for (int hb = 0; hb < 2; ++hb)
#pragma unroll
                        for (int v = 0; v < 16; ++v)
                            if (t * TK + 32 * hb + 8 * (v >> 2) + 4 * g + (v & 3) >= limit || !(exist >> (2 * hb + (v >> 3)) & 1)) s_acc[hb][v] = -INFINITY;
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
        auto phase_y = [&]() __attribute__((always_inline)) {
            // The reference is the maximum itself, as in paged_attn.hip: weights near 1 lose least when they are rounded to bf16.  Chunks
            // of 201 to 780 tokens over caches of up to 37440 an error of 0.0018 of the output (0.0017 to 0.0019 by the inputs)
            // where a reference that may lag 8 octaves has 0.0020 on the same inputs, for 434 us instead of 429.
            if (__any(mx_tile > m)) {
                const float mn = fmaxf(m, mx_tile);
                const float alpha = weight_of(m, mn, scale_log2);
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
            read_v(0, va);
            wait_b<0>(va);
        };
        // Half steps as in prompt_attn.hip.  X(t) writes tile t + 1 (half steps 2t and 2t+1), whose K group 0 reads from 2t+2 on; the
        // stages are those of K(t-1) and V(t-2), last read in half step 2t-1.  Tiles ta and ta + 1 are written before the first.
        if (ta < t_end) {
            const int i0 = ids_of(ta), i1 = ids_of(ta + 1), i2 = ids_of(ta + 2);
            ids = ids_of(ta + 3);
            e1 = fetch(i0);
            put(ta);
            int of_next = 15;
            if (ta + 1 < t_end) {
                of_next = fetch(i1);
                put(ta + 1);
            }
            if (ta + 2 < t_end) e2 = fetch(i2);
            wg_barrier();
            if (grp == 1) wg_barrier();
            phase_x(ta, std::false_type{}, std::true_type{});
            e1 = of_next;
            for (int t = ta; t < t_end - 1; ++t) {
                wg_barrier();
                phase_y();
                wg_barrier();
                phase_x(t + 1, std::true_type{}, std::true_type{});
            }
            wg_barrier();
            phase_y();
            wg_barrier();
            phase_x(t_end, std::true_type{}, std::false_type{});
            if (grp == 0) wg_barrier();
        }

        // rows anew, so that the loop need not hold them in registers
        int qt_e = qt, lane_e = lane;
        asm volatile("" : "+s"(qt_e), "+v"(lane_e));
        const int row0_e = qt_e * R + wave * 32, col_e = lane_e & 31, g_e = lane_e >> 5;
        const int my_row_e = min(row0_e + col_e, n_rows - 1);
        const int my_tok_e = my_row_e / a.group, my_head_e = h * a.group + my_row_e - my_tok_e * a.group;
        const float l_lane = l0 + l1;
        const float l = l_lane + shfl_xor(l_lane, 32);
        bool odd = !sums_up(m, l);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) odd |= !(fabsf(o[db][v]) < INFINITY);
        __syncthreads();   // the tiles are dead
        float *frag = a.frag + (size_t)(2 * r.share + (begins ? 1 : 0)) * FRAG_FLOATS;
        if (whole) {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            constexpr int OSTR = D + 8;
            unsigned short *Os = (unsigned short *)lds + (size_t)wave * 32 * OSTR;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const bf16x4 w = {(__bf16)(o[db][4 * q4] * inv), (__bf16)(o[db][4 * q4 + 1] * inv), (__bf16)(o[db][4 * q4 + 2] * inv),
                                      (__bf16)(o[db][4 * q4 + 3] * inv)};
                    *(bf16x4 *)(Os + col_e * OSTR + 32 * db + 8 * q4 + 4 * g_e) = w;
                }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 32 * CPR / 64; ++i) {
                const int x = i * (64 / CPR) + lane_e / CPR, rr = row0_e + x;
                if (rr < n_rows) {
                    const int tok = rr / a.group, head = h * a.group + rr - tok * a.group;
                    *(u32x4 *)(a.O.p + head * a.O.head + (int64_t)(sq.q0 + tok) * a.O.row + (lane_e % CPR) * 16) = *(const u32x4 *)(Os + x * OSTR + (lane_e % CPR) * 8);
                }
            }
            if (a.lse && g_e == 0 && row0_e + col_e < n_rows)
                a.lse[(size_t)my_head_e * a.n_tok + sq.q0 + my_tok_e] = lse_of(m, l, scale_log2);
        } else {   // [wavefront][block of 32 coordinates][q4][lane_e] of four floats, then maxima and sums
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const f32x4 x = {o[db][4 * q4], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]};
                    ((f32x4 *)frag)[((wave * DB + db) * 4 + q4) * 64 + lane_e] = x;
                }
            if (g_e == 0) {
                frag[R * D + wave * 32 + col_e] = m;
                frag[R * D + R + wave * 32 + col_e] = l;
            }
        }
        // as in paged_attn.hip: rows whose sums are not finite, or none
        if (__builtin_expect(__any(odd), 0)) {
            const Args a = args_anew<Args>();
            const int32_t *pages = a.table + (size_t)r.b * a.max_pages;
            float *frag = a.frag + (size_t)(2 * r.share + (begins ? 1 : 0)) * FRAG_FLOATS;
            const bool again = (a.causal && sq.n_q > 1) || __any(!sums_up(m, l) && !no_number(m, l, a.scale_log2)) ||
                               !paged_sums_stand(a, pages, h, ta * TK, min(sq.L, te * TK));
            __threadfence();
            for (int x = 0; again && x < 32 && row0_e + x < n_rows; ++x) {
                const int rr = row0_e + x, tok = rr / a.group, head = h * a.group + rr - tok * a.group;
                float mr, lr, acc[D / 64];
                row_by_paged_keys<D>(a, a.Q.p + head * a.Q.head + (int64_t)(sq.q0 + tok) * a.Q.row, pages, h, ta * TK, min(a.causal ? min(max(sq.L - sq.n_q + tok + 1, 0), sq.L) : sq.L, te * TK), mr, lr, acc);
#pragma unroll
                for (int c = 0; c < D / 64; ++c) {
                    const int co = 64 * c + lane_e;
                    if (whole) ((__bf16 *)(a.O.p + head * a.O.head + (int64_t)(sq.q0 + tok) * a.O.row))[co] = (__bf16)acc[c];
                    else frag[(((wave * DB + (co >> 5)) * 4 + ((co & 31) >> 3)) * 64 + ((co & 7) >> 2) * 32 + x) * 4 + (co & 3)] = acc[c];
                }
                if (lane_e == 0) {
                    if (whole) {
                        if (a.lse) a.lse[(size_t)head * a.n_tok + sq.q0 + tok] = lse_of(mr, lr, a.scale_log2);
                    } else {
                        frag[R * D + wave * 32 + x] = mr;
                        frag[R * D + R + wave * 32 + x] = -lr;   // its sums add up to one
                    }
                }
            }
        }
        __syncthreads();   // the next piece's tiles go where this one's rows were
        if (SPLIT && begins && !ends) d = Desc{r.b, h, qt, share_of(r, its.last)};
    }
    if (SPLIT && tid == 0) a.desc[r.share] = d;
}

// Puts the fragments of an item together: a workgroup per share, 32 rows and 32 coordinates; most find nothing to do.
template <int D>
__global__ __launch_bounds__(256) void combine_chunk_kernel(const Args a) {
    constexpr int DB = D / 32;
    const Desc d = a.desc[blockIdx.x];
    if (d.last < 0) return;
    const int wave = blockIdx.y / DB, db = blockIdx.y % DB;
    const Seq sq = seq_of<R>(a, d.b);
    const int n_rows = sq.n_q * a.group;
    if (d.qt * R + wave * 32 >= n_rows) return;
    const int lane = threadIdx.x & 63, q4 = threadIdx.x >> 6, col = lane & 31, g = lane >> 5;
    const int first = blockIdx.x, n = d.last - first + 1;
    float m_all = -INFINITY;
#pragma unroll 4
    for (int i = 0; i < n; ++i) m_all = fmaxf(m_all, fragment<FRAG_FLOATS>(a, first, i)[R * D + wave * 32 + col]);
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const float *f = fragment<FRAG_FLOATS>(a, first, i);
        const float wt = weight_of(f[R * D + wave * 32 + col], m_all, a.scale_log2), lf = f[R * D + R + wave * 32 + col];
        x += ((const f32x4 *)f)[((wave * DB + db) * 4 + q4) * 64 + lane] * parts_of(lf, wt);
        l += fabsf(lf) * wt;
    }
    const int rr = d.qt * R + wave * 32 + col;
    if (rr >= n_rows) return;
    const int tok = rr / a.group, head = d.h * a.group + rr - tok * a.group;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    x *= inv;
    if (!finite(x)) {   // sums beyond the range: again with weights that add up to one
        x = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int i = 0; i < n; ++i) {
            const float *f = fragment<FRAG_FLOATS>(a, first, i);
            x += ((const f32x4 *)f)[((wave * DB + db) * 4 + q4) * 64 + lane] *
                 parts_of(f[R * D + R + wave * 32 + col], weight_of(f[R * D + wave * 32 + col], m_all, a.scale_log2) * inv);
        }
    }
    const bf16x4 y = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
    *(bf16x4 *)(a.O.p + head * a.O.head + (int64_t)(sq.q0 + tok) * a.O.row + (32 * db + 8 * q4 + 4 * g) * 2) = y;
    if (a.lse && db == 0 && q4 == 0 && g == 0)
        a.lse[(size_t)head * a.n_tok + sq.q0 + tok] = lse_of(m_all, l, a.scale_log2);
}

}  // namespace chunk

}  // namespace paged

size_t paged_chunk_frag_bytes() { return (size_t)2 * paged::chunk::SHARES * paged::chunk::FRAG_FLOATS * 4; }

namespace paged {

namespace chunk {

template <int D>
int setup() {
    for (const void *f : {(const void *)attn_chunk_kernel<D, true>, (const void *)attn_chunk_kernel<D, false>})
        if (hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes<D>()) != hipSuccess) return FASTAR_ERR_HIP;
    return FASTAR_OK;
}
template <int D>
int launch(const Args &a, int64_t items, bool split, hipStream_t s) {
    if (!split) {
        hipLaunchKernelGGL((attn_chunk_kernel<D, false>), dim3((unsigned)items), dim3(2 * NWG * 64), lds_bytes<D>(), s, a);
        FASTAR_LAUNCH_CHECK();
        return FASTAR_OK;
    }
    hipLaunchKernelGGL((attn_chunk_kernel<D, true>), dim3(SHARES), dim3(2 * NWG * 64), lds_bytes<D>(), s, a);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(combine_chunk_kernel<D>, dim3(SHARES, 8 * D / 32), dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}

}  // namespace chunk

}  // namespace paged

int paged_chunk_setup() {
    static DeviceOnce once;
    return once.run([](int) { return paged::chunk::setup<128>(); });   // the tiles of d = 64 fit without
}

int launch_paged_chunk(const paged::Args &a, int64_t rows, int64_t keys, bool one_launch, hipStream_t s) {
    using namespace paged::chunk;
    if (const int rc = paged_chunk_setup(); rc != FASTAR_OK) return rc;
    const int64_t items = ((rows + R - 1) / R + a.B) * a.pg.Hkv;   // at most
    const bool split = !one_launch || (items < SHARES && keys > FEW_KEYS) || !launch_ok(items, 2 * NWG * 64);
    return a.pg.d == 128 ? launch<128>(a, items, split, s) : launch<64>(a, items, split, s);
}

}  // namespace fastar
