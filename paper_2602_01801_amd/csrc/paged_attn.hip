// Attention of packed queries over a paged cache of E4M3 codes (paged_attn_fwd): the kernel for few rows per sequence (single
// tokens above all), and the entry point.
//
// A wavefront walks tiles of 64 keys for 16 RT rows, with both contractions transposed, so that what belongs to a row stays in
// its lanes (lane l: row l % 16, quarter q = l / 16):
//     S^T = K Q^T    A row 4 q + v of product j is key 16 q + 4 j + v of the tile, so that a lane's 16 scores are the keys
//                    16 q .. 16 q + 15; a lane loads 16 bytes, one token's coordinates of a cell: two products' operands
//     O^T = V^T P^T  A = 16 coordinates x 32 keys: 16 bytes of a lane are 16 tokens of one coordinate, the keys of its quarter,
//                    two products' operands; B = P^T, from the score registers as they are
// Codes go from global memory into registers and are widened there, with their page's scale, to bf16 (exact: a power of two
// times four significant bits), two per instruction; nothing passes through LDS but the wavefronts' partial results: a
// workgroup's wavefronts take every NW-th tile of its share and put their sums together at the end of an item.
// Tables that are so short that there is nothing to cut take one launch (SPLIT = false), a workgroup of eight wavefronts per item.
// What bounds it: bytes.  Tokens of two requests of 200000 and 230400 keys x 8 key heads x 128, 881 MB: 154 us = 5.7 TB/s and 8 us for
// the fragments; of 48 requests of 100 to 37440 keys 951 MB in 174 us and 6.  Short ones: the chain lengths, page numbers, codes, sums,
// each a trip to memory (1560 keys x 12 heads 10.8 us).
#include "paged_dev.hpp"

namespace fastar {

int pages_check(const fastar_pages *pg);

namespace paged {

constexpr int SHARES = 512;        // workgroups that share the tiles: two per compute unit
// Units of a share at least (tiles, and the ENDS in front of an item's): few workgroups put fragments together.  3 / 6 / 12 / 24 / 48: one
// sequence of 100000 keys, one key head 41 / 28 / 20 / 19 / 25 us, of 16000 keys x 8 key heads 27 / 19 / 18 / 19 / 25, 16 of 2100 x 8
// 25 / 25 / 22.5 / 22.3 / 27.5; launches with more work have longer shares anyway.
constexpr int LEAST = 12;
constexpr int MAX_RT = 2;
constexpr int FRAG_FLOATS = MAX_RT * (16 * 128 + 32);
static_assert(SHARES <= MAX_SHARES, "descriptors");
// Tables of up to this many keys are not cut.  Whole / cut, a token each: one request of 12 heads with 1000 keys 9.1 / 14.0 us, 2000
// 12.3 / 14.1, 4000 18.7 / 13.1; 48 requests of 40 heads on 8 with 1000 24 / 30, 2000 38 / 45, 4000 79 / 89.
constexpr int ONE_LAUNCH_KEYS = 2048;

__device__ __forceinline__ f32x4 mfma_16x16x32(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// The value of the lane eight further (lane % 16 above 7: eight before).
__device__ __forceinline__ float other_half_of_16(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xf, 0xf, true));   // row_ror:8
}

template <int D, int RT, bool SPLIT, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attn_kernel(const Args a) {
    constexpr int R = 16 * RT, DB = D / 16, KS = D / 64;
    constexpr int NS = NW < 4 ? NW : 4;   // wavefronts' sums that LDS holds at a time
    __shared__ int s_odd;   // the last piece with sums that are not finite
    __shared__ float s_m[NW][R], s_l[NW][R];
    __shared__ f32x4 s_o[NS][DB][64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 15, quarter = lane >> 4;
    const int Hkv = a.pg.Hkv;
    const float scale_log2 = a.scale_log2;

    Range r;
    Seq sq;
    if (!first_unit<R, SPLIT>(a, SHARES, LEAST, r, sq)) {
        if (SPLIT && tid == 0) a.desc[r.share].last = -1;
        return;
    }
    Desc d = {0, 0, 0, -1};
    if (tid == 0) s_odd = 0;   // read behind the first barriers
    int turn = 0;
    while (r.u < r.u_end) {   // uniform: one piece of one item per turn
        if (SPLIT && r.u >= r.base + (long long)sq.n_qt * Hkv * (sq.n_tiles + ENDS)) find_unit<R, SPLIT>(a, r.u, r.b, r.base, sq);
        const PieceOf piece = next_piece<SPLIT>(r, sq);
        if (piece.te <= piece.ta) continue;
        ++turn;
        const int h = piece.h, qt = piece.qt, ta = piece.ta, te = piece.te;
        const bool begins = ta == 0, ends = te == sq.n_tiles;

        const int n_rows = sq.n_q * a.group;
        const int tok0 = (qt * R) / a.group, tok1 = min(qt * R + R - 1, n_rows - 1) / a.group;
        const int limit_min = a.causal ? min(max(sq.L - sq.n_q + tok0 + 1, 0), sq.L) : sq.L;   // keys that the first row sees
        const int limit_max = a.causal ? min(max(sq.L - sq.n_q + tok1 + 1, 0), sq.L) : sq.L;   // ... the last
        // Up to eight rows leave half of a product's columns empty: column c + 8 then holds row c too, with what rounding takes from its
        // weights in place of the weights, so that these rows have weights of 16 bits without a product more.  One token of 12 heads,
        // 1560 keys each: an error of 0.0015 (the output's rounding) instead of 0.0018 to 0.0028, for 0.5 us more; 48 tokens
        // x 40 heads 184 us instead of 183.  With more rows peaked ones are fewer among them and products of their own cost 3 to 17 %:
        // weights of 8 bits.
        const bool fold = RT == 1 && n_rows - qt * R <= 8;
        const bool rest = fold && row >= 8;
        int limit[RT];
        bf16x8 qf[RT][2 * KS];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int rr = min(qt * R + 16 * rt + (fold ? row & 7 : row), n_rows - 1);
            const int tok = rr / a.group, head = h * a.group + rr - tok * a.group;
            limit[rt] = a.causal ? sq.L - sq.n_q + tok + 1 : sq.L;
            const char *qp = a.Q.p + head * a.Q.head + (int64_t)(sq.q0 + tok) * a.Q.row;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) qf[rt][2 * s + hh] = *(const bf16x8 *)(qp + (16 * (4 * s + quarter) + 8 * hh) * 2);
        }
        f32x4 o[RT][DB];
        float m[RT], neg[RT], l[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -INFINITY;
            neg[rt] = l[rt] = 0.0f;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[rt][db] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }

        // ---- the wavefront's tiles ----
        const int t_end = min(te, (limit_max + TK - 1) / TK);
        const int32_t *pages = a.table + (size_t)r.b * a.max_pages;
        const int last_page = (limit_max - 1) >> a.pshift;
        const int kblk = row >> 2, blk_mask = (1 << (a.pshift - 4)) - 1;   // block of 16 tokens of this lane's K rows (of its V bytes: quarter)
        const size_t page_bytes = (size_t)D << a.pshift;
        const uint8_t *K8 = a.pg.K8 + h * page_bytes + (kblk & blk_mask) * (16 * D) + quarter * 256 + (row & 3) * 16;
        const uint8_t *V8 = a.pg.V8 + h * page_bytes + (quarter & blk_mask) * (16 * D) + row * 16;
        struct Ids {
            int k, v;
        };
        auto ids_of = [&](int t) __attribute__((always_inline)) {
            return Ids{pages[min((t * TK + 16 * kblk) >> a.pshift, last_page)], pages[min((t * TK + 16 * quarter) >> a.pshift, last_page)]};
        };
        u32x4 kr[4][KS], vr[DB];
        float ks, vs;
        bool v_ok = true;
        auto load_k = [&](int id) __attribute__((always_inline)) {
            id = page_exists(a, id) ? id : 0;
            const uint8_t *p = K8 + (size_t)id * Hkv * page_bytes;
            ks = a.pg.kscale[(size_t)id * Hkv + h];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int s = 0; s < KS; ++s) kr[j][s] = *(const u32x4 *)(p + j * 64 + s * 1024);
        };
        auto load_v = [&](int id) __attribute__((always_inline)) {
            v_ok = page_exists(a, id);
            id = v_ok ? id : 0;
            const uint8_t *p = V8 + (size_t)id * Hkv * page_bytes;
            vs = a.pg.vscale[(size_t)id * Hkv + h];
#pragma unroll
            for (int db = 0; db < DB; ++db) vr[db] = *(const u32x4 *)(p + db * 256);
        };
        int t = ta + w;
        Ids next{0, 0};
        if (t < t_end) {
            const Ids now = ids_of(t);
            next = ids_of(t + NW);
            load_k(now.k);
            load_v(now.v);
        }
        for (; t < t_end; t += NW) {
            const Ids after = ids_of(t + 2 * NW);
            f32x4 s[RT][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) s[rt][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < KS; ++c) {
                    const bf16x8 k0 = widen(kr[j][c][0], kr[j][c][1], ks), k1 = widen(kr[j][c][2], kr[j][c][3], ks);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        s[rt][j] = mfma_16x16x32(k0, qf[rt][2 * c], s[rt][j]);
                        s[rt][j] = mfma_16x16x32(k1, qf[rt][2 * c + 1], s[rt][j]);
                    }
                }
            }
            if (t + NW < t_end) load_k(next.k);
            if (t * TK + TK > limit_min || !__all(v_ok)) {   // uniform: some key of the tile is not seen by some row
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (!v_ok || t * TK + 16 * quarter + 4 * j + v >= limit[rt]) s[rt][j][v] = -INFINITY;
                // values that no row sees need not be numbers, nor page 0's scale
                if (!v_ok) vs = 1.0f;
                const u32x4 mask = first_bytes(v_ok ? limit_max - (t * TK + 16 * quarter) : 0);
#pragma unroll
                for (int db = 0; db < DB; ++db) vr[db] &= mask;
            }
            bf16x8 p[RT][2];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float mx = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v) mx = fmaxf(mx, s[rt][j][v]);
                mx = max_of_quarters(mx);
                // The reference is the maximum itself, so that the weight of a row that one key rules is 1 and loses nothing: 20 tokens
                // of 16 rows an error of 0.0017 instead of 0.0019 with a reference that may lag 8 octaves, 3 of 9 rows 0.0018 instead
                // of 0.002, for 0 to 1 % (8 tokens of 24 rows on 1560 keys 4 %).
                if (__any(mx > m[rt])) {
                    const float mn = fmaxf(m[rt], mx);
                    const float alpha = weight_of(m[rt], mn, scale_log2);
                    m[rt] = mn;
                    neg[rt] = mn == -INFINITY ? 0.0f : -mn * scale_log2;
                    l[rt] *= alpha;
#pragma unroll
                    for (int db = 0; db < DB; ++db) o[rt][db] *= alpha;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float x = __builtin_amdgcn_exp2f(fmaf(s[rt][j][v], scale_log2, neg[rt]));
                        l[rt] += x;
                        const __bf16 y = (__bf16)x;
                        p[rt][j >> 1][4 * (j & 1) + v] = RT == 1 ? (__bf16)(x - (rest ? (float)y : 0.0f)) : y;
                    }
            }
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const bf16x8 v0 = widen(vr[db][0], vr[db][1], vs), v1 = widen(vr[db][2], vr[db][3], vs);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    o[rt][db] = mfma_16x16x32(v0, p[rt][0], o[rt][db]);
                    o[rt][db] = mfma_16x16x32(v1, p[rt][1], o[rt][db]);
                }
            }
            if (t + NW < t_end) load_v(next.v);
            next = after;
        }

        if (fold) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int v = 0; v < 4; ++v) o[0][db][v] += other_half_of_16(o[0][db][v]);
        }

        // ---- the wavefronts' sums together ----
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            l[rt] = sum_of_quarters(l[rt]);
            if (quarter == 0) {
                s_m[w][16 * rt + row] = m[rt];
                s_l[w][16 * rt + row] = l[rt];
            }
        }
        __syncthreads();
        const bool whole = begins && ends;
        float *frag = SPLIT ? a.frag + (size_t)(2 * r.share + (begins ? 1 : 0)) * FRAG_FLOATS : nullptr;
        bool odd = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float m_all = s_m[0][16 * rt + row];
#pragma unroll
            for (int i = 1; i < NW; ++i) m_all = fmaxf(m_all, s_m[i][16 * rt + row]);
            float l_all = 0.0f;
#pragma unroll
            for (int i = 0; i < NW; ++i) l_all += s_l[i][16 * rt + row] * weight_of(s_m[i][16 * rt + row], m_all, scale_log2);
            odd |= !sums_up(m_all, l_all);
            const float wt = weight_of(m[rt], m_all, scale_log2);
#pragma unroll
            for (int db = 0; db < DB; ++db) o[rt][db] *= wt;
            if constexpr (NW > NS) {   // the upper half of the wavefronts first
                if (w >= NS) {
#pragma unroll
                    for (int db = 0; db < DB; ++db) s_o[w - NS][db][lane] = o[rt][db];
                }
                __syncthreads();
                if (w < NS) {
#pragma unroll
                    for (int db = 0; db < DB; ++db) o[rt][db] += s_o[w][db][lane];
                }
                __syncthreads();
            }
            if (w < NS) {
#pragma unroll
                for (int db = 0; db < DB; ++db) s_o[w][db][lane] = o[rt][db];
            }
            __syncthreads();
            const int rr = qt * R + 16 * rt + row;
            const int tok = rr / a.group, head = h * a.group + rr - tok * a.group;
            for (int db = w; db < DB; db += NW) {
                f32x4 x = s_o[0][db][lane];
#pragma unroll
                for (int i = 1; i < NS; ++i) x += s_o[i][db][lane];
#pragma unroll
                for (int v = 0; v < 4; ++v) odd |= !(fabsf(x[v]) < INFINITY);
                if (whole) {
                    const float inv = l_all == 0.0f ? 0.0f : 1.0f / l_all;
                    if (rr < n_rows) {
                        const bf16x4 y = {(__bf16)(x[0] * inv), (__bf16)(x[1] * inv), (__bf16)(x[2] * inv), (__bf16)(x[3] * inv)};
                        *(bf16x4 *)(a.O.p + head * a.O.head + (int64_t)(sq.q0 + tok) * a.O.row + (16 * db + 4 * quarter) * 2) = y;
                    }
                } else {
                    ((f32x4 *)frag)[(rt * DB + db) * 64 + lane] = x;
                }
            }
            if (w == 0 && quarter == 0) {
                if (whole) {
                    if (a.lse && rr < n_rows)
                        a.lse[(size_t)head * a.n_tok + sq.q0 + tok] = lse_of(m_all, l_all, scale_log2);
                } else {
                    frag[R * D + 16 * rt + row] = m_all;
                    frag[R * D + R + 16 * rt + row] = l_all;
                }
            }
            if (odd) s_odd = turn;
            __syncthreads();
        }
        // Sums that are not finite, or none: a value that a row does not see may have come in as 0 * x (a product of tiles has no other
        // way), or they or the weights have left the range.  Those rows are done again key by key, over the keys that they see.
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(s_odd) == turn, 0)) {
            const Args a = args_anew<Args>();
            const int32_t *pages = a.table + (size_t)r.b * a.max_pages;
            float *frag = SPLIT ? a.frag + (size_t)(2 * r.share + (begins ? 1 : 0)) * FRAG_FLOATS : nullptr;
            for (int i = w; i < R && qt * R + i < n_rows; i += NW) {
                const int rr = qt * R + i, tok = rr / a.group, head = h * a.group + rr - tok * a.group;
                float mr, lr, acc[D / 64];
                row_by_paged_keys<D>(a, a.Q.p + head * a.Q.head + (int64_t)(sq.q0 + tok) * a.Q.row, pages, h, ta * TK,
                                     min(a.causal ? min(sq.L - sq.n_q + tok + 1, sq.L) : sq.L, te * TK), mr, lr, acc);
#pragma unroll
                for (int c = 0; c < D / 64; ++c) {
                    const int co = 64 * c + lane;
                    if (whole) ((__bf16 *)(a.O.p + head * a.O.head + (int64_t)(sq.q0 + tok) * a.O.row))[co] = (__bf16)acc[c];
                    else frag[(((i >> 4) * DB + (co >> 4)) * 64 + ((co & 15) >> 2) * 16 + (i & 15)) * 4 + (co & 3)] = acc[c];
                }
                if (lane == 0) {
                    if (whole) {
                        if (a.lse) a.lse[(size_t)head * a.n_tok + sq.q0 + tok] = lse_of(mr, lr, a.scale_log2);
                    } else {
                        frag[R * D + i] = mr;
                        frag[R * D + R + i] = -lr;   // its sums add up to one
                    }
                }
            }
        }
        if (SPLIT && begins && !ends) d = Desc{r.b, h, qt, share_of(r, piece.last)};
    }
    if (SPLIT && tid == 0) a.desc[r.share] = d;
}

// Puts the fragments of an item together: a workgroup per share and block of 16 coordinates x 16 rows, most of which find
// nothing to do; its wavefronts take every fourth fragment.
template <int D, int RT>
__global__ __launch_bounds__(256) void combine_kernel(const Args a) {
    constexpr int R = 16 * RT, DB = D / 16, NW = 4;
    __shared__ float s_l[NW][16];
    __shared__ f32x4 s_o[NW][64];
    const Desc d = a.desc[blockIdx.x];
    if (d.last < 0) return;
    const int rt = blockIdx.y / DB, db = blockIdx.y % DB;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, row = lane & 15, quarter = lane >> 4;
    const int first = blockIdx.x, n = d.last - first + 1;
    auto frag = [&](int i) { return fragment<FRAG_FLOATS>(a, first, i); };
    float m_all = -INFINITY;
#pragma unroll 8
    for (int i = quarter; i < n; i += 4) m_all = fmaxf(m_all, frag(i)[R * D + 16 * rt + row]);
    m_all = max_of_quarters(m_all);
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
#pragma unroll 8
    for (int i = w; i < n; i += NW) {
        const float *f = frag(i);
        const float wt = weight_of(f[R * D + 16 * rt + row], m_all, a.scale_log2), lf = f[R * D + R + 16 * rt + row];
        x += ((const f32x4 *)f)[(rt * DB + db) * 64 + lane] * parts_of(lf, wt);
        l += fabsf(lf) * wt;
    }
    s_o[w][lane] = x;
    if (quarter == 0) s_l[w][row] = l;
    __syncthreads();
    if (w != 0) return;
    l = s_l[0][row];
#pragma unroll
    for (int i = 1; i < NW; ++i) {
        x += s_o[i][lane];
        l += s_l[i][row];
    }
    const Seq sq = seq_of<R>(a, d.b);
    const int rr = d.qt * R + 16 * rt + row;
    if (rr >= sq.n_q * a.group) return;
    const int tok = rr / a.group, head = d.h * a.group + rr - tok * a.group;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    x *= inv;
    if (!finite(x)) {   // sums beyond the range: again with weights that add up to one
        x = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int i = 0; i < n; ++i) {
            const float *f = frag(i);
            x += ((const f32x4 *)f)[(rt * DB + db) * 64 + lane] * parts_of(f[R * D + R + 16 * rt + row], weight_of(f[R * D + 16 * rt + row], m_all, a.scale_log2) * inv);
        }
    }
    const bf16x4 y = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
    *(bf16x4 *)(a.O.p + head * a.O.head + (int64_t)(sq.q0 + tok) * a.O.row + (16 * db + 4 * quarter) * 2) = y;
    if (a.lse && db == 0 && quarter == 0)
        a.lse[(size_t)head * a.n_tok + sq.q0 + tok] = lse_of(m_all, l, a.scale_log2);
}

template <int D, int RT>
int launch(const Args &a, int64_t items, bool split, hipStream_t s) {
    if (!split) {
        hipLaunchKernelGGL((attn_kernel<D, RT, false, 8>), dim3((unsigned)items), dim3(512), 0, s, a);
        FASTAR_LAUNCH_CHECK();
        return FASTAR_OK;
    }
    hipLaunchKernelGGL((attn_kernel<D, RT, true, 4>), dim3(SHARES), dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL((combine_kernel<D, RT>), dim3(SHARES, RT * D / 16), dim3(256), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}

}  // namespace paged

size_t paged_chunk_frag_bytes();
int launch_paged_chunk(const paged::Args &a, int64_t rows, int64_t keys, bool one_launch, hipStream_t s);

size_t paged_attn_ws_bytes() {
    using namespace paged;
    const size_t own = (size_t)2 * SHARES * FRAG_FLOATS * 4, chunk = paged_chunk_frag_bytes();
    return (MAX_SHARES * sizeof(Desc) + (own > chunk ? own : chunk) + 255) / 256 * 256;
}

}  // namespace fastar

extern "C" int paged_attn_fwd(const fastar_rows *Q, const int32_t *cu_q, const int32_t *len, const int32_t *table, int B,
                              int max_pages, int n_tok, int Hq, const fastar_pages *pages, int dtype, int causal, float scale,
                              const fastar_rows *O, float *lse, void *ws, size_t ws_bytes, void *stream) {
    using namespace fastar;
    if (dtype != FASTAR_F32 && dtype != FASTAR_BF16) return FASTAR_ERR_INVALID_ARG;
    if (B < 0 || n_tok < 0 || max_pages <= 0 || Hq <= 0) return FASTAR_ERR_INVALID_ARG;
    if (!scale_ok(scale) || (causal & ~1)) return FASTAR_ERR_INVALID_ARG;
    if (const int rc = pages_check(pages); rc != FASTAR_OK) return rc;
    if (Hq % pages->Hkv) return FASTAR_ERR_INVALID_ARG;
    if (dtype != FASTAR_BF16 || (int64_t)max_pages * pages->P > MAX_KEYS) return FASTAR_ERR_UNSUPPORTED;
    if ((int64_t)n_tok * Hq > INT32_MAX / 2) return FASTAR_ERR_UNSUPPORTED;
    if (!ws || ((uintptr_t)ws & 255)) return FASTAR_ERR_INVALID_ARG;
    if (ws_bytes < paged_attn_ws_bytes()) return FASTAR_ERR_WORKSPACE;
    if (n_tok == 0 || B == 0) return FASTAR_OK;
    if (!cu_q || !len || !table || !view_ok(Q, Hq, n_tok, 2) || !view_ok(O, Hq, n_tok, 2) || !rows_apart(O, Hq, n_tok, pages->d)) return FASTAR_ERR_INVALID_ARG;
    const int group = Hq / pages->Hkv;
    const paged::Args a = {view_of(Q, Hq, n_tok, 2), view_of(O, Hq, n_tok, 2), cu_q, len, table, B, max_pages, n_tok, group, causal,
                           __builtin_ctz((unsigned)pages->P), *pages, scale * 1.4426950408889634f, lse,
                           (paged::Desc *)ws, (float *)((char *)ws + paged::MAX_SHARES * sizeof(paged::Desc))};
    const int64_t rows = (int64_t)n_tok * group;
    const hipStream_t s = (hipStream_t)stream;
    // By the rows that a sequence has on average: 16 or 32 per item, or the kernel whose wavefronts share their tiles.  8 heads on 8, one
    // sequence of 1500 keys, 8 of 1500, 8 of 9000 and 48 of 9000: 16 rows an item / 32, at 16 rows 11.3 / 14.5, 11.7 / 14.9, 38.5 / 50, 178 / 205 us,
    // at 20 11.3 / 14.9, 14.0 / 15.3, 38 / 52, 322 / 207; 32 rows an item / the other kernel, at 32 15.5 / 27, 16 / 34, 52 / 86, 207 / 426, at 40
    // 15.5 / 28.8, 17.9 / 38, 50 / 90, 354 / 430, at 96 15.6 / 29, 20 / 39, 88 / 92, 453 / 449: long batches decide on the first line; the
    // second is low for them and for few sequences (64 to 96 rows).
    const int64_t keys = (int64_t)max_pages * pages->P;
    const bool one_launch = keys <= paged::ONE_LAUNCH_KEYS;
    if (rows > (int64_t)32 * B) return launch_paged_chunk(a, rows, keys, one_launch, s);
    const int rt = rows <= (int64_t)16 * B ? 1 : 2;
    const int64_t items = ((rows + 16 * rt - 1) / (16 * rt) + B) * pages->Hkv;   // at most
    const bool split = !one_launch || !launch_ok(items, 512);
    if (pages->d == 128) return rt == 1 ? paged::launch<128, 1>(a, items, split, s) : paged::launch<128, 2>(a, items, split, s);
    return rt == 1 ? paged::launch<64, 1>(a, items, split, s) : paged::launch<64, 2>(a, items, split, s);
}
