// Attention of packed queries over a paged cache of E4M3 codes (paged_attn_fwd).
//
// An item is a tile of R = 16 RT rows of one sequence and key head; a row is a (token, query head of the group) pair, so that
// the heads that share keys share their loads.  A wavefront walks tiles of 64 keys with both contractions transposed, so that
// what belongs to a row stays in its lanes (lane l: row l % 16, quarter q = l / 16):
//     S^T = K Q^T    A row 4 q + v of product j is key 16 q + 4 j + v of the tile, so that a lane's 16 scores are the keys
//                    16 q .. 16 q + 15; a lane loads 16 bytes, one token's coordinates of a cell: two products' operands
//     O^T = V^T P^T  A = 16 coordinates x 32 keys: 16 bytes of a lane are 16 tokens of one coordinate, the keys of its quarter,
//                    two products' operands; B = P^T, from the score registers as they are
// Codes go from global memory into registers and are widened there, with their page's scale, to bf16 (exact: a power of two
// times four significant bits), two per instruction; nothing passes through LDS but the wavefronts' partial results.
//
// The lengths are on the device, so the device deals out the work: the items' tiles, one after the other, are cut into equal
// shares, a workgroup each; its four wavefronts take every fourth tile and put their sums together through LDS.  A share
// that holds a part of an item leaves a fragment (sums, reference maxima, row sums) in the workspace, and a second launch
// puts the fragments of an item together.  Tables that are so short that there is nothing to cut take one launch.
#include "packed.hpp"

namespace fastar {

int pages_check(const fastar_pages *pg);

namespace paged {

constexpr int TK = 64;             // keys per tile
constexpr int NW = 4;              // wavefronts per workgroup
constexpr int SHARES = 512;        // workgroups that share the tiles: two per compute unit
constexpr int MAX_RT = 4;
constexpr int FRAG_FLOATS = MAX_RT * (16 * 128 + 32);
constexpr float LN2 = 0.6931471805599453f;
constexpr float TAU = 8.0f;        // the reference maximum may lag the true one by 8 octaves: weights up to 256

struct Desc {   // an item that was cut: its first share writes this
    int b, h, qt, last;   // last share that holds a part of it; -1: none
};
constexpr size_t WS_DESC = 0, WS_FRAG = SHARES * sizeof(Desc);

__device__ __forceinline__ f32x4 mfma_16x16x32(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Eight codes times a power of two, exactly.
__device__ __forceinline__ bf16x8 widen(unsigned lo, unsigned hi, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    const bf16x8 r = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    return r;
}
// Over the four lanes of a row (lane % 16).
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
// Weight of sums taken against reference m among those against m_all; a reference of -inf means sums of 0, or of no numbers.
__device__ __forceinline__ float weight_of(float m, float m_all, float scale_log2) {
    return m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - m_all) * scale_log2);
}

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
__device__ __forceinline__ Seq seq_of(const Args &a, int b) {
    const Rows r = rows_of(a.cu_q, b, a.n_tok);
    Seq s;
    s.q0 = r.first;
    s.n_q = r.n;
    s.L = min(max(a.len[b], 0), a.max_pages << a.pshift);
    s.n_qt = (r.n * a.group + R - 1) / R;
    s.n_tiles = max((s.L + TK - 1) / TK, 1);
    return s;
}

template <int D, int RT, bool SPLIT>
__global__ __launch_bounds__(NW * 64, RT <= 2 ? 2 : 1) void attn_kernel(const Args a) {
    constexpr int R = 16 * RT, DB = D / 16, KS = D / 64;
    __shared__ long long s_part[NW], s_base;
    __shared__ int s_b, s_flag;
    __shared__ float s_m[NW][R], s_l[NW][R];
    __shared__ f32x4 s_o[NW][DB][64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 15, quarter = lane >> 4;
    const int Hkv = a.pg.Hkv;
    const float scale_log2 = a.scale_log2;

    auto units_of = [&](int b) -> long long {
        if (b >= a.B) return 0;
        const Seq s = seq_of<R>(a, b);
        return (long long)s.n_qt * Hkv * (SPLIT ? s.n_tiles : 1);
    };
    // Inclusive prefix sum over the workgroup and the total, in all threads.
    auto scan = [&](long long v, long long &all) -> long long {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long long u = __shfl_up(v, o, 64);
            if (lane >= o) v += u;
        }
        __syncthreads();
        if (lane == 63) s_part[w] = v;
        __syncthreads();
        long long base = 0;
        all = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            if (i < w) base += s_part[i];
            all += s_part[i];
        }
        return v + base;
    };
    // The sequence that holds unit u, and its first unit.
    auto find = [&](long long u, int &b_out, long long &base_out) {
        long long before = 0;
        for (int b0 = 0; b0 < a.B; b0 += NW * 64) {
            const long long v = units_of(b0 + tid);
            long long all;
            const long long upto = before + scan(v, all);
            if (u >= upto - v && u < upto) {
                s_b = b0 + tid;
                s_base = upto - v;
            }
            before += all;
            if (u < before) break;   // uniform
        }
        __syncthreads();
        b_out = __builtin_amdgcn_readfirstlane(s_b);
        base_out = s_base;
        __syncthreads();
    };

    long long W = 0;
    for (int b0 = 0; b0 < a.B; b0 += NW * 64) {
        long long all;
        scan(units_of(b0 + tid), all);
        W += all;
    }
    long long u, u_end, share;
    long long n_shares = 0;
    if constexpr (SPLIT) {
        // a share holds a tile for every wavefront at least; when all are used, neighbours go to the same XCD
        n_shares = min((long long)SHARES, (W + NW - 1) / NW);
        share = n_shares == SHARES ? (int)(blockIdx.x & 7) * (SHARES / 8) + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
        if (share >= n_shares) {
            if (tid == 0) a.desc[share].last = -1;
            return;
        }
        u = W * share / n_shares;
        u_end = W * (share + 1) / n_shares;
    } else {
        share = blockIdx.x;
        u = share;
        u_end = u + 1;
        if (u >= W) return;
    }
    Desc d = {0, 0, 0, -1};
    int b = 0;
    long long base = 0;
    find(u, b, base);
    Seq sq = seq_of<R>(a, b);
    while (u < u_end) {   // uniform: one piece of one item per turn
        const int per = SPLIT ? sq.n_tiles : 1;
        const long long seq_units = (long long)sq.n_qt * Hkv * per;
        if (u >= base + seq_units) {
            base += seq_units;
            ++b;
            if (b >= a.B || units_of(b) == 0) find(u, b, base);
            sq = seq_of<R>(a, b);
            continue;
        }
        const long long local = u - base;
        const int item = (int)(local / per);
        const int h = item / sq.n_qt, qt = item - h * sq.n_qt;
        const int ta = SPLIT ? (int)(local - (long long)item * per) : 0;
        const int te = SPLIT ? (int)min((long long)per, ta + (u_end - u)) : sq.n_tiles;
        const bool begins = ta == 0, ends = te == sq.n_tiles;
        u += SPLIT ? te - ta : 1;

        const int n_rows = sq.n_q * a.group;
        const int tok0 = (qt * R) / a.group, tok1 = min(qt * R + R - 1, n_rows - 1) / a.group;
        const int limit_min = a.causal ? min(max(sq.L - sq.n_q + tok0 + 1, 0), sq.L) : sq.L;   // keys that the first row sees
        const int limit_max = a.causal ? min(max(sq.L - sq.n_q + tok1 + 1, 0), sq.L) : sq.L;   // ... the last
        int limit[RT];
        bf16x8 qf[RT][2 * KS];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int rr = min(qt * R + 16 * rt + row, n_rows - 1);
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
        const int32_t *pages = a.table + (size_t)b * a.max_pages;
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
        auto exists = [&](int id) { return (unsigned)id < (unsigned)a.pg.n_pages; };
        u32x4 kr[4][KS], vr[DB];
        float ks, vs;
        bool v_ok = true;
        auto load_k = [&](int id) __attribute__((always_inline)) {
            id = exists(id) ? id : 0;
            const uint8_t *p = K8 + (size_t)id * Hkv * page_bytes;
            ks = a.pg.kscale[(size_t)id * Hkv + h];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int s = 0; s < KS; ++s) kr[j][s] = *(const u32x4 *)(p + j * 64 + s * 1024);
        };
        auto load_v = [&](int id) __attribute__((always_inline)) {
            v_ok = exists(id);
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
                // values that no row sees need not be numbers
                const int live = v_ok ? limit_max - (t * TK + 16 * quarter) : 0;
                u32x4 mask;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int n = min(max(live - 4 * e, 0), 4);
                    mask[e] = n == 4 ? ~0u : (1u << (8 * n)) - 1u;
                }
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
                if (__any((mx - m[rt]) * scale_log2 > TAU)) {
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
                        p[rt][j >> 1][4 * (j & 1) + v] = (__bf16)x;
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

        // ---- the wavefronts' sums together ----
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            l[rt] = sum_of_quarters(l[rt]);
            if (quarter == 0) {
                s_m[w][16 * rt + row] = m[rt];
                s_l[w][16 * rt + row] = l[rt];
            }
        }
        if (tid == 0) s_flag = 0;
        __syncthreads();
        const bool whole = begins && ends;
        float *frag = SPLIT ? a.frag + (size_t)(2 * share + (begins ? 1 : 0)) * FRAG_FLOATS : nullptr;
        bool odd = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float m_all = s_m[0][16 * rt + row];
#pragma unroll
            for (int i = 1; i < NW; ++i) m_all = fmaxf(m_all, s_m[i][16 * rt + row]);
            float l_all = 0.0f;
#pragma unroll
            for (int i = 0; i < NW; ++i) l_all += s_l[i][16 * rt + row] * weight_of(s_m[i][16 * rt + row], m_all, scale_log2);
            const float wt = weight_of(m[rt], m_all, scale_log2);
#pragma unroll
            for (int db = 0; db < DB; ++db) s_o[w][db][lane] = o[rt][db] * wt;
            __syncthreads();
            const int rr = qt * R + 16 * rt + row;
            const int tok = rr / a.group, head = h * a.group + rr - tok * a.group;
#pragma unroll
            for (int e = 0; e < DB / NW; ++e) {
                const int db = w * (DB / NW) + e;
                f32x4 x = s_o[0][db][lane];
#pragma unroll
                for (int i = 1; i < NW; ++i) x += s_o[i][db][lane];
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
                        a.lse[(size_t)head * a.n_tok + sq.q0 + tok] = l_all == 0.0f ? -INFINITY : (m_all * scale_log2 + __log2f(l_all)) * LN2;
                } else {
                    frag[R * D + 16 * rt + row] = m_all;
                    frag[R * D + R + 16 * rt + row] = l_all;
                }
            }
            __syncthreads();
        }
        // Sums that are no numbers, where rows see different keys: a value that a row does not see may have come in as 0 * x
        // (a product of tiles has no other way).  Those rows are done again key by key, over the keys that they see.
        if (a.causal && sq.n_q > 1) {
            if (odd) s_flag = 1;
            __syncthreads();
            if (s_flag) {
                for (int r = w; r < R && qt * R + r < n_rows; r += NW) {
                    const int rr = qt * R + r, tok = rr / a.group, head = h * a.group + rr - tok * a.group;
                    const int seen = min(min(sq.L - sq.n_q + tok + 1, sq.L), te * TK);
                    const __bf16 *q = (const __bf16 *)(a.Q.p + head * a.Q.head + (int64_t)(sq.q0 + tok) * a.Q.row);
                    float mr = -INFINITY, lr = 0.0f, acc[D / 64];
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) acc[c] = 0.0f;
                    for (int k0 = ta * TK; k0 < seen; ++k0) {
                        const int page = pages[k0 >> a.pshift];
                        if (!exists(page)) continue;
                        const size_t ph = (size_t)page * Hkv + h;
                        const int off = k0 & ((1 << a.pshift) - 1);
                        const size_t cell = ph * page_bytes + (off >> 4) * (16 * D);
                        float x = 0.0f;
#pragma unroll
                        for (int c = 0; c < D / 64; ++c) {
                            const int co = 64 * c + lane;
                            x = fmaf((float)q[co], __builtin_amdgcn_cvt_f32_fp8((int)a.pg.K8[cell + (co >> 4) * 256 + (off & 15) * 16 + (co & 15)], 0) * a.pg.kscale[ph], x);
                        }
#pragma unroll
                        for (int i = 32; i > 0; i >>= 1) x += __shfl_xor(x, i, 64);
                        const float mn = fmaxf(mr, x);
                        const float al = weight_of(mr, mn, scale_log2), pw = __builtin_amdgcn_exp2f((x - (mn == -INFINITY ? 0.0f : mn)) * scale_log2);
                        mr = mn;
                        lr = lr * al + pw;
#pragma unroll
                        for (int c = 0; c < D / 64; ++c) {
                            const int co = 64 * c + lane;
                            acc[c] = acc[c] * al + pw * (__builtin_amdgcn_cvt_f32_fp8((int)a.pg.V8[cell + (co >> 4) * 256 + (co & 15) * 16 + (off & 15)], 0) * a.pg.vscale[ph]);
                        }
                    }
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) {
                        const int co = 64 * c + lane;
                        if (whole) ((__bf16 *)(a.O.p + head * a.O.head + (int64_t)(sq.q0 + tok) * a.O.row))[co] = (__bf16)(lr == 0.0f ? 0.0f : acc[c] / lr);
                        else frag[(((r >> 4) * DB + (co >> 4)) * 64 + ((co & 15) >> 2) * 16 + (r & 15)) * 4 + (co & 3)] = acc[c];
                    }
                    if (lane == 0) {
                        if (whole) {
                            if (a.lse) a.lse[(size_t)head * a.n_tok + sq.q0 + tok] = lr == 0.0f ? -INFINITY : (mr * scale_log2 + __log2f(lr)) * LN2;
                        } else {
                            frag[R * D + r] = mr;
                            frag[R * D + R + r] = lr;
                        }
                    }
                }
            }
            __syncthreads();
        }
        if (SPLIT && begins && !ends) {
            const long long x = base + (long long)(item + 1) * per - 1;   // the item's last unit
            d = Desc{b, h, qt, (int)(((x + 1) * n_shares + W - 1) / W) - 1};
        }
    }
    if (SPLIT && tid == 0) a.desc[share] = d;
}

// Puts the fragments of an item together: a workgroup per share and block of 16 coordinates x 16 rows, most of which find
// nothing to do; its wavefronts take every fourth fragment.
template <int D, int RT>
__global__ __launch_bounds__(NW * 64) void combine_kernel(const Args a) {
    constexpr int R = 16 * RT, DB = D / 16;
    __shared__ float s_l[NW][16];
    __shared__ f32x4 s_o[NW][64];
    const Desc d = a.desc[blockIdx.x];
    if (d.last < 0) return;
    const int rt = blockIdx.y / DB, db = blockIdx.y % DB;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, row = lane & 15, quarter = lane >> 4;
    const int first = blockIdx.x, n = d.last - first + 1;
    auto frag = [&](int i) { return a.frag + (size_t)(i == 0 ? 2 * first + 1 : 2 * (first + i)) * FRAG_FLOATS; };
    float m_all = -INFINITY;
    for (int i = quarter; i < n; i += 4) m_all = fmaxf(m_all, frag(i)[R * D + 16 * rt + row]);
    m_all = max_of_quarters(m_all);
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    float l = 0.0f;
    for (int i = w; i < n; i += NW) {
        const float *f = frag(i);
        const float wt = weight_of(f[R * D + 16 * rt + row], m_all, a.scale_log2);
        x += ((const f32x4 *)f)[(rt * DB + db) * 64 + lane] * wt;
        l += f[R * D + R + 16 * rt + row] * wt;
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
    const bf16x4 y = {(__bf16)(x[0] * inv), (__bf16)(x[1] * inv), (__bf16)(x[2] * inv), (__bf16)(x[3] * inv)};
    *(bf16x4 *)(a.O.p + head * a.O.head + (int64_t)(sq.q0 + tok) * a.O.row + (16 * db + 4 * quarter) * 2) = y;
    if (a.lse && db == 0 && quarter == 0)
        a.lse[(size_t)head * a.n_tok + sq.q0 + tok] = l == 0.0f ? -INFINITY : (m_all * a.scale_log2 + __log2f(l)) * LN2;
}

template <int D, int RT>
int launch(const Args &a, int64_t items, bool split, hipStream_t s) {
    if (!split) {
        hipLaunchKernelGGL((attn_kernel<D, RT, false>), dim3((unsigned)items), dim3(NW * 64), 0, s, a);
        FASTAR_LAUNCH_CHECK();
        return FASTAR_OK;
    }
    hipLaunchKernelGGL((attn_kernel<D, RT, true>), dim3(SHARES), dim3(NW * 64), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL((combine_kernel<D, RT>), dim3(SHARES, RT * D / 16), dim3(NW * 64), 0, s, a);
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}

}  // namespace paged

size_t paged_attn_ws_bytes() {
    using namespace paged;
    return ((WS_FRAG + (size_t)2 * SHARES * FRAG_FLOATS * 4) + 255) / 256 * 256;
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
    if (dtype != FASTAR_BF16 || (int64_t)max_pages * pages->P > INT32_MAX) return FASTAR_ERR_UNSUPPORTED;
    if ((int64_t)n_tok * Hq > INT32_MAX / 2) return FASTAR_ERR_UNSUPPORTED;
    if (!ws || ((uintptr_t)ws & 255)) return FASTAR_ERR_INVALID_ARG;
    if (ws_bytes < paged_attn_ws_bytes()) return FASTAR_ERR_WORKSPACE;
    if (n_tok == 0 || B == 0) return FASTAR_OK;
    if (!cu_q || !len || !table || !view_ok(Q, 2) || !view_ok(O, 2) || !rows_apart(O, Hq, n_tok, pages->d)) return FASTAR_ERR_INVALID_ARG;
    const int group = Hq / pages->Hkv;
    const paged::Args a = {view_of(Q, 2), view_of(O, 2), cu_q, len, table, B, max_pages, n_tok, group, causal,
                           __builtin_ctz((unsigned)pages->P), *pages, scale * 1.4426950408889634f, lse,
                           (paged::Desc *)((char *)ws + paged::WS_DESC), (float *)((char *)ws + paged::WS_FRAG)};
    // rows of a tile by the rows that a sequence has on average
    const int64_t rows = ((int64_t)n_tok * group + B - 1) / B;
    const int rt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const int64_t items = (((int64_t)n_tok * group + 16 * rt - 1) / (16 * rt) + B) * pages->Hkv;   // at most
    const bool split = (int64_t)max_pages * pages->P > 512 || items > INT32_MAX;
    const hipStream_t s = (hipStream_t)stream;
    if (pages->d == 128)
        return rt == 1 ? paged::launch<128, 1>(a, items, split, s) : rt == 2 ? paged::launch<128, 2>(a, items, split, s)
                                                                              : paged::launch<128, 4>(a, items, split, s);
    return rt == 1 ? paged::launch<64, 1>(a, items, split, s) : rt == 2 ? paged::launch<64, 2>(a, items, split, s)
                                                                         : paged::launch<64, 4>(a, items, split, s);
}
