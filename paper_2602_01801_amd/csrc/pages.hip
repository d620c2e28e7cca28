// The paged 8-bit cache: block tables and slot maps from the requests' lengths (kv_pages_plan), and new keys and values into
// its pages (kv_pages_write).
#include "packed.hpp"

namespace fastar {

namespace pages {

constexpr int PT = 1024;   // threads of the planning workgroup

// Inclusive prefix sum over the workgroup's PT threads (64-bit: lengths are the caller's and may be anything); the total in *all.
__device__ __forceinline__ long long wg_incl_scan(long long v, long long *part, long long *all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
    }
    __syncthreads();   // the last call's partial sums have been read
    if (lane == 63) part[wave] = v;
    __syncthreads();
    long long base = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < PT / 64; ++w) {
        const long long x = part[w];
        if (w < wave) base += x;
        sum += x;
    }
    *all = sum;
    return v + base;
}

__device__ __forceinline__ int slot_of(const int32_t *__restrict__ row, long long pos, int pshift, int n_pages) {
    const int page = row[pos >> pshift];
    return (unsigned)page < (unsigned)n_pages ? (page << pshift) + (int)(pos & ((1 << pshift) - 1)) : -1;
}

// Up to PT requests: a thread each, sums in 32 bits (the launch sees to it that they fit).  Everything that is read -- lengths, table
// entries below a request's own pages, the pool below its top -- is left as it is by the call, so that pages which go from one
// request to another by way of the pool are looked up where they come from, and tables, pool and slots are written side by side:
// two rounds of loads in all (one for lengths, one for pages), against six of the kernel for more requests.  With many tokens more
// workgroups repeat the sums and write slots only; that needs the lengths to stay in place, so not if len_out or pool_n_out is an input.
// 192 requests, a token each 14.1 -> 6.0 us, 64 prompts of 90122 tokens 13 -> 4.6; 1024 requests 5.8, 1025 by the other kernel 51, 10000 249.
constexpr int SMALL_LIMIT = 1 << 20;   // PT times this much stays below 2^31
__global__ __launch_bounds__(PT) void plan_small_kernel(const int32_t *__restrict__ n_new, const int32_t *len, int32_t *table, int B,
                                                        int max_pages, int32_t *pool, const int32_t *pool_n, int n_pages, int pshift,
                                                        int n_tok, int32_t *len_out, int32_t *pool_n_out, int32_t *__restrict__ cu,
                                                        int32_t *__restrict__ slot, int32_t *__restrict__ status, int n_slots) {
    __shared__ int part[3][PT / 64];
    __shared__ int s_rows[PT], s_back[PT], s_upto[PT], s_have[PT], s_len[PT];   // the first three: inclusive prefix sums
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int P = 1 << pshift;
    int n = 0, L = 0;
    bool ended = false;
    if (tid < B) {
        n = n_new[tid];
        L = (int)min(max((long long)len[tid], 0ll), (long long)max_pages << pshift);
        ended = n < 0;
        n = max(n, 0);
    }
    const int free0 = min(max(pool_n[0], 0), n_pages);
    const int have = (L + P - 1) >> pshift;
    int rows = (int)wave_incl_scan((unsigned)min(n, n_tok + 1)), back = (int)wave_incl_scan(ended ? (unsigned)have : 0u);
    if (lane == 63) {
        part[0][wave] = rows;
        part[1][wave] = back;
    }
    __syncthreads();
    auto add_before = [&](int which, int &v) {
        int all = 0;
#pragma unroll
        for (int i = 0; i < PT / 64; ++i) {
            const int x = part[which][i];
            if (i < wave) v += x;
            all += x;
        }
        return all;
    };
    const int n_rows = min(add_before(0, rows), n_tok), n_back = add_before(1, back);
    const int free1 = (int)min((long long)free0 + n_back, (long long)n_pages);
    const long long want = ((long long)L + n + P - 1) >> pshift;
    int st = want > max_pages ? 2 : rows > n_tok && n > 0 ? 3 : 0;
    const int ask = ended || st ? 0 : (int)max(want - have, 0ll);
    int upto = (int)wave_incl_scan((unsigned)ask);
    if (lane == 63) part[2][wave] = upto;
    __syncthreads();
    const int n_ask = add_before(2, upto);
    if (ask > 0 && upto > free1) st = 1;
    s_rows[tid] = min(rows, n_tok);
    s_back[tid] = back;
    s_upto[tid] = upto;
    s_have[tid] = have;
    s_len[tid] = st ? -1 : L;
    __syncthreads();
    auto owner = [&](const int *incl, int x) {   // the request whose part of the sums holds x
        int lo = 0, hi = B - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (incl[mid] > x) hi = mid;
            else lo = mid + 1;
        }
        return lo;
    };
    auto given_back = [&](int r) {
        const int i = owner(s_back, r);
        return table[(size_t)i * max_pages + r - (s_back[i] - s_have[i])];
    };
    auto taken = [&](int f) {   // the f-th page that is taken
        const int at = free1 - 1 - f;
        return at < free0 ? pool[at] : given_back(at - free0);
    };
    for (int t = blockIdx.x * PT + tid; t < min(n_rows, n_slots); t += gridDim.x * PT) {
        const int i = owner(s_rows, t);
        int y = -1;
        if (s_len[i] >= 0) {
            const int pos = s_len[i] + t - (i ? s_rows[i - 1] : 0), pg = pos >> pshift;
            const int page = pg < s_have[i] ? table[(size_t)i * max_pages + pg] : taken((i ? s_upto[i - 1] : 0) + pg - s_have[i]);
            if ((unsigned)page < (unsigned)n_pages) y = (page << pshift) + (pos & (P - 1));
        }
        slot[t] = y;
    }
    if (blockIdx.x) return;
    int n_take = n_ask;   // those asked for by requests before the first for which they do not suffice
    if (n_ask > free1) {
        const int i = owner(s_upto, free1);
        n_take = i ? s_upto[i - 1] : 0;
    }
    for (int f = tid; f < n_take; f += PT) {
        const int i = owner(s_upto, f);
        table[(size_t)i * max_pages + s_have[i] + f - (i ? s_upto[i - 1] : 0)] = taken(f);
    }
    for (int r = tid; r < free1 - free0; r += PT) pool[free0 + r] = given_back(r);
    if (tid < B) {
        cu[tid] = tid ? s_rows[tid - 1] : 0;
        len_out[tid] = ended ? 0 : st ? L : L + n;
        status[tid] = st;
    }
    if (tid == 0) {
        cu[B] = n_rows;
        pool_n_out[0] = free1 - n_take;
    }
}

// Any number of requests, 64-bit sums.  One workgroup: requests in rounds of PT.  Tables and the pool are updated by wavefronts, a request each, so that requests
// with many pages are copied 64 entries at a time.
template <bool SLOTS>
__global__ __launch_bounds__(PT) void plan_kernel(const int32_t *__restrict__ n_new, const int32_t *len, int32_t *table, int B,
                                                  int max_pages, int32_t *pool, const int32_t *pool_n, int n_pages, int pshift,
                                                  int n_tok, int32_t *len_out, int32_t *pool_n_out, int32_t *__restrict__ cu,
                                                  int32_t *__restrict__ slot, int32_t *__restrict__ status) {
    __shared__ long long part[PT / 64];
    __shared__ int s_first[PT], s_have[PT], s_n[PT], s_row[PT], s_len[PT];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int P = 1 << pshift;
    const long long cap = (long long)max_pages << pshift;
    const int free0 = min(max(pool_n[0], 0), n_pages);
    auto held = [&](int b) { return (int)min(max((long long)len[b], 0ll), cap); };
    // 1. pages of ended requests go back
    long long back = 0;
    for (int b0 = 0; b0 < B; b0 += PT) {
        const int b = b0 + tid;
        int have = 0;
        if (b < B && n_new[b] < 0) have = (held(b) + P - 1) >> pshift;
        long long all;
        const long long upto = wg_incl_scan(have, part, &all);
        s_have[tid] = have;
        s_first[tid] = (int)min(back + upto - have, (long long)n_pages);
        __syncthreads();
        for (int i = wave; i < min(PT, B - b0); i += PT / 64)
            for (int j = lane; j < s_have[i]; j += 64) {
                const long long at = (long long)free0 + s_first[i] + j;
                if (at < n_pages) pool[at] = table[(size_t)(b0 + i) * max_pages + j];
            }
        back += all;
        __syncthreads();
    }
    const long long free1 = min((long long)free0 + back, (long long)n_pages);
    __syncthreads();   // the pool is complete (and visible to the workgroup)
    // 2. requests take pages, in order
    long long rows = 0, need_sum = 0, taken = 0;
    for (int b0 = 0; b0 < B; b0 += PT) {
        const int b = b0 + tid;
        int n = 0, have = 0, L = 0, st = 0;
        bool ended = false;
        if (b < B) {
            ended = n_new[b] < 0;
            n = max(n_new[b], 0);
            L = held(b);
            have = (L + P - 1) >> pshift;
        }
        long long n_all;
        const long long end = rows + wg_incl_scan(n, part, &n_all);
        const long long want = ((long long)L + n + P - 1) >> pshift;
        if (want > max_pages) st = 2;
        else if (end > n_tok && n > 0) st = 3;
        const int ask = ended || st ? 0 : (int)max(want - have, 0ll);
        long long ask_all;
        const long long upto = need_sum + wg_incl_scan(ask, part, &ask_all);
        if (ask > 0 && upto > free1) st = 1;
        const int take = st ? 0 : ask;
        if (take > 0) taken = upto;   // admitted requests come first among those that ask
        s_first[tid] = (int)min(upto - ask, (long long)n_pages);
        s_have[tid] = have;
        s_n[tid] = take;
        __syncthreads();
        for (int i = wave; i < min(PT, B - b0); i += PT / 64)
            for (int j = lane; j < s_n[i]; j += 64)
                table[(size_t)(b0 + i) * max_pages + s_have[i] + j] = pool[free1 - 1 - s_first[i] - j];
        if (b < B) {
            cu[b] = (int)min(end - n, (long long)n_tok);
            if (b == B - 1) cu[B] = (int)min(end, (long long)n_tok);
            len_out[b] = ended ? 0 : st ? L : L + n;
            status[b] = st;
        }
        if constexpr (SLOTS) {
            __syncthreads();   // table entries are visible; s_n is free
            s_n[tid] = b < B ? (int)(min(end, (long long)n_tok) - min(end - n, (long long)n_tok)) : 0;
            s_row[tid] = (int)min(end - n, (long long)n_tok);
            s_len[tid] = st ? -1 : L;
            __syncthreads();
            for (int i = wave; i < min(PT, B - b0); i += PT / 64)
                for (int j = lane; j < s_n[i]; j += 64)
                    slot[s_row[i] + j] = s_len[i] < 0 ? -1 : slot_of(table + (size_t)(b0 + i) * max_pages, (long long)s_len[i] + j, pshift, n_pages);
        }
        rows += n_all;
        need_sum += ask_all;
        __syncthreads();
    }
    // the largest number taken by any thread's requests
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) taken = max(taken, (long long)__shfl_xor(taken, o, 64));
    if (lane == 0) part[wave] = taken;
    __syncthreads();
    if (tid == 0) {
        for (int w = 0; w < PT / 64; ++w) taken = max(taken, part[w]);
        pool_n_out[0] = (int)(free1 - taken);
        if (B == 0) cu[0] = 0;
    }
}

// Slots of many tokens: a thread each, its request by bisection of cu.
__global__ __launch_bounds__(256) void slots_kernel(const int32_t *__restrict__ table, int B, int max_pages, int n_pages, int pshift,
                                                    int n_tok, const int32_t *__restrict__ len_out, const int32_t *__restrict__ cu,
                                                    int32_t *__restrict__ slot, const int32_t *__restrict__ status) {
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= n_tok || t >= cu[B]) return;
    int lo = 0, hi = B;   // cu[lo] <= t < cu[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int n = cu[lo + 1] - cu[lo];
    slot[t] = status[lo] ? -1 : slot_of(table + (size_t)lo * max_pages, (long long)len_out[lo] - n + (t - cu[lo]), pshift, n_pages);
}

// ---- writing ----------------------------------------------------------------------------------------------------

constexpr float F8_MAX = 448.0f;

__device__ __forceinline__ float f8_in_range(float x) { return x != x ? x : fminf(fmaxf(x, -F8_MAX), F8_MAX); }
__device__ __forceinline__ unsigned f8_of(float a, float b, float c, float d) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f8_in_range(a), f8_in_range(b), w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f8_in_range(c), f8_in_range(d), w, true);
    return (unsigned)w;
}
__device__ __forceinline__ float finite_abs(float x) {
    x = fabsf(x);
    return x < INFINITY ? x : 0.0f;
}
// Exponent of the least power of two, 2^-100 at least, whose 448-fold is not below amax.
__device__ __forceinline__ int scale_exp(float amax) {
    int e;
    const float m = frexpf(amax, &e);   // 448 = 0.875 * 2^9
    return max(-100, amax == 0.0f ? -100 : m <= 0.875f ? e - 9 : e - 8);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
typedef __attribute__((ext_vector_type(2))) short s16x2;

// EPL consecutive elements of a row as they lie in memory.
template <bool BF16, int EPL>
struct Piece {
    static constexpr int W = EPL * (BF16 ? 2 : 4) / 4;
    unsigned w[W];
    __device__ __forceinline__ void load(const char *p) {
        if constexpr (W == 1) {
            w[0] = *(const unsigned *)p;
        } else if constexpr (W == 2) {
            const u32x2 x = *(const u32x2 *)p;
            w[0] = x[0], w[1] = x[1];
        } else {
#pragma unroll
            for (int q = 0; q < W / 4; ++q) {
                const u32x4 x = ((const u32x4 *)p)[q];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[4 * q + e] = x[e];
            }
        }
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (BF16) return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
        else return __uint_as_float(w[i]);
    }
    // Largest |x| by its bits, with what `top` holds (two 16-bit maxima for bf16): numbers that are not finite come out on top.
    __device__ __forceinline__ unsigned top(unsigned top) const {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (BF16) top = __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu)));
            else top = max(top, w[i] & 0x7FFFFFFFu);
        }
        return top;
    }
    // Codes of elements i, i + 1, in the lower or the upper half of r: the conversion instructions divide by a power of two and round
    // to nearest, ties to even (what goes beyond 464 becomes no number; here nothing goes beyond 448).
    template <bool UPPER>
    __device__ __forceinline__ void codes(int i, float scale, unsigned &r) const {
        const s16x2 old = __builtin_bit_cast(s16x2, r);
        if constexpr (BF16) r = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, __builtin_bit_cast(bf16x2, w[i / 2]), scale, UPPER));
        else r = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(old, (*this)[i], (*this)[i + 1], scale, UPPER));
    }
};
// Codes carried over to a scale 1 / ratio times as large.
__device__ __forceinline__ unsigned rescaled(unsigned w, float ratio) {
    return f8_of(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * ratio,
                 __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * ratio, __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * ratio);
}
__device__ __forceinline__ float wave_max(float x) {   // of numbers that are not negative
    return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)wave_max_last(__float_as_uint(x)), 63));
}
// Rows o .. e - 1 of a page where some number is not finite, one after the other.
template <bool BF16, int D>
__device__ __forceinline__ void write_odd_run(const char *row0, int64_t pitch, int o, int e, bool is_v, uint8_t *cell0, int page_bytes,
                                              float old_scale, float *scale_out) {
    const int lane = threadIdx.x & 63;
    auto at = [&](int r, int c) {
        const char *p = row0 + r * pitch;
        if constexpr (BF16) return bf16_bits_to_f32(((const unsigned short *)p)[c]);
        else return ((const float *)p)[c];
    };
    float amax = 0.0f;
    for (int r = o; r < e; ++r)
        for (int c = lane; c < D; c += 64) amax = fmaxf(amax, finite_abs(at(r, c)));
    const float scale = fmaxf(pow2(scale_exp(wave_max(amax))), old_scale), inv = 1.0f / scale, ratio = old_scale * inv;
    if (o > 0 && ratio < 1.0f) {
        for (int i = lane; i < page_bytes / 4; i += 64) ((unsigned *)cell0)[i] = rescaled(((unsigned *)cell0)[i], ratio);
        __threadfence();   // before other lanes' new codes go to the same words
    }
    for (int r = o; r < e; ++r)
        for (int c = lane; c < D; c += 64) {
            const float x = at(r, c) * inv;
            cell0[((r >> 4) * (D / 16) + (c >> 4)) * 256 + (is_v ? (c & 15) * 16 + (r & 15) : (r & 15) * 16 + (c & 15))] = (uint8_t)f8_of(x, x, x, x);
        }
    if (lane == 0) *scale_out = scale;
}

// A workgroup looks at `chunk` rows of one head of K or V and writes the runs that begin there, a wavefront for every 16 tokens of
// a page, whose rows stay in registers between the run's maximum and the codes.  Bound by memory: every row is read once and every
// code written once, in whole lines: K by rows, whose halves of a cell's 16 bytes neighbouring lanes exchange; V two coordinates of
// every row per lane, whose codes over the rows are the lane's 32 consecutive bytes of the page (d = 64: twice 8), exchanged within
// the lane.  (A wavefront per page and tensor with 64 registers of data, K in pieces of 64 bytes, V of 16: 76 us where this takes
// 43 for 34612 tokens x 8 heads; a third of the wavefronts were resident, and they read and wrote in turn.)
template <bool BF16, int D, int PSHIFT>
__global__ __launch_bounds__(4 << PSHIFT) void write_kernel(View Kn, View Vn, const int32_t *__restrict__ slot, int n_tok, int chunk,
                                                            fastar_pages pg) {
    constexpr int P = 1 << PSHIFT, ELT = BF16 ? 2 : 4, NW = P / 16;
    __shared__ unsigned s_top[2][NW];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = blockIdx.x % pg.Hkv, rest = blockIdx.x / pg.Hkv;
    const bool is_v = rest & 1;
    const int first = (rest >> 1) * chunk;
    const View x = is_v ? Vn : Kn;
    const char *xh = x.p + h * x.head;
    uint8_t *codes = is_v ? pg.V8 : pg.K8;
    float *scales = is_v ? pg.vscale : pg.kscale;
    const unsigned n_slots = (unsigned)pg.n_pages << PSHIFT, pitch = (unsigned)x.row;
    // rows first - 1 .. first + 127: which are valid, and which go on where the row before them ended
    auto at = [&](int t) { return t >= 0 && t < n_tok ? slot[t] : -1; };
    const int s0 = at(first + lane), s1 = at(first + 64 + lane);
    const int s_before = at(first - 1);
    const bool ok0 = (unsigned)s0 < n_slots, ok1 = (unsigned)s1 < n_slots;
    int p0 = __shfl_up(s0, 1, 64), p1 = __shfl_up(s1, 1, 64);   // all lanes together: a lane that is not there gives nothing
    if (lane == 0) {
        p0 = s_before;
        p1 = __builtin_amdgcn_readlane(s0, 63);
    }
    const unsigned long long valid = __ballot(ok0);
    const unsigned long long go0 = __ballot(ok0 && (s0 & (P - 1)) && p0 == s0 - 1), go1 = __ballot(ok1 && (s1 & (P - 1)) && p1 == s1 - 1);
    unsigned long long begin = valid & ~go0;
    if (chunk < 64) begin &= (1ull << chunk) - 1ull;
    for (int turn = 0; begin; begin &= begin - 1ull, turn ^= 1) {   // uniform over the workgroup
        const int pos = __builtin_ctzll(begin);
        const unsigned long long after = pos == 63 ? go1 : (go0 >> (pos + 1)) | (go1 << (63 - pos));   // bit i: row pos + 1 + i goes on
        const int n = 1 + (~after ? __builtin_ctzll(~after) : 63);   // at most P: a run ends with its page
        const int t0 = first + pos, sl = __builtin_amdgcn_readlane(s0, pos);
        const int page = sl >> PSHIFT, o = sl & (P - 1), e = o + n;
        const size_t ph = (size_t)page * pg.Hkv + h;
        uint8_t *page0 = codes + ph * (size_t)(D * P), *blk = page0 + wave * (16 * D);
        const float old_scale = o > 0 ? scales[ph] : 0.0f;
        const char *row0 = xh + (int64_t)(t0 - o) * x.row;   // of offset 0
        const int r0 = 16 * wave;
        const bool touches = r0 < e && r0 + 16 > o, all = r0 >= o && r0 + 16 <= e;   // rows of the run among the wavefront's 16
        auto row_of = [&](int r) { return row0 + (unsigned)min(max(r0 + r, o), e - 1) * pitch; };   // rows beside the run: one of its own again
        // K: row i RPI + lr, coordinates 8 lc .. ; V: rows VR g .., coordinates 2 c
        constexpr int LPR = D / 8, RPI = 64 / LPR, IT = 16 / RPI, VL = D / 2, VR = 16 * VL / 64;
        const int lr = lane / LPR, lc = lane % LPR, vc = lane % VL, vg = lane / VL;
        Piece<BF16, 8> k[IT];
        Piece<BF16, 2> v[VR];
        u32x2 old[4];   // of V: what is there of a block that the run covers in part
        u32x2 *vp = (u32x2 *)(blk + vc * 32 + vg * VR);   // a coordinate's VR bytes; the next one's are 16 bytes on
        auto vword = [&](int i) -> u32x2 & { return D == 128 ? vp[i] : vp[2 * i]; };   // 8 bytes: D = 128: two per coordinate
        constexpr int VW = VR / 4;   // such words: 4 or 2
        unsigned top = 0;
        if (touches) {
            if (!is_v) {
#pragma unroll
                for (int i = 0; i < IT; ++i) k[i].load(row_of(i * RPI + lr) + lc * 8 * ELT);
#pragma unroll
                for (int i = 0; i < IT; ++i) top = k[i].top(top);
            } else {
#pragma unroll
                for (int i = 0; i < VR; ++i) v[i].load(row_of(vg * VR + i) + vc * 2 * ELT);
                if (!all) {
#pragma unroll
                    for (int i = 0; i < VW; ++i) old[i] = vword(i);
                }
#pragma unroll
                for (int i = 0; i < VR; ++i) top = v[i].top(top);
            }
        }
        if constexpr (BF16) top = max(top & 0xFFFFu, top >> 16) << 16;
        top = (unsigned)__builtin_amdgcn_readlane((int)wave_max_last(top), 63);
        if constexpr (NW > 1) {
            if (lane == 0) s_top[turn][wave] = top;
            __syncthreads();   // the other half of s_top is free by the next one
#pragma unroll
            for (int i = 0; i < NW; ++i) top = max(top, s_top[turn][i]);
        }
        if (top >= 0x7F800000u) {   // some number is not finite
            if (wave == 0) write_odd_run<BF16, D>(row0, x.row, o, e, is_v, page0, D * P, old_scale, scales + ph);
            continue;
        }
        const float scale = fmaxf(pow2(scale_exp(__uint_as_float(top))), old_scale), ratio = old_scale / scale;
        const bool grows = o > 0 && ratio < 1.0f;
        if (lane == 0 && wave == 0) scales[ph] = scale;
        if (!touches && !grows) continue;
        if (!is_v) {
            u32x2 c[IT];
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                unsigned w0 = 0, w1 = 0;
                k[i].template codes<false>(0, scale, w0);
                k[i].template codes<true>(2, scale, w0);
                k[i].template codes<false>(4, scale, w1);
                k[i].template codes<true>(6, scale, w1);
                c[i] = u32x2{w0, w1};
            }
#pragma unroll
            for (int i = 0; i < IT; i += 2) {   // even lanes take row i of the pair's cell, odd ones row i + 1
                const bool odd = lane & 1;
                const u32x2 give = odd ? c[i] : c[i + 1], keep = odd ? c[i + 1] : c[i];
                const u32x2 got = {lane_of_eight<0>(give[0]), lane_of_eight<0>(give[1])};
                const int r = (i + (odd ? 1 : 0)) * RPI + lr;
                u32x4 y = odd ? u32x4{got[0], got[1], keep[0], keep[1]} : u32x4{keep[0], keep[1], got[0], got[1]};
                u32x4 *p = (u32x4 *)(blk + (lc >> 1) * 256 + r * 16);
                const bool mine = r0 + r >= o && r0 + r < e;
                if (!mine && grows) {
                    y = *p;
#pragma unroll
                    for (int q = 0; q < 4; ++q) y[q] = rescaled(y[q], ratio);
                }
                if (mine || grows) *p = y;
            }
        } else {
            unsigned c[VR / 2];   // of rows 2 i, 2 i + 1: codes of the two coordinates
#pragma unroll
            for (int i = 0; i < VR / 2; ++i) {
                c[i] = 0;
                v[2 * i].template codes<false>(0, scale, c[i]);
                v[2 * i + 1].template codes<true>(0, scale, c[i]);
            }
            u32x2 y[VW];   // coordinate by coordinate, four rows a word
#pragma unroll
            for (int co = 0; co < 2; ++co)
#pragma unroll
                for (int q = 0; q < VR / 4; ++q)
                    y[(co * (VR / 4) + q) / 2][(co * (VR / 4) + q) % 2] = __builtin_amdgcn_perm(c[2 * q + 1], c[2 * q], co ? 0x07050301u : 0x06040200u);
            if (!all) {
#pragma unroll
                for (int i = 0; i < VW; ++i) {
                    u32x2 w = touches ? old[i] : vword(i);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (grows) w[j] = rescaled(w[j], ratio);
                        const int row = r0 + vg * VR + ((2 * i + j) % (VR / 4)) * 4;   // of the word's first byte
                        unsigned mask = 0;
#pragma unroll
                        for (int b = 0; b < 4; ++b) mask |= row + b >= o && row + b < e ? 0xFFu << (8 * b) : 0u;
                        w[j] = touches ? (y[i][j] & mask) | (w[j] & ~mask) : w[j];
                    }
                    y[i] = w;
                }
            }
            if constexpr (D == 128) {
                ((u32x4 *)vp)[0] = u32x4{y[0][0], y[0][1], y[1][0], y[1][1]};
                ((u32x4 *)vp)[1] = u32x4{y[2][0], y[2][1], y[3][0], y[3][1]};
            } else {
#pragma unroll
                for (int i = 0; i < VW; ++i) vword(i) = y[i];
            }
        }
    }
}

}  // namespace pages

}  // namespace fastar

extern "C" int kv_pages_plan(const int32_t *n_new, const int32_t *len, int32_t *table, int B, int max_pages, int32_t *pool,
                             const int32_t *pool_n, int n_pages, int P, int n_tok, int32_t *len_out, int32_t *pool_n_out,
                             int32_t *cu, int32_t *slot, int32_t *status, void *stream) {
    using namespace fastar;
    if (B < 0 || n_tok < 0 || max_pages <= 0 || n_pages <= 0) return FASTAR_ERR_INVALID_ARG;
    if (!pool || !pool_n || !pool_n_out || !cu || (n_tok > 0 && !slot)) return FASTAR_ERR_INVALID_ARG;
    if (B > 0 && (!n_new || !len || !table || !len_out || !status)) return FASTAR_ERR_INVALID_ARG;
    if (!page_size_ok(P)) return FASTAR_ERR_UNSUPPORTED;
    if ((int64_t)max_pages * P > INT32_MAX || (int64_t)n_pages * P > INT32_MAX) return FASTAR_ERR_UNSUPPORTED;
    const int pshift = __builtin_ctz((unsigned)P);
    const hipStream_t s = (hipStream_t)stream;
    if (B <= pages::PT && n_tok < pages::SMALL_LIMIT && max_pages < pages::SMALL_LIMIT) {
        // One workgroup writes ONE_SLOTS slots beside the rest; beyond that there are more workgroups, or a launch of their own where the
        // call works in place.  64 prompts of 2048 / 3840 / 6400 / 16000 slots in all: one workgroup 5.6 / 6.8 / 8.7 / 14.5 us, more of them 4.9
        // each; in place one 4.5 / 5.7 / 7.6 / 13.8, a second launch 6.2 / 6.7 / 6.5 / 6.7.
        constexpr int ONE_SLOTS = 4096;
        const bool alone = len_out == len || pool_n_out == pool_n;
        const int wgs = n_tok <= ONE_SLOTS || alone ? 1 : (n_tok + pages::PT - 1) / pages::PT;
        const bool later = n_tok > ONE_SLOTS && alone;
        hipLaunchKernelGGL(pages::plan_small_kernel, dim3((unsigned)wgs), dim3(pages::PT), 0, s, n_new, len, table, B, max_pages, pool,
                           pool_n, n_pages, pshift, n_tok, len_out, pool_n_out, cu, slot, status, later ? 0 : n_tok);
        FASTAR_LAUNCH_CHECK();
        if (later) {
            hipLaunchKernelGGL(pages::slots_kernel, dim3((unsigned)((n_tok + 255) / 256)), dim3(256), 0, s, table, B, max_pages, n_pages,
                               pshift, n_tok, len_out, cu, slot, status);
            FASTAR_LAUNCH_CHECK();
        }
        return FASTAR_OK;
    }
    if (n_tok <= 4096) {
        hipLaunchKernelGGL(pages::plan_kernel<true>, dim3(1), dim3(pages::PT), 0, s, n_new, len, table, B, max_pages, pool, pool_n,
                           n_pages, pshift, n_tok, len_out, pool_n_out, cu, slot, status);
        FASTAR_LAUNCH_CHECK();
        return FASTAR_OK;
    }
    hipLaunchKernelGGL(pages::plan_kernel<false>, dim3(1), dim3(pages::PT), 0, s, n_new, len, table, B, max_pages, pool, pool_n,
                       n_pages, pshift, n_tok, len_out, pool_n_out, cu, slot, status);
    FASTAR_LAUNCH_CHECK();
    hipLaunchKernelGGL(pages::slots_kernel, dim3((unsigned)((n_tok + 255) / 256)), dim3(256), 0, s, table, B, max_pages, n_pages,
                       pshift, n_tok, len_out, cu, slot, status);
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}

namespace fastar {
int pages_check(const fastar_pages *pg) {
    if (!pg || !pg->K8 || !pg->V8 || !pg->kscale || !pg->vscale) return FASTAR_ERR_INVALID_ARG;
    if (((uintptr_t)pg->K8 & 15) || ((uintptr_t)pg->V8 & 15)) return FASTAR_ERR_INVALID_ARG;
    if (pg->n_pages <= 0 || pg->Hkv <= 0) return FASTAR_ERR_INVALID_ARG;
    if (!page_size_ok(pg->P) || (pg->d != 64 && pg->d != 128)) return FASTAR_ERR_UNSUPPORTED;
    if ((int64_t)pg->n_pages * pg->P > INT32_MAX || (int64_t)pg->Hkv * pg->P * pg->d > INT32_MAX) return FASTAR_ERR_UNSUPPORTED;
    return FASTAR_OK;
}
}  // namespace fastar

extern "C" int kv_pages_write(const fastar_pages *pages, const fastar_rows *K_new, const fastar_rows *V_new, int dtype,
                              const int32_t *slot, int n_tok, void *stream) {
    using namespace fastar;
    if (dtype != FASTAR_F32 && dtype != FASTAR_BF16) return FASTAR_ERR_INVALID_ARG;
    const int elt = dtype == FASTAR_BF16 ? 2 : 4;
    if (n_tok < 0) return FASTAR_ERR_INVALID_ARG;
    if (const int rc = pages_check(pages); rc != FASTAR_OK) return rc;
    if (n_tok == 0) return FASTAR_OK;
    if (!slot || !view_ok(K_new, pages->Hkv, n_tok, elt) || !view_ok(V_new, pages->Hkv, n_tok, elt)) return FASTAR_ERR_INVALID_ARG;
    const View k = view_of(K_new, pages->Hkv, n_tok, elt), v = view_of(V_new, pages->Hkv, n_tok, elt);
    if (k.row > MAX_PITCH || v.row > MAX_PITCH) return FASTAR_ERR_UNSUPPORTED;
    // Rows per workgroup: a page's where that makes enough of them; fewer, down to one, so that the runs of single tokens are not
    // done one after the other.  At least 1024 / 4096 / 16384 workgroups, pages of 64, 8 heads: 512 single tokens 17.5 / 19.4 / 21.7 us, 16 runs
    // of 16 4.5 / 6.0 / 6.0, 8 of 200 6.3 / 9.2 / 18.6, 8 of 4680 38.6 / 37.4 / 52; 30000 tokens of one head 9.5 / 23 / 49: for runs fewer would do.
    int chunk = pages->P;
    while (chunk > 1 && (int64_t)n_tok * pages->Hkv * 2 / chunk < 4096) chunk /= 2;
    const int64_t units = (int64_t)((n_tok + chunk - 1) / chunk) * pages->Hkv * 2;
    if (!launch_ok(units, 4 * pages->P)) return FASTAR_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)units);
#define FASTAR_WRITE(BF16, D, PSHIFT) \
    hipLaunchKernelGGL((pages::write_kernel<BF16, D, PSHIFT>), grid, dim3(4 << PSHIFT), 0, (hipStream_t)stream, k, v, slot, n_tok, chunk, *pages)
#define FASTAR_WRITE_P(BF16, D)                      \
    do {                                             \
        if (pages->P == 64) FASTAR_WRITE(BF16, D, 6); \
        else if (pages->P == 32) FASTAR_WRITE(BF16, D, 5); \
        else FASTAR_WRITE(BF16, D, 4);               \
    } while (0)
    if (dtype == FASTAR_BF16) {
        if (pages->d == 128) FASTAR_WRITE_P(true, 128);
        else FASTAR_WRITE_P(true, 64);
    } else {
        if (pages->d == 128) FASTAR_WRITE_P(false, 128);
        else FASTAR_WRITE_P(false, 64);
    }
#undef FASTAR_WRITE_P
#undef FASTAR_WRITE
    FASTAR_LAUNCH_CHECK();
    return FASTAR_OK;
}
