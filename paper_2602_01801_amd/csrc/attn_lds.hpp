// Matrix operands from LDS tiles for the attention kernels whose wavefronts share their tiles (prompt_attn.hip, paged_chunk.hip):
// reads as inline assembly with explicit waits, so that operands of one product arrive under the products before it.
#pragma once

#include "common.hpp"

namespace fastar {

namespace attn_lds {

typedef __attribute__((ext_vector_type(4))) short s16x4;

template <int OFF>
__device__ __forceinline__ s16x4 lds_read_tr16(unsigned addr) {
    s16x4 r;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "n"(OFF));
    return r;
}
template <int OFF>
__device__ __forceinline__ bf16x8 lds_read_b128(unsigned addr) {
    bf16x8 r;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "n"(OFF));
    return r;
}
// Waits until at most N LDS operations are outstanding (they complete in order): the operands named have landed then.
template <int N, int KF>
__device__ __forceinline__ void wait_k(bf16x8 (&f)[KF]) {
    if constexpr (KF == 8)
        asm volatile("s_waitcnt lgkmcnt(%8)"
                     : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]), "+v"(f[4]), "+v"(f[5]), "+v"(f[6]), "+v"(f[7])
                     : "n"(N));
    else
        asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]) : "n"(N));
}
template <int N, int DB>
__device__ __forceinline__ void wait_v(s16x4 (&f)[2][DB][2]) {
    if constexpr (DB == 4)
        asm volatile("s_waitcnt lgkmcnt(%16)"
                     : "+v"(f[0][0][0]), "+v"(f[0][0][1]), "+v"(f[0][1][0]), "+v"(f[0][1][1]), "+v"(f[0][2][0]),
                       "+v"(f[0][2][1]), "+v"(f[0][3][0]), "+v"(f[0][3][1]), "+v"(f[1][0][0]), "+v"(f[1][0][1]),
                       "+v"(f[1][1][0]), "+v"(f[1][1][1]), "+v"(f[1][2][0]), "+v"(f[1][2][1]), "+v"(f[1][3][0]),
                       "+v"(f[1][3][1])
                     : "n"(N));
    else
        asm volatile("s_waitcnt lgkmcnt(%8)"
                     : "+v"(f[0][0][0]), "+v"(f[0][0][1]), "+v"(f[0][1][0]), "+v"(f[0][1][1]), "+v"(f[1][0][0]),
                       "+v"(f[1][0][1]), "+v"(f[1][1][0]), "+v"(f[1][1][1])
                     : "n"(N));
}
template <int N, int DB>
__device__ __forceinline__ void wait_b(bf16x8 (&f)[2][DB]) {
    if constexpr (DB == 4)
        asm volatile("s_waitcnt lgkmcnt(%8)"
                     : "+v"(f[0][0]), "+v"(f[0][1]), "+v"(f[0][2]), "+v"(f[0][3]), "+v"(f[1][0]), "+v"(f[1][1]), "+v"(f[1][2]), "+v"(f[1][3])
                     : "n"(N));
    else
        asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(f[0][0]), "+v"(f[0][1]), "+v"(f[1][0]), "+v"(f[1][1]) : "n"(N));
}
// K operands of 32 keys; BASE = byte offset of the first row in the stage.  The address of operand s is exclusive or with 32 s.
template <int BASE, int KF>
__device__ __forceinline__ void read_k(bf16x8 (&f)[KF], unsigned kaddr) {
#pragma unroll
    for (int s = 0; s < KF; ++s) f[s] = lds_read_b128<BASE>(kaddr ^ (32 * s));
}
// V^T operands of 32 keys (two steps of 16) for the blocks of 32 columns; the address of block db is exclusive or with 64 db.
template <int BASE, int ROWB, int DB>
__device__ __forceinline__ void read_vt(s16x4 (&f)[2][DB][2], unsigned vaddr) {
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        f[0][db][0] = lds_read_tr16<BASE>(vaddr ^ (64 * db));
        f[0][db][1] = lds_read_tr16<BASE + 8 * ROWB>(vaddr ^ (64 * db));
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        f[1][db][0] = lds_read_tr16<BASE + 16 * ROWB>(vaddr ^ (64 * db));
        f[1][db][1] = lds_read_tr16<BASE + 24 * ROWB>(vaddr ^ (64 * db));
    }
}
template <int DB>
__device__ __forceinline__ void pv_mfma(f32x16 (&o)[DB], const s16x4 (&f)[2][DB][2], const bf16x8 (&p)[2]) {
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            struct { s16x4 a, b; } pr = {f[st][db][0], f[st][db][1]};
            bf16x8 a;
            __builtin_memcpy(&a, &pr, 16);
            o[db] = mfma_bf16_32x32x16(a, p[st], o[db]);
        }
}
__device__ __forceinline__ float max_across_halves(float x) {
    const unsigned u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Barrier that waits for this wavefront's LDS traffic but not for its outstanding tile loads; the scheduling fences keep
// register-only work of one phase from drifting into the next.
__device__ __forceinline__ void wg_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

}  // namespace attn_lds

}  // namespace fastar
