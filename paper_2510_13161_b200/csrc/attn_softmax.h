// A row's softmax out of tensor memory, shared by the attention kernels whose softmax warps have a thread per row (attn_verify.cu,
// attn_prompt.cu).
#pragma once
#include "attn_common.h"

namespace attn {

// A half tile whose sum of P stays below this is as it should be: no P of it overflows f16 (e4m3 cache), and sums of P V stay in
// fp32's range for values up to 2^113 (bf16 P would allow more, but values of 1e25 under P of 2^43 already overflow).
constexpr float kSumLimit = 16384.f;

// ---- packed fp32 pairs, tensor memory ---------------------------------------------------------------------------
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ void tmem_st_32x32b_x32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
          "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
          "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st_32x32b_x16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Wait for this thread's tcgen05.ld, naming the registers it filled: without the dependence the compiler may move
// arithmetic on them ahead of the wait.
__device__ __forceinline__ void tmem_ld_wait32(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]),
                   "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]),
                   "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :: "memory");
}
__device__ __forceinline__ void tmem_ld_wait16(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :: "memory");
}

// 32 scores of a row -> 16 words of bf16 (F8: f16) P = exp2(s * c - offset); the fp32 values are added to four running sums
// (two packed pairs).
template <bool F8>
__device__ __forceinline__ void exp_chunk(const uint32_t (&r)[32], uint64_t sc2, uint64_t neg_off2, uint32_t* pk, uint64_t& s0, uint64_t& s1) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        float a, b;
        unpack2(fma2(pack2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])), sc2, neg_off2), a, b);
        a = ptx::ex2_approx(a);
        b = ptx::ex2_approx(b);
        if (j & 1) s1 = add2(s1, pack2(a, b));
        else s0 = add2(s0, pack2(a, b));
        if (F8) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(pk[j]) : "f"(b), "f"(a));
        else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(pk[j]) : "f"(b), "f"(a));
    }
}

// Row maximum over chunks of 32 scores (a unit's first tile, and what is redone).
static __device__ __noinline__ float tile_max(uint32_t s_addr, int chunks) {
    float m = -INFINITY;
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
        uint32_t r[32];
        ptx::tmem_ld_32x32b_x32(s_addr + (uint32_t)(c * 32), r);
        tmem_ld_wait32(r);
#pragma unroll
        for (int j = 0; j < 32; j += 2)          // (three operands: one instruction for two scores)
            asm("max.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(__uint_as_float(r[j])), "f"(__uint_as_float(r[j + 1])));
    }
    return m;
}
// A new offset for the rows whose sum over the 64 scores at s_addr outgrew the limit (`grow`): the maximum of those scores.
// The row's accumulator (o_cols columns, 0: none yet) is rescaled to it.  Returns (offset, factor).
static __device__ __noinline__ float2 move_offset(uint32_t s_addr, uint32_t o_addr, int o_cols, bool grow, float off, float sc) {
    const float mx = tile_max(s_addr, 2);
    const float next = grow ? mx * sc : off, alpha = grow ? exp2f(off - next) : 1.f;
#pragma unroll 1
    for (int c = 0; c < o_cols; c += 16) {
        uint32_t r[16];
        ptx::tmem_ld_32x32b_x16(o_addr + (uint32_t)c, r);
        tmem_ld_wait16(r);
#pragma unroll
        for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * alpha);
        tmem_st_32x32b_x16(o_addr + (uint32_t)c, r);
    }
    tmem_st_wait();
    return make_float2(next, alpha);
}

}  // namespace attn
