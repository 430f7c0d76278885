// Matrix products of microscaled 4-bit floating point (tcgen05.mma kind::mxf4nvf4, 64 columns per instruction) and the copies that bring
// their scales to tensor memory.
#pragma once

#include "sm100_ptx.cuh"

namespace ee {
namespace ptx {

// Contiguous copy global -> shared, 16-byte aligned, a multiple of 16 bytes; its bytes are signalled on `bar`.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// Shared-memory matrix descriptors.  The thread that issues the products has some hundred cycles for a unit and takes four to five for an
// instruction, so a descriptor is a low word -- the address in 16-byte steps, which the loop moves along by additions -- and a constant high
// word: the distance of 8-row groups in 16-byte steps, version 1 (bit 14) and the swizzle (bits 29 to 31).
__device__ __forceinline__ uint32_t desc_low(uint32_t saddr) { return ((saddr & 0x3ffffu) >> 4) | (1u << 16); }
constexpr uint32_t kDescK64 = (512 >> 4) | (1u << 14) | (4u << 29);     // K-major, rows of 64 bytes, 64-byte swizzle
constexpr uint32_t kDescScales = (128 >> 4) | (1u << 14);               // 32 rows of 16 bytes, one behind the other

// 512 bytes of scales to four columns of tensor memory, the same in all four quarters of its lanes (kPair: in each CTA of a pair from its own
// shared memory to its own tensor memory).  Products issued behind it by the same thread see it.
template <bool kPair = false>
__device__ __forceinline__ void tmem_cp_scales(uint32_t taddr, uint32_t low) {
    if constexpr (kPair)
        asm volatile("{\n\t.reg .b64 d;\n\tmov.b64 d, {%1, %2};\n\ttcgen05.cp.cta_group::2.32x128b.warpx4 [%0], d;\n\t}"
                     ::"r"(taddr), "r"(low), "n"(kDescScales) : "memory");
    else
        asm volatile("{\n\t.reg .b64 d;\n\tmov.b64 d, {%1, %2};\n\ttcgen05.cp.cta_group::1.32x128b.warpx4 [%0], d;\n\t}"
                     ::"r"(taddr), "r"(low), "n"(kDescScales) : "memory");
}

// Instruction descriptor of kind::mxf4nvf4: A and B e2m1 (1 in bits [7,10) and [10,13)), both K-major, N >> 3 in bits [17,23), the scales'
// type in bit 23 (0: four exponent and three mantissa bits, 1: a power of two), M >> 4 in bits [24,29).  Where a word of scales serves two
// instructions (groups of 32), bits [4,6) and [29,31) say which half of B's and A's the instruction takes: 0 or 2.
template <int kGroup>
__host__ __device__ constexpr uint32_t idesc_fp4(int m, int n) {
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((kGroup == 32 ? 1u : 0u) << 23) | ((uint32_t)(m >> 4) << 24);
}
constexpr uint32_t kIdescFp4SecondHalf = (2u << 4) | (2u << 29);

// D[tmem] (+)= (A scales_a)[smem] * (B scales_b)[smem], fp32 accumulation; issued by one thread (of rank 0 of a pair: each CTA has its 128 rows
// of A and of D and half of B's rows, and the scales of its own rows of A and of all of B).
#define EE_MMA_FP4(cta_group, scale_vec)                                                                                                      \
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 a, {%1, %7};\n\tmov.b64 b, {%2, %7};\n\t"              \
                 "tcgen05.mma.cta_group::" cta_group ".kind::mxf4nvf4.block_scale.scale_vec::" scale_vec " [%0], a, b, %3, [%4], [%5], p;\n\t}" \
                 ::"r"(d_tmem), "r"(a_low), "r"(b_low), "r"(idesc), "r"(scales_a), "r"(scales_b), "r"(accumulate), "n"(kDescK64)              \
                 : "memory")
template <int kGroup, bool kPair = false>
__device__ __forceinline__ void mma_fp4(uint32_t d_tmem, uint32_t a_low, uint32_t b_low, uint32_t idesc, uint32_t scales_a, uint32_t scales_b,
                                        uint32_t accumulate) {
    if constexpr (kGroup == 16 && kPair) EE_MMA_FP4("2", "4X");
    else if constexpr (kGroup == 16) EE_MMA_FP4("1", "4X");
    else if constexpr (kPair) EE_MMA_FP4("2", "2X");
    else EE_MMA_FP4("1", "2X");
}
#undef EE_MMA_FP4

}  // namespace ptx
}  // namespace ee
