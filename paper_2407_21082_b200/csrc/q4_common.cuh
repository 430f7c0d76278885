// The packed form of a head in 4 bits, as its writer, its reader and the two head kernels see it.
//
// 16-row tiles; a tile is a sequence of blocks of 64 columns, 512 bytes each; lane (g, c) = (lane / 4, lane % 4) of a warp owns
// 16 bytes of a block: columns 16c .. 16c + 15 of row g, then of row g + 8.  Inside a 32-bit word (8 columns) column 2i is
// nibble i and column 2i + 1 nibble i + 4, each as q + 8, so that one shift and one logic operation make the two bf16 numbers
// 128 + (q + 8) of a register; subtracting 136 is exact.  The scales lie behind the weights: [tile][group][8] words holding
// rows g and g + 8.  Rows beyond V and columns beyond d are q = 0.
#pragma once

#include "common.cuh"

namespace ee {

struct Q4Layout {
    int tiles, blocks, groups;                   // 16-row tiles, 64-column blocks, scale groups per row
};
__host__ __device__ inline Q4Layout q4_layout(int V, int d, int group) {
    Q4Layout l;
    l.tiles = (V + 15) / 16;
    l.blocks = (d + 63) / 64;
    l.groups = (l.blocks * 64 + group - 1) / group;
    return l;
}

__device__ __forceinline__ uint32_t hsub2_bf16(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t hmul2_bf16(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Columns 2i and 2i + 1 of a word's eight, times the scale (in both halves of s2), as two bf16 numbers.
__device__ __forceinline__ uint32_t q4_pair(uint32_t word, int i, uint32_t s2) {
    const uint32_t biased = ((word >> (4 * i)) & 0x000f000fu) | 0x43004300u;      // 128 + (q + 8)
    return hmul2_bf16(hsub2_bf16(biased, 0x43084308u), s2);                       // the difference is exact, the product rounded once
}
__device__ __forceinline__ uint32_t low_twice(uint32_t v) { return __byte_perm(v, 0, 0x1010); }
__device__ __forceinline__ uint32_t high_twice(uint32_t v) { return __byte_perm(v, 0, 0x3232); }

struct Q4Params {
    const uint4* weights;
    const uint32_t* scales;
    const __nv_bfloat16* y;        // [M][d rounded up to 64], columns permuted (tensor-core kernel)
    const __nv_bfloat16* h;        // rows before the LayerNorm, stride ld_h (streaming kernel, which normalises them itself)
    long long ld_h;
    const float* gamma;
    const float* beta;
    float ln_eps;
    int M, d, V, group;
    State* parts;                  // [ctas][rows of the launch]
    const float* tau_per_row;
    float tau;
    int* argmax;
    float* entropy;
    float* maxprob;
    unsigned char* exit_mask;
    Control* ctrl;
};

// The tensor-core kernel (q4_gemm.cu): up to kQ4GemmRows rows per launch.
constexpr int kQ4GemmRows = 64;
ee_status q4_gemm_launch(const Q4Params& p, int num_sms, int device, cudaStream_t stream);

}  // namespace ee
