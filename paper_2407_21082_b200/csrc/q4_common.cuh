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

// ---------------------------------------------------------------------------------------------
// Softmax state of a subset of the vocabulary, like State, but with its largest term left out of the sum:
//   m = max z_v,  s = sum e^(z_v - m) - 1,  t = sum e^(z_v - m) (z_v - m),  idx = lowest v with z_v = m;  s = -1 for no logits.
// A row that is nearly certain has an entropy of about s - t with s << 1.  Next to the 1 of its largest term, s would be rounded to
// 2^-24 of 1, which is more than the last digits of such an entropy; by itself it keeps all of its own.
// The entropy of the full softmax = ln(1 + s) - t / (1 + s), the largest probability = 1 / (1 + s).
// ---------------------------------------------------------------------------------------------
struct __align__(16) RestState {
    float m, s, t;
    int idx;
};

__device__ __forceinline__ RestState rest_empty() { return RestState{-CUDART_INF_F, -1.f, 0.f, 0x7fffffff}; }

__device__ __forceinline__ RestState rest_load_cg(const RestState* p) {
    const int4 raw = __ldcg(reinterpret_cast<const int4*>(p));
    return RestState{__int_as_float(raw.x), __int_as_float(raw.y), __int_as_float(raw.z), raw.w};
}

// One more logit, indices in increasing order.
__device__ __forceinline__ void rest_push(RestState& a, float z, int idx) {
    if (z > a.m) {
        const float dl = a.m - z;                                  // <= 0, -inf for an empty state
        const bool none = a.s == -1.f;
        const float al = none ? 0.f : ex2(dl * kLog2e), n = 1.f + a.s;
        a.t = none ? 0.f : al * fmaf(dl, n, a.t);
        a.s = none ? 0.f : al * n;
        a.m = z;
        a.idx = idx;
    } else {
        const float dz = z - a.m;                                  // <= 0 (NaN propagates into s, t)
        const float e = ex2(dz * kLog2e);
        a.s += e;
        a.t = fmaf(e, dz, a.t);
    }
}

// a <- merge(a, b).  Of equal maxima the one with the lower index stays out of the sum.
__device__ __forceinline__ void rest_merge(RestState& a, const RestState& b) {
    if (b.s == -1.f) return;
    if (a.s == -1.f) { a = b; return; }
    const float m = fmaxf(a.m, b.m);
    const float da = a.m - m, db = b.m - m;                        // <= 0
    const float ea = ex2(da * kLog2e), eb = ex2(db * kLog2e);
    const bool take_a = (a.m > b.m) || (a.m == b.m && a.idx < b.idx);
    const float na = 1.f + a.s, nb = 1.f + b.s;
    const float t = ea * fmaf(da, na, a.t) + eb * fmaf(db, nb, b.t);
    a.s = ea * (take_a ? a.s : na) + eb * (take_a ? nb : b.s);
    a.t = t;
    a.idx = take_a ? a.idx : b.idx;
    a.m = m;
}

// n states (at(k)) of one row: the maximum first and then the sums, so that no step waits for the one before.  Each of the states
// that have the maximum leaves a term out; all but one of those are added at the end.
template <class At>
__device__ __forceinline__ RestState rest_combine(int n, At at) {
    float m = -CUDART_INF_F;
#pragma unroll 8
    for (int k = 0; k < n; ++k) m = fmaxf(m, at(k).m);
    float s = 0.f, t = 0.f;
    int idx = 0x7fffffff, tops = 0;
#pragma unroll 8
    for (int k = 0; k < n; ++k) {
        const RestState o = at(k);
        const bool live = !(o.s == -1.f), top = live && o.m == m;  // NaN counts as live and propagates
        const float dl = o.m - m, al = live ? ex2(dl * kLog2e) : 0.f, all = 1.f + o.s;
        s += live ? al * (top ? o.s : all) : 0.f;
        t += live ? al * fmaf(dl, all, o.t) : 0.f;
        idx = top ? min(idx, o.idx) : idx;
        tops += top ? 1 : 0;
    }
    return RestState{m, s + (float)(tops - 1), t, idx};            // no live state: s = -1
}

// The states of the lanes that differ in the bits LO .. 16 of the lane index, the result in every one of them.
template <int LO>
__device__ __forceinline__ RestState rest_reduce_lanes(const RestState& a) {
    float m = a.m;
#pragma unroll
    for (int msk = LO; msk <= 16; msk <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, msk));
    const bool live = !(a.s == -1.f), top = live && a.m == m;
    const float dl = a.m - m, al = live ? ex2(dl * kLog2e) : 0.f, all = 1.f + a.s;
    float s = live ? al * (top ? a.s : all) : 0.f;
    float t = live ? al * fmaf(dl, all, a.t) : 0.f;
    int idx = top ? a.idx : 0x7fffffff;
    constexpr unsigned lanes = LO == 1 ? 0xffffffffu : 0x11111111u;
    static_assert(LO == 1 || LO == 4, "lanes of a row");
    const int tops = __popc(__ballot_sync(0xffffffffu, top) & (lanes << (threadIdx.x & (LO - 1))));
#pragma unroll
    for (int msk = LO; msk <= 16; msk <<= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, msk);
        t += __shfl_xor_sync(0xffffffffu, t, msk);
        idx = min(idx, __shfl_xor_sync(0xffffffffu, idx, msk));
    }
    return RestState{m, s + (float)(tops - 1), t, idx};
}

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
    RestState* parts;              // [ctas][rows of the launch]
    const float* tau_per_row;
    float tau;
    int* argmax;
    float* entropy;
    float* maxprob;
    unsigned char* exit_mask;
    Control* ctrl;
};

// A row's results, and whether it may leave.
__device__ __forceinline__ void rest_finish(const RestState& a, const Q4Params& p, int row) {
    const float n = 1.f + a.s, H = log1pf(a.s) - a.t / n;
    p.argmax[row] = a.idx;
    p.entropy[row] = H;
    p.maxprob[row] = 1.f / n;
    p.exit_mask[row] = H < (p.tau_per_row ? ld_dep(p.tau_per_row + row) : p.tau) ? 1 : 0;
}

// The tensor-core kernel (q4_gemm.cu): up to kQ4GemmRows rows per launch.
constexpr int kQ4GemmRows = 64;
ee_status q4_gemm_launch(const Q4Params& p, int num_sms, int device, cudaStream_t stream);

}  // namespace ee
