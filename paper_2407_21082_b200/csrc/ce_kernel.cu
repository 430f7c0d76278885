// Cross-entropy of a head over the whole vocabulary and its gradient (the supervised objective of paper section 3.3,
// "Losses", as a training step needs it), without keeping the M x V logits.
//
//   y = bf16(LN(h)),  z = y W^T,  lse_i = ln sum_v e^{z_iv},  ce_i = lse_i - z_i,label_i
//   G_iv = w_i (e^{z_iv - lse_i} - [v = label_i]),  dy = G W,  dW = G^T y,  and dy through the LayerNorm:
//   t = dy gamma,  dh = rstd (t - mean t - xhat mean(t xhat)),  dgamma = sum_i dy xhat,  dbeta = sum_i dy
//
// Four matrix products of 2 M V d operations each (the logits twice: they are recomputed in the backward pass), all by
// one persistent TMA + tcgen05 kernel whose mode decides which operand runs which way and what its epilogue does:
//   kStats  A = y, B = W (both K-major): per row and tile the maximum and the sum of the other exponentials, and
//           the logit at the label; nothing else leaves the chip
//   kGrad   the same product for a piece of the vocabulary; the epilogue turns it into G, rounded to bf16
//   kDy     A = G, B = W with the contraction over the vocabulary: W is read as it lies, as an MN-major operand; fp32
//           results are stored (first piece) or added (later ones, one launch after the other, so in a fixed order)
//           into one slab per split of the contraction
//   kDw     A = G, B = y with the contraction over the rows: both MN-major as they lie
// The pieces keep G at 128 MB, or a quarter of the whole where that is more, up to 512 MB (2 GB where less leaves SMs without a tile of
// dW): a piece costs three launches and, in kDy, one way of dy to memory and back.  For small batches one piece is all of it.
// G is rounded to bf16 because the tensor cores take dW and dy from it: each of its elements is off by at most 2^-8 of itself,
// independently.  The entry at a row's label is as large as all the others of the row together, and its rounding would be shared by the
// whole row of dy (with few rows dbeta was off by 3.5e-3 where its own rounding is 1.8e-3): what the rounding leaves of it is kept
// in fp32 and added to dy, times W's row, on the way back.  In dW it stays: a row of it that one label dominates is off by up to 2^-8 from G
// and 2^-8 from its own rounding.  G is held without the mean's 1 / n, which is applied to the fp32 results.  Rows whose label is outside [0, V) take no part: their
// row of G and of y is zero, whatever their hidden state holds.
//
// What bounds it, and what it measured (one B200; loss and gradient, times per step):
//   16384 x 2560 x 50304   13.5 ms (13.4 to 14.0 by box), 1.25 PFLOP/s over the four products: 0.89 of what cuBLAS sustains under the power cap
//   4096 x 1024 x 50304    1.52 ms, 1.11 PFLOP/s; tensor pipe 78 to 84 % active in the products, 69 % where G is written, at 1.6 GHz
//   1003 x 520 x 32003     210 us: tiles of nine k-blocks, a third of a product's time is its start, its end and the tile borders
//   64 x 512 x 50304       22.5 us, the loss alone: three launches for 8 us of weights
// The tensor core's accumulator cuts off what falls below its last bit, which adds up: above 1024 columns a logit is summed in parts of up to
// that many, which the epilogue adds in fp32 while the next part's products run.  lse is off by 1e-7 of itself at d = 512, 5e-7 at 1024, 4e-7 at
// 2560 (the plain form in fp32: 5e-8, 1.5e-7, 2.7e-7); in one go 1.1e-6 at 2560 and 5e-6 at 8192.  Parts of 512 columns halve that
// and cost short rows more (1003 x 520: the loss 47 us instead of 43.5); 16384 x 2560 pays 2 % for its three parts.
#include "common.cuh"
#include "layer_norm.cuh"
#include "kernels.h"
#include "sm100_operands.cuh"
#include "gemm_roles.cuh"
#include "tensor_map.h"

namespace ee {

namespace {

constexpr int BM = 128;
constexpr int BK = kRoleBK;
constexpr int BN = 256;                         // widest column tile; dy and dW take 192 or 128 where that wastes less of d
constexpr int kThreads = 576;                   // producer warp, MMA warp, sixteen epilogue warps
constexpr int kATileBytes = BM * BK * 2;
constexpr int kBarBytes = 512 + 8192;             // barriers, then two sets of 4 x 128 partial statistics (kStats)
constexpr size_t kSmemBudget = 226 * 1024;
constexpr int kMaxStages = 12;
constexpr int kAccStride = 256;
constexpr int kTmemCols = 512;
constexpr int kMinTile = 64;                    // narrowest tile of the logits
constexpr int kSegment = 16;                    // k-blocks of a logit that one accumulator sums
constexpr int kNarrowUnits = 4;                 // row tiles (of pairs: 256 rows) up to which it may be narrower than BN
constexpr int kNarrowRows = kNarrowUnits * 2 * BM;
constexpr int kMaxSplits = 32;
constexpr size_t kGradPieceBytes = (size_t)128 << 20;      // or a quarter of all of G, whichever is more,
constexpr size_t kGradMostBytes = (size_t)512 << 20;       // but no more than this, or than what gives every SM a tile of dW,
constexpr size_t kGradRoundBytes = (size_t)2 << 30;        // up to this (65536 x 512 x 128256: 32.4 ms with a quarter of G, 3.7 GB;
                                                           // 33.0 with a tile of dW for every SM, 1.2 GB; 37.7 with 512 MB)

enum CeMode { kStats, kGrad, kDy, kDw };
template <int kMode> struct Layout {
    static constexpr bool a_mn = kMode == kDw;
    static constexpr bool b_mn = kMode == kDy || kMode == kDw;
};

// A part of a row's softmax: m = its largest logit, r = sum of e^(z - m) over the others (m itself left out once); r = -1 for no
// logits.  Beside the 1 of its largest term the sum of a nearly certain row, and with it a loss of 1e-7, would be rounded to 2^-24.
struct Part {
    float m, r;
};
__device__ __forceinline__ Part no_part() { return Part{-CUDART_INF_F, -1.f}; }

struct CeMaps {
    CUtensorMap a, b;
};

struct CeParams {
    int M, d;              // token rows, width
    int m_tiles;           // 128-row tiles of the output (tokens, or vocabulary rows of dW)
    int n_tiles;           // 256-column tiles of the output
    int splits;            // kDy: parts of the contraction, each with a slab of its own
    int k_blocks;          // contraction in blocks of 64
    int seg_blocks;        // how many of them an accumulator sums: all, or (kStats, kGrad) an even number
    int n_cols;            // columns of the output that exist (vocabulary of the piece, or d)
    int m_rows;            // rows of the output that exist
    int v0;                // first vocabulary row of the piece
    int bn;                // columns of a tile: a multiple of 16 up to 256 (kStats, kGrad), 256, 192 or 128 (kDy, kDw)
    int a_rows;            // rows of A a CTA loads: 128, or 64 where no more exist (the products read on into what follows in
                           // shared memory, which reaches nothing but accumulator rows that nobody reads)
    int n_stages;
    int kbs;               // k-blocks per ring slot: 2 if the operands' widths allow one request for both, else 1
    int a_3d, b_3d;        // an MN-major operand's 64-wide blocks come with one request
    int add;               // kDy: add into the slab; kDw: add to what dW holds
    Part* parts;           // kStats: [n_tiles][M]
    float* z_label;        // kStats: [M]
    const int* labels;
    const float* lse;      // kGrad
    const float* ce;       // kGrad: the rows' losses, or NULL
    const float* dce;      // row weights, or NULL: every counted row 1, and `scale` at the end
    const float* dloss;    // fp32 [1] or NULL (one)
    const float* loss;     // loss[1] = number of counted rows
    __nv_bfloat16* G;      // kGrad: [M][ld_g]
    int ld_g;
    float* label_rest;     // kGrad: [M] what the rounding of a counted row's entry at its label left
    float* dy;             // kDy: [splits][M][d]
    __nv_bfloat16* dW;
    int sectors;           // kDw: rows of dW begin on 32-byte sectors
    int V;
    Control* ctrl;
};

// 1 / n times the incoming gradient of the mean, unless the rows carry weights of their own; 0 when no row counts.
__device__ __forceinline__ float grad_scale(const float* dce, const float* dloss, const float* loss) {
    if (dce) return 1.f;
    const float n = ld_dep(loss + 1);
    return n > 0.f ? (dloss ? ld_dep(dloss) : 1.f) / n : 0.f;
}
// Weight of a row in G: 0 for rows that do not count.
__device__ __forceinline__ float row_weight(const int* labels, const float* dce, int V, int row) {
    const int label = ld_dep(labels + row);
    if ((unsigned)label >= (unsigned)V) return 0.f;
    return dce ? ld_dep(dce + row) : 1.f;
}

// An operand tile: `rows` elements of its M or N dimension from mn0 on, kbs blocks of 64 of the contraction from k0 on.  K-major
// tiles of two blocks come as [block][row][64], MN-major ones as [64 of the rows][128 of the contraction][64]; both with one
// request where the maps allow it (three_d).
template <bool kMn, bool kPair>
__device__ __forceinline__ void load_operand(uint32_t dst, const CUtensorMap* m, int k0, int mn0, int rows, int kbs, int three_d, uint32_t bar) {
    if (!kMn) {
        if (three_d) {
            if (kPair) ptx::tma_load_3d_pair(dst, m, 0, mn0, k0 >> 6, bar);
            else ptx::tma_load_3d(dst, m, 0, mn0, k0 >> 6, bar);
        } else {
            for (int b = 0; b < kbs; ++b) {
                if (kPair) ptx::tma_load_2d_pair(dst + b * rows * 128, m, k0 + b * 64, mn0, bar);
                else ptx::tma_load_2d(dst + b * rows * 128, m, k0 + b * 64, mn0, bar);
            }
        }
    } else if (three_d) {
        if (kPair) ptx::tma_load_3d_pair(dst, m, 0, k0, mn0 >> 6, bar);
        else ptx::tma_load_3d(dst, m, 0, k0, mn0 >> 6, bar);
    } else {
        for (int c = 0; c < rows; c += 64) {
            if (kPair) ptx::tma_load_2d_pair(dst + c * 128 * kbs, m, mn0 + c, k0, bar);
            else ptx::tma_load_2d(dst + c * 128 * kbs, m, mn0 + c, k0, bar);
        }
    }
}

// exp(z - shift) of two logits: the difference and its product with log2 e are rounded one after the other, two to an instruction.
__device__ __forceinline__ float2 exp_pair(float z0, float z1, unsigned long long minus_shift) {
    const unsigned long long x = ptx::mul_f32x2(ptx::add_f32x2(ptx::pack_f32x2(z0, z1), minus_shift), ptx::pack_f32x2(kLog2e, kLog2e));
    const float2 v = ptx::unpack_f32x2(x);
    return make_float2(ex2(v.x), ex2(v.y));
}

// What a part adds to the sum of a row whose largest logit is m: without the 1 where the two are the same (`tops` counts those).
__device__ __forceinline__ float part_rest(const Part& o, float m, int& tops) {
    if (o.r == -1.f) return 0.f;                                         // NaN is not: it goes through
    if (o.m == m) {
        ++tops;
        return o.r;
    }
    return (1.f + o.r) * ex2((o.m - m) * kLog2e);
}
template <int N>
__device__ __forceinline__ Part join(const Part (&v)[N]) {
    float m = v[0].m, r = 0.f;
#pragma unroll
    for (int k = 1; k < N; ++k) m = fmaxf(m, v[k].m);
    int tops = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) r += part_rest(v[k], m, tops);
    return Part{m, r + (float)(tops - 1)};                               // no logits at all: -1
}

// The part of 64 logits (the first nvalid real).  Whole tiles take some four issue slots an element besides the exponential, two to
// leave the largest one out, so that for short rows, whose products do not hide it, the epilogue still comes near the exponentials'
// own rate (512 rows of 512: 37.5 us with the largest in the sum, 38.5 so; summing again without it where it outweighs the others
// 39, but 55 on logits so unequal that most warps have such a row).
template <bool kFull>
__device__ __forceinline__ Part fold_stats(const float (&z)[2][32], int nvalid) {
    float cm[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        if (kFull) {
            cm[j & 3] = ptx::max3(cm[j & 3], z[0][j], z[1][j]);
        } else {
            if (j < nvalid) cm[j & 3] = fmaxf(cm[j & 3], z[0][j]);
            if (32 + j < nvalid) cm[j & 3] = fmaxf(cm[j & 3], z[1][j]);
        }
    }
    const float m = ptx::max3(fmaxf(cm[0], cm[1]), cm[2], cm[3]);
    const unsigned long long minus_m = ptx::pack_f32x2(-m, -m);
    unsigned long long rest[2] = {ptx::pack_f32x2(0.f, 0.f), ptx::pack_f32x2(0.f, 0.f)}, tops[2] = {rest[0], rest[0]};
#pragma unroll
    for (int j = 0; j < 64; j += 2) {
        const float z0 = z[j >> 5][j & 31], z1 = z[j >> 5][(j & 31) + 1];
        float2 e = exp_pair(z0, z1, minus_m);
        float t0 = ptx::one_if_equal(z0, m), t1 = ptx::one_if_equal(z1, m);              // e is 1 there
        if (!kFull) {
            if (j >= nvalid) e.x = t0 = 0.f;
            if (j + 1 >= nvalid) e.y = t1 = 0.f;
        }
        const int c = (j >> 1) & 1;
        rest[c] = ptx::add_f32x2(rest[c], ptx::add_f32x2(ptx::pack_f32x2(e.x, e.y), ptx::pack_f32x2(-t0, -t1)));
        tops[c] = ptx::add_f32x2(tops[c], ptx::pack_f32x2(t0, t1));
    }
    const float2 r = ptx::unpack_f32x2(ptx::add_f32x2(rest[0], rest[1])), t = ptx::unpack_f32x2(ptx::add_f32x2(tops[0], tops[1]));
    return Part{m, (r.x + r.y) + (t.x + t.y - 1.f)};
}

// 32 consecutive values of a row (the first n of them, a multiple of eight) to memory: as bf16 in whole sectors of 32 bytes where
// rows begin on one, in halves otherwise; as fp32 (rows are multiples of 32 bytes), stored or added.
__device__ __forceinline__ void store_bf16x32(__nv_bfloat16* out, const float (&z)[32], int n, bool sectors) {
    uint32_t w[16];
#pragma unroll
    for (int q = 0; q < 16; ++q) w[q] = pack_bf16(z[2 * q], z[2 * q + 1]);
    if (sectors) {
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (q * 16 < n)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + q * 16), "r"(w[q * 8]), "r"(w[q * 8 + 1]),
                             "r"(w[q * 8 + 2]), "r"(w[q * 8 + 3]), "r"(w[q * 8 + 4]), "r"(w[q * 8 + 5]), "r"(w[q * 8 + 6]), "r"(w[q * 8 + 7])
                             : "memory");
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q * 8 < n) *reinterpret_cast<uint4*>(out + q * 8) = make_uint4(w[q * 4], w[q * 4 + 1], w[q * 4 + 2], w[q * 4 + 3]);
    }
}
__device__ __forceinline__ void store_f32x32(float* out, const float (&z)[32], int n, int add) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q * 8 >= n) break;
        const float* v = z + q * 8;
        if (add) {
            asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(out + q * 8), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory");
            asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(out + q * 8 + 4), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
        } else {
            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + q * 8), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                         "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                         : "memory");
        }
    }
}
__device__ __forceinline__ void add_bf16x32(const __nv_bfloat16* old, float (&z)[32], int n) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q * 8 >= n) break;
        const uint4 o = ld_dep(reinterpret_cast<const uint4*>(old + q * 8));
        z[q * 8 + 0] += bf16_lo(o.x); z[q * 8 + 1] += bf16_hi(o.x);
        z[q * 8 + 2] += bf16_lo(o.y); z[q * 8 + 3] += bf16_hi(o.y);
        z[q * 8 + 4] += bf16_lo(o.z); z[q * 8 + 5] += bf16_hi(o.z);
        z[q * 8 + 6] += bf16_lo(o.w); z[q * 8 + 7] += bf16_hi(o.w);
    }
}

// kSegmented: the contraction of a tile goes through several accumulators, seg_blocks k-blocks each, added up in the epilogue's registers.
template <int kMode, bool kPair, bool kSegmented>
__global__ void __launch_bounds__(kThreads, 1) ce_gemm_kernel(const __grid_constant__ CeMaps maps, const CeParams p) {
    constexpr bool a_mn = Layout<kMode>::a_mn, b_mn = Layout<kMode>::b_mn;
    const int b_rows = kPair ? p.bn / 2 : p.bn;                          // columns whose operand this CTA stages,
    const int b_blocks = b_mn ? (b_rows + 63) & ~63 : b_rows;             // whole blocks of 64 of an MN-major one
    const int kbs = p.kbs;
    const int a_block = p.a_rows * BK * 2;
    const int a_stage = a_block * kbs, b_stage = b_blocks * BK * 2 * kbs;
    const int S = p.n_stages;
    const uint32_t rank = kPair ? ptx::cluster_cta_rank() : 0u;
    const int worker = kPair ? (int)(blockIdx.x >> 1) : (int)blockIdx.x;
    const int n_workers = kPair ? (int)(gridDim.x >> 1) : (int)gridDim.x;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw_addr = ptx::smem_addr(smem_raw);
    unsigned char* smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
    const uint32_t a_base = ptx::smem_addr(smem);
    const uint32_t b_base = a_base + S * a_stage;
    unsigned char* bar_mem = smem + S * (a_stage + b_stage);
    const uint32_t bar_base = ptx::smem_addr(bar_mem);
    auto full_bar = [&](int s) { return bar_base + 8u * s; };
    auto empty_bar = [&](int s) { return bar_base + 8u * (S + s); };
    auto tfull_bar = [&](int b) { return bar_base + 8u * (2 * S + b); };
    auto tempty_bar = [&](int b) { return bar_base + 8u * (2 * S + 2 + b); };
    const uint32_t drain_bar = bar_base + 8u * (2 * S + 4);
    volatile uint32_t* tmem_holder = reinterpret_cast<volatile uint32_t*>(bar_mem + 8 * (2 * S + 5));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bar_mem + 8 * (2 * S + 5) + 4);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            ptx::mbar_init(full_bar(s), 1);
            ptx::mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(tfull_bar(b), 1);
            ptx::mbar_init(tempty_bar(b), kPair && rank == 0 ? 17 : 16);           // a CTA's epilogue warps, and the partner's word for its own
        }
        ptx::mbar_init(drain_bar, 1);
        *abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&maps.a);
        ptx::prefetch_tensormap(&maps.b);
    }
    if (warp == 1) {
        if (kPair) {
            ptx::tmem_alloc_pair(ptx::smem_addr(const_cast<uint32_t*>(tmem_holder)), kTmemCols);
            ptx::tmem_relinquish_pair();
        } else {
            ptx::tmem_alloc(ptx::smem_addr(const_cast<uint32_t*>(tmem_holder)), kTmemCols);
            ptx::tmem_relinquish();
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (kPair) ptx::cluster_sync_all();                      // the partner's barriers exist before anything signals them
    ptx::tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_holder;
    const int m_units = kPair ? (p.m_tiles + 1) >> 1 : p.m_tiles;
    const int mn_tiles = m_units * p.n_tiles;
    const int total_tiles = mn_tiles * p.splits;
    // tile -> row tile of this CTA, column tile, range of k-blocks (empty for a split that has nothing to do)
    auto locate = [&](int tile, int& m_tile, int& n_tile, int& split, int& kb0, int& kb1) {
        // one part is the rule; the general quotients, a few hundred cycles, would lie between any two tiles of every role
        split = 0;
        kb0 = 0;
        kb1 = p.k_blocks;
        if (p.splits > 1) {                                              // at most 32 parts of at most 2^24 blocks
            split = tile / mn_tiles;
            kb0 = split * p.k_blocks / p.splits;
            kb1 = (split + 1) * p.k_blocks / p.splits;
        }
        tile_coords(tile - split * mn_tiles, m_units, p.n_tiles, m_tile, n_tile);
        if (kPair) m_tile = 2 * m_tile + (int)rank;
    };
    auto load_full_bar = [&](int s) { return kPair ? ptx::map_to_cta(full_bar(s), 0) : full_bar(s); };
    const uint32_t arm_bytes = (uint32_t)(a_stage + b_stage) * (kPair ? 2u : 1u);
    // where the piece of the vocabulary lies in W: rows of B for the logits, the contraction for dy
    const int b_mn_off = (kMode == kStats || kMode == kGrad) ? p.v0 : 0;
    const int b_k_off = kMode == kDy ? p.v0 : 0;

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, armed = 0, armed_parity = 0;
            bool ok = true;
            int n_pre = 0, issued = 0;
            if ((kMode == kStats || kMode == kGrad) && worker < total_tiles) {        // W was complete before this kernel could start
                int m_tile, n_tile, split, kb0, kb1;                                  // (see ce_layer_norm_kernel): the first slots' share
                locate(worker, m_tile, n_tile, split, kb0, kb1);
                n_pre = min(S, (kb1 - kb0 + kbs - 1) / kbs);                          // of it before the wait
                for (int s = 0; s < n_pre; ++s) {
                    if (rank == 0) ptx::mbar_arrive_expect_tx(full_bar(s), arm_bytes);
                    load_operand<b_mn, kPair>(b_base + s * b_stage, &maps.b, s * kbs * BK, b_mn_off + n_tile * p.bn + (int)rank * b_rows, b_rows,
                                              kbs, p.b_3d, load_full_bar(s));
                    armed |= 1u << s;
                }
            }
            grid_dependency_wait();
            for (int tile = worker; ok && tile < total_tiles; tile += n_workers) {
                int m_tile, n_tile, split, kb0, kb1;
                locate(tile, m_tile, n_tile, split, kb0, kb1);
                for (int kb = kb0; kb < kb1; kb += kbs, ++issued) {
                    if (issued < n_pre) {
                        load_operand<a_mn, kPair>(a_base + stage * a_stage, &maps.a, kb * BK, m_tile * BM, a_mn ? BM : p.a_rows, kbs, p.a_3d, load_full_bar(stage));
                        if (++stage == S) { stage = 0; phase ^= 1u; }
                        continue;
                    }
                    if (!ptx::mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) {
                        record_failure(p.ctrl, abort_flag, 1, stage, tile);
                        ok = false;
                        break;
                    }
                    if (rank == 0) ptx::mbar_arrive_expect_tx(full_bar(stage), arm_bytes);
                    load_operand<a_mn, kPair>(a_base + stage * a_stage, &maps.a, kb * BK, m_tile * BM, a_mn ? BM : p.a_rows, kbs, p.a_3d, load_full_bar(stage));
                    load_operand<b_mn, kPair>(b_base + stage * b_stage, &maps.b, b_k_off + kb * BK,
                                              b_mn_off + n_tile * p.bn + (int)rank * b_rows, b_rows, kbs, p.b_3d, load_full_bar(stage));
                    armed |= 1u << stage;
                    armed_parity = (armed_parity & ~(1u << stage)) | (phase << stage);
                    if (++stage == S) { stage = 0; phase ^= 1u; }
                }
            }
            if (*abort_flag) producer_drain(rank, S, full_bar(0), armed, armed_parity);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = ptx::idesc_bf16_f32(kPair ? 2 * BM : BM, p.bn) | (a_mn ? ptx::kIdescAMnMajor : 0u) |
                                   (b_mn ? ptx::kIdescBMnMajor : 0u);
            constexpr uint32_t a_step = a_mn ? 2048 >> 4 : 32 >> 4, b_step = b_mn ? 2048 >> 4 : 32 >> 4;   // per K = 16
            const uint32_t mn_lead = (uint32_t)kbs * 8192u;              // from one block of 64 columns to the next
            int stage = 0;
            uint32_t phase = 0;
            int local = 0;
            bool ok = true;
            for (int tile = worker; ok && tile < total_tiles; tile += n_workers) {
                int m_tile, n_tile, split, kb0, kb1;
                locate(tile, m_tile, n_tile, split, kb0, kb1);
                for (int s0 = kb0; ok && s0 < kb1; s0 = kSegmented ? s0 + p.seg_blocks : kb1) {
                    const int s1 = kSegmented ? min(kb1, s0 + p.seg_blocks) : kb1;
                    const int buf = local & 1;
                    const uint32_t acc_phase = (uint32_t)(local >> 1) & 1u;
                    ++local;
                    if (!ptx::mbar_wait(tempty_bar(buf), acc_phase ^ 1u, abort_flag)) {
                        record_failure(p.ctrl, abort_flag, 2, 0x80 | buf, tile);
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after_sync();
                    const uint32_t d_tmem = tmem_base + (uint32_t)(buf * kAccStride);
                    for (int kb = s0; kb < s1; kb += kbs) {
                        if (!ptx::mbar_wait(full_bar(stage), phase, abort_flag)) {
                            record_failure(p.ctrl, abort_flag, 2, stage, tile);
                            ok = false;
                            break;
                        }
                        ptx::tc_fence_after_sync();
                        const uint32_t a_addr = a_base + stage * a_stage, b_addr = b_base + stage * b_stage;
                        const int blocks = min(kbs, s1 - kb);             // the range's last slot may hold one block too many
                        for (int h = 0; h < blocks; ++h) {
                            const uint64_t adesc = a_mn ? ptx::smem_desc_mn128(a_addr + h * 8192, mn_lead) : ptx::smem_desc_k128(a_addr + h * a_block);
                            const uint64_t bdesc = b_mn ? ptx::smem_desc_mn128(b_addr + h * 8192, mn_lead) : ptx::smem_desc_k128(b_addr + h * b_rows * 128);
#pragma unroll
                            for (int k = 0; k < BK / 16; ++k) {
                                const uint32_t accumulate = (kb == s0 && h == 0 && k == 0) ? 0u : 1u;
                                if (kPair) ptx::mma_bf16_ss_pair(d_tmem, adesc + a_step * k, bdesc + b_step * k, idesc, accumulate);
                                else ptx::mma_bf16_ss(d_tmem, adesc + a_step * k, bdesc + b_step * k, idesc, accumulate);
                            }
                        }
                        mma_commit_all<kPair>(empty_bar(stage));
                        if (++stage == S) { stage = 0; phase ^= 1u; }
                    }
                    if (ok) mma_commit_all<kPair>(tfull_bar(buf));
                }
            }
            if (*abort_flag) mma_drain<kPair>(drain_bar);
        } else if (lane == 0 && kPair) {
            // The second CTA's thread, which has no products to issue, passes its epilogue's hand-over on: an arrival at the
            // partner waits some 600 cycles for its release, which each of the sixteen warps would otherwise spend at every tile.
            int local = 0;
            bool ok = true;
            for (int tile = worker; ok && tile < total_tiles; tile += n_workers) {
                int m_tile, n_tile, split, kb0, kb1;
                locate(tile, m_tile, n_tile, split, kb0, kb1);
                for (int s0 = kb0; ok && s0 < kb1; s0 = kSegmented ? s0 + p.seg_blocks : kb1) {
                    const int buf = local & 1;
                    const uint32_t acc_phase = (uint32_t)(local >> 1) & 1u;
                    ++local;
                    if (!ptx::mbar_wait(tempty_bar(buf), acc_phase, abort_flag)) {
                        record_failure(p.ctrl, abort_flag, 2, 0xc0 | buf, tile);
                        ok = false;
                        break;
                    }
                    ptx::mbar_arrive_remote(ptx::map_to_cta(tempty_bar(buf), 0));
                }
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue (warps 2..17)
        // A warp takes 32 rows x 64 columns of every tile: all of it goes into registers at once, the accumulator is handed back
        // as soon as it is there, and the arithmetic runs beside the next tile's products.
        const int quarter = warp & 3;
        const int group = (warp - 2) >> 2;                  // 64 columns of the tile
        int local = 0, turn = 0;                             // accumulators taken so far; tiles, modulo two
        grid_dependency_wait();
        const float scale = kMode == kDw ? grad_scale(p.dce, p.dloss, p.loss) : 1.f;
        Part* xchg = reinterpret_cast<Part*>(bar_mem + 512);
        auto epilogue_barrier = [] { asm volatile("bar.sync 1, 512;" ::: "memory"); };
        bool given_up = false;
        for (int tile = worker; tile < total_tiles; tile += n_workers) {
            int m_tile, n_tile, split, kb0, kb1;
            locate(tile, m_tile, n_tile, split, kb0, kb1);
            if (kb0 == kb1) continue;
            const int row0 = m_tile * BM + quarter * 32, row = row0 + lane;
            const bool live = row < p.m_rows;
            const int col0 = n_tile * p.bn + group * 64;
            const int col1 = min(n_tile * p.bn + p.bn, kMode == kGrad ? (p.n_cols + 63) & ~63 : p.n_cols);     // columns of the tile end here
            const bool work = row0 < p.m_rows && col0 < col1;            // the same for the whole warp
            float weight = 0.f, lse = 0.f;
            int label = -1;
            if ((kMode == kStats || kMode == kGrad) && live) {
                label = p.labels ? (int)((unsigned)ld_dep(p.labels + row) - (unsigned)p.v0) : -1;      // any label, INT_MIN too
                if (kMode == kGrad) {
                    weight = row_weight(p.labels, p.dce, p.V, row);
                    lse = ld_dep(p.lse + row);
                }
            }
            float z[2][32];
            auto take = [&](bool first) {                                // the next accumulator into z
                const int buf = local & 1;
                const uint32_t acc_phase = (uint32_t)(local >> 1) & 1u;
                ++local;
                if (given_up || !__all_sync(0xffffffffu, ptx::mbar_wait(tfull_bar(buf), acc_phase, abort_flag))) {
                    if (!given_up && lane == 0) record_failure(p.ctrl, abort_flag, 3, buf, tile);
                    given_up = true;
                    return;
                }
                ptx::tc_fence_after_sync();
                if (work) {
                    const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * kAccStride + group * 64);
                    if (first) {
                        ptx::tmem_ld_32x32(taddr, z[0]);
                        ptx::tmem_ld_32x32(taddr + 32, z[1]);
                        ptx::tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int b = 0; b < 64; b += 16) {
                            float x[2][8];
                            ptx::tmem_ld_32x8(taddr + b, x[0]);
                            ptx::tmem_ld_32x8(taddr + b + 8, x[1]);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) z[b >> 5][(b & 31) + j] += x[j >> 3][j & 7];
                        }
                    }
                }
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(tempty_bar(buf));
            };
            take(true);
            if (kSegmented)
                for (int s0 = kb0 + p.seg_blocks; s0 < kb1 && !given_up; s0 += p.seg_blocks) take(false);
            if (given_up) {
                if (kMode == kStats) epilogue_barrier();                 // the other warps may still be on their way to it
                continue;
            }
            if (kMode == kStats) {
                Part part = no_part();
                if (work) {
                    const int nvalid = col1 - col0;
                    part = nvalid >= 64 ? fold_stats<true>(z, 64) : fold_stats<false>(z, nvalid);
                    if (live && (unsigned)(label - col0) < (unsigned)min(nvalid, 64)) {
                        float zl = 0.f;
#pragma unroll
                        for (int j = 0; j < 64; ++j) zl = (col0 + j == label) ? z[j >> 5][j & 31] : zl;
                        p.z_label[row] = zl;
                    }
                }
                // the tile's four groups of columns meet in shared memory; two buffers, so that one barrier a tile is enough
                Part* slot = xchg + turn * 512 + quarter * 32 + lane;
                turn ^= 1;
                slot[group * 128] = part;
                epilogue_barrier();
                if (group == 0 && live) {
                    const Part all[4] = {part, slot[128], slot[256], slot[384]};
                    p.parts[(size_t)n_tile * p.M + row] = join(all);
                }
                continue;
            }
            if (!work || !live) continue;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int base = col0 + c * 32;
                if (kMode == kGrad) {
                    // G, zeros in the columns that fill up the last block of 64 and in rows that take no part
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        const float2 e = exp_pair(z[c][j], z[c][j + 1], ptx::pack_f32x2(-lse, -lse));
                        const float2 g = ptx::unpack_f32x2(ptx::mul_f32x2(ptx::pack_f32x2(e.x, e.y), ptx::pack_f32x2(weight, weight)));
                        z[c][j] = g.x;
                        z[c][j + 1] = g.y;
                    }
                    if ((unsigned)(label - base) < 32u && label < col1) {               // what lies beyond col1 is another tile's
                        // p - 1 from the loss: of exp(z - lse) - 1 a nearly certain row keeps no digit, lse being rounded to 1e-6
                        float g = p.ce ? weight * expm1f(-ld_dep(p.ce + row)) : 0.f;
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (base + j == label) z[c][j] = g = p.ce ? g : z[c][j] - weight;
                        p.label_rest[row] = g - __bfloat162float(__float2bfloat16_rn(g));
                    }
                    if (weight == 0.f || base + 32 > p.n_cols) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[c][j] = (weight == 0.f || base + j >= p.n_cols) ? 0.f : z[c][j];
                    }
                    if (base < col1) store_bf16x32(p.G + (size_t)row * p.ld_g + base, z[c], col1 - base, true);
                } else if (kMode == kDy) {
                    if (base < p.n_cols) store_f32x32(p.dy + ((size_t)split * p.M + row) * p.d + base, z[c], p.n_cols - base, p.add);
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) z[c][j] *= scale;
                    __nv_bfloat16* out = p.dW + (size_t)(p.v0 + row) * p.d + base;
                    if (base < p.n_cols) {
                        if (p.add) add_bf16x32(out, z[c], p.n_cols - base);
                        store_bf16x32(out, z[c], p.n_cols - base, p.sectors);
                    }
                }
            }
        }
    }

    ptx::tc_fence_before_sync();
    __syncthreads();
    if (kPair) ptx::cluster_sync_all();       // neither CTA leaves while the other may still signal it or write its accumulators
    if (warp == 1) {
        __syncwarp();
        ptx::tc_fence_after_sync();
        if (kPair) ptx::tmem_dealloc_pair(tmem_base, kTmemCols);
        else ptx::tmem_dealloc(tmem_base, kTmemCols);
    }
}

// Vector c (columns 8c .. 8c + 7) of a row of y.  Permuted, column 16m + 4j + i of every 64 (m, j, i < 4) lies at 16j + 4m + i.
__device__ __forceinline__ void put_vec8(uint4* yrow, int c, uint4 v, int permuted) {
    if (!permuted) {
        yrow[c] = v;
        return;
    }
    uint2* block = reinterpret_cast<uint2*>(yrow + (c & ~7));            // pieces of four columns
    const int m = (c & 7) >> 1, j = 2 * (c & 1);
    block[4 * j + m] = make_uint2(v.x, v.y);
    block[4 * (j + 1) + m] = make_uint2(v.z, v.w);
}

// LayerNorm of the rows into y (rounded to fp32 and then to bf16, see layer_norm.cuh), a warp per row.  In the backward pass (`stats` given) it also leaves each row's mean
// and 1/sigma for the way back, and a row that takes no part in the gradient becomes zeros with 1/sigma = 0.
//
// Either form comes first in its call, and W, gamma and beta may have been written by whatever is in front of it in the stream, an
// optimiser's step or the packing of a table.  So neither lets the next kernel start before that has completed: every other kernel
// of the call finds the parameters complete, may request W ahead of its own wait, and reads gamma as a constant.  This one is an
// ordinary launch (a step on 4096 rows of 1024 took 1517 us so, and 1523 launched early with its parameters read through the L2);
// the other one, for small batches, is there early, waits, and then signals.
struct CeLnArgs {
    const __nv_bfloat16* h;
    long long ld_h;
    const float* gamma;
    const float* beta;
    float ln_eps;
    const int* labels;
    const float* dce;
    int V;
    __nv_bfloat16* y;
    int ld_y;              // columns of y from d on are zeros
    int permuted;          // y in the column order of the 4-bit heads (q4_gemm.cu)
    float2* stats;
    int M, d;
};

__global__ void __launch_bounds__(256) ce_layer_norm_kernel(const __grid_constant__ CeLnArgs a) {
    launch_dependents();                                                 // everything in front of this launch has completed
    const int row = blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= a.M) return;
    const int nvec = a.d >> 3;
    uint4* yrow = reinterpret_cast<uint4*>(a.y + (size_t)row * a.ld_y);
    if (nvec + lane < a.ld_y >> 3) put_vec8(yrow, nvec + lane, make_uint4(0, 0, 0, 0), a.permuted);      // fewer than eight vectors
    if (a.stats && row_weight(a.labels, a.dce, a.V, row) == 0.f) {
        for (int c = lane; c < nvec; c += 32) yrow[c] = make_uint4(0, 0, 0, 0);
        if (lane == 0) a.stats[row] = make_float2(0.f, 0.f);
        return;
    }
    const uint4* hrow = reinterpret_cast<const uint4*>(a.h + (size_t)row * a.ld_h);
    const RowStats st = row_stats_strided([&](int c) { return ld_dep(hrow + c); }, nvec, a.ln_eps, lane);
    for (int c = lane; c < nvec; c += 32) put_vec8(yrow, c, layer_norm_vec8<true>(ld_dep(hrow + c), st, a.gamma, a.beta, c), a.permuted);
    if (a.stats && lane == 0) a.stats[row] = make_float2(st.mu_f, st.rstd_f);
}

constexpr int kMergeThreads = 1024;

// The same with a CTA per row, for batches that do not fill the SMs with a warp per row: every step of the chain -- the loads,
// the sums, the normalisation -- is one vector per thread (up to four at d = 8192) instead of d / 256.
constexpr int kLnCtaThreads = 256;
__global__ void __launch_bounds__(kLnCtaThreads) ce_layer_norm_cta_kernel(const __grid_constant__ CeLnArgs a) {
    __shared__ double sums[2][kLnCtaThreads / 32];
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int nvec = a.d >> 3, warps = blockDim.x >> 5;
    float4 g[2], b[2];
    const bool first = (int)threadIdx.x < nvec;
    uint4* yrow = reinterpret_cast<uint4*>(a.y + (size_t)row * a.ld_y);
    grid_dependency_wait();
    launch_dependents();
    if (first) {                                                         // the first vector's parameters beside the row's loads
        g[0] = ld_param4_dep(a.gamma + 8 * threadIdx.x); g[1] = ld_param4_dep(a.gamma + 8 * threadIdx.x + 4);
        b[0] = ld_param4_dep(a.beta + 8 * threadIdx.x); b[1] = ld_param4_dep(a.beta + 8 * threadIdx.x + 4);
    }
    for (int c = nvec + threadIdx.x; c < a.ld_y >> 3; c += blockDim.x) put_vec8(yrow, c, make_uint4(0, 0, 0, 0), a.permuted);
    if (a.stats && row_weight(a.labels, a.dce, a.V, row) == 0.f) {
        for (int c = threadIdx.x; c < nvec; c += blockDim.x) yrow[c] = make_uint4(0, 0, 0, 0);
        if (threadIdx.x == 0) a.stats[row] = make_float2(0.f, 0.f);
        return;
    }
    const uint4* hrow = reinterpret_cast<const uint4*>(a.h + (size_t)row * a.ld_h);
    uint4 x[4];
    Moments m;
    m.clear();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int c = threadIdx.x + k * blockDim.x;
        if (c < nvec) x[k] = ld_dep(hrow + c);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if ((int)(threadIdx.x + k * blockDim.x) < nvec) m.add(x[k], k);
    auto cta_sums = [&](double& s, double& q) {                          // in a fixed order, the same bits in every thread
        warp_sum2_d(s, q);
        if (lane == 0) { sums[0][warp] = s; sums[1][warp] = q; }
        __syncthreads();
        s = q = 0.0;
        for (int w = 0; w < warps; ++w) { s += sums[0][w]; q += sums[1][w]; }
        __syncthreads();
    };
    const double d = (double)a.d, inv_d = 1.0 / d;
    double s = m.sum(), q = m.sum_sq(), mu, var;
    cta_sums(s, q);
    if (!row_variance_one_pass(s, q, d, inv_d, mu, var)) {
        double q0 = 0.0, q1 = 0.0;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if ((int)(threadIdx.x + k * blockDim.x) < nvec) vec8_sqdev_d(x[k], mu, q0, q1);
        double v = q0 + q1, none = 0.0;
        cta_sums(v, none);
        var = v * inv_d;
    }
    const RowStats st = row_stats(mu, var, a.ln_eps);
    if (first) put_vec8(yrow, threadIdx.x, layer_norm_vec8<true>(x[0], st, g[0], g[1], b[0], b[1]), a.permuted);
#pragma unroll
    for (int k = 1; k < 4; ++k) {
        const int c = threadIdx.x + k * blockDim.x;
        if (c < nvec) put_vec8(yrow, c, layer_norm_vec8<true, true>(x[k], st, a.gamma, a.beta, c), a.permuted);
    }
    if (a.stats && threadIdx.x == 0) a.stats[row] = make_float2(st.mu_f, st.rstd_f);
}

// Sum of v over the threads of a merging CTA, in a fixed order.
__device__ __forceinline__ double cta_sum_d(double v, double* part) {
    v = warp_sum_d(v);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    const double r = warp_sum_d(part[threadIdx.x & 31]);
    __syncthreads();
    return r;
}

// 32 rows per CTA, lane = row, the 32 warps stride over the parts, nine loads in flight: one turn for up to 288 parts, as many as the
// narrow tiles of some 50000 columns give (64 rows of 512: 0.3 us less than with four; more parts take more turns); then the CTA that finishes last adds up the mean over the counted rows, in a fixed order whichever
// CTA that is.
__global__ void __launch_bounds__(kMergeThreads) ce_merge_kernel(const Part* parts, int n_parts, const float* z_label, const int* labels, int M,
                                                                 int V, float* ce, float* lse, float* loss, Control* ctrl) {
    constexpr int kWarps = kMergeThreads / 32, kAhead = 9;
    __shared__ Part part[kWarps][33];
    __shared__ double sums[kWarps];
    __shared__ int is_last;
    launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.x * 32 + lane;
    grid_dependency_wait();
    Part o[1 + kAhead];                                                  // what is joined so far, and what comes next
    o[0] = no_part();
    if (row < M)
        for (int n0 = warp; n0 < n_parts; n0 += kWarps * kAhead) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int n = n0 + i * kWarps;
                o[1 + i] = no_part();
                if (n < n_parts) {
                    const float2 x = ld_dep(reinterpret_cast<const float2*>(parts) + (size_t)n * M + row);
                    o[1 + i] = Part{x.x, x.y};
                }
            }
            o[0] = join(o);
        }
    part[warp][lane] = o[0];
    __syncthreads();
    {   // one row per warp: its 32 parts, one per lane, by shuffles
        const Part mine = part[lane][warp];
        const int r = blockIdx.x * 32 + warp;
        float mm = mine.m;
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, k));
        int tops = 0;
        const float sum = warp_sum(part_rest(mine, mm, tops));
        const float rest = sum + (float)(__popc(__ballot_sync(0xffffffffu, tops > 0)) - 1);
        if (lane == 0 && r < M) {
            const float l = log1pf(rest);
            lse[r] = mm + l;
            const bool counted = (unsigned)ld_dep(labels + r) < (unsigned)V;
            ce[r] = counted ? (mm - ld_dep(z_label + r)) + l : 0.f;      // not from lse, whose rounding is 1e-6
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) is_last = ticket_arrive_is_last(&ctrl->head_ticket[0], gridDim.x) ? 1 : 0;
    __syncthreads();
    if (!is_last) return;
    double total = 0.0, n = 0.0;
    for (int i = threadIdx.x; i < M; i += kMergeThreads)
        if ((unsigned)ld_dep(labels + i) < (unsigned)V) {
            total += (double)ld_dep(ce + i);
            n += 1.0;
        }
    total = cta_sum_d(total, sums);
    n = cta_sum_d(n, sums);
    if (threadIdx.x == 0) {
        loss[0] = n > 0.0 ? (float)(total / n) : 0.f;
        loss[1] = (float)n;
        ctrl->head_ticket[0] = 0;                                       // ready for the next call
    }
}

// dy (the sum of its slabs) back through the LayerNorm, and the column sums behind dgamma and dbeta, in one pass over dy and h.
// A thread owns eight columns and walks a strip of rows, kBackRows at a time (their loads are in flight together, their two
// row sums are reduced together); the columns' threads are one of `groups` groups of a CTA that take alternate batches.
// Four rows take 96 registers (d <= 5120: 640 threads; two CTAs of 320 threads on an SM at d = 2560); above that it is one row.
struct CeBackArgs {
    const __nv_bfloat16* h;
    long long ld_h;
    const float* gamma;
    const float2* stats;
    const float* dy;       // [splits][M][d]
    int splits;
    const int* labels;     // of counted rows: the row of W that label_rest belongs to
    const float* label_rest;
    const __nv_bfloat16* W;
    int V;
    const float* dce;
    const float* dloss;
    const float* loss;
    __nv_bfloat16* dh;     // or NULL
    long long ld_dh;
    float* cols;           // [CTAs][groups][2][d] sums of dy xhat and of dy, or NULL
    int M, d;
    int warps;             // warps of a group
    int groups;
    int strip;             // rows per CTA
};
__device__ __forceinline__ void add8(float (&v)[8], const float* p) {
    const float4 a = __ldcg(reinterpret_cast<const float4*>(p)), b = __ldcg(reinterpret_cast<const float4*>(p) + 1);
    v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
    v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
}
__device__ __forceinline__ void unpack8(uint4 o, float (&x)[8]) {
    x[0] = bf16_lo(o.x); x[1] = bf16_hi(o.x); x[2] = bf16_lo(o.y); x[3] = bf16_hi(o.y);
    x[4] = bf16_lo(o.z); x[5] = bf16_hi(o.z); x[6] = bf16_lo(o.w); x[7] = bf16_hi(o.w);
}

template <int kBackRows, int kMostThreads>
__global__ void __launch_bounds__(kMostThreads) ce_back_kernel(const __grid_constant__ CeBackArgs a) {
    __shared__ float2 red[2][kBackRows][32];
    launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int group = warp / a.warps, gwarp = warp - group * a.warps;
    const int c = gwarp * 32 + lane;                                     // the thread's vector of eight columns
    const bool on = c * 8 < a.d;
    float gamma[8] = {};
    if (on) {
        const float4 g0 = ld_param4(a.gamma + c * 8), g1 = ld_param4(a.gamma + c * 8 + 4);
        gamma[0] = g0.x; gamma[1] = g0.y; gamma[2] = g0.z; gamma[3] = g0.w;
        gamma[4] = g1.x; gamma[5] = g1.y; gamma[6] = g1.z; gamma[7] = g1.w;
    }
    grid_dependency_wait();
    const float scale = grad_scale(a.dce, a.dloss, a.loss);
    const float inv_d = 1.f / (float)a.d;
    float dg[8] = {}, db[8] = {};
    const int r0 = blockIdx.x * a.strip, r1 = min(a.M, r0 + a.strip);
    const int step = kBackRows * a.groups;
    int turn = 0;
    for (int base = r0; base < r1; base += step, turn ^= 1) {
        float v[kBackRows][8];
        uint4 xw[kBackRows];                                             // h as it lies, unpacked where it is used: registers are short
        float2 st[kBackRows];
#pragma unroll
        for (int k = 0; k < kBackRows; ++k) {
            const int row = base + group * kBackRows + k;
            st[k] = make_float2(0.f, 0.f);
            xw[k] = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = 0.f;
            if (row < r1) st[k] = __ldcg(a.stats + row);
            if (on && row < r1) {
                xw[k] = ld_dep(reinterpret_cast<const uint4*>(a.h + (size_t)row * a.ld_h) + c);
                const int label = ld_dep(a.labels + row);
                if ((unsigned)label < (unsigned)a.V) {                   // a row that takes no part for its weight is dead below
                    const float rest = __ldcg(a.label_rest + row);
                    unpack8(ld_dep(reinterpret_cast<const uint4*>(a.W + (size_t)label * a.d) + c), v[k]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[k][j] *= rest;
                }
                for (int s = 0; s < a.splits; ++s) add8(v[k], a.dy + ((size_t)s * a.M + row) * a.d + c * 8);
            }
        }
#pragma unroll
        for (int k = 0; k < kBackRows; ++k) {
            float sum = 0.f, dot = 0.f, x[8];
            unpack8(xw[k], x);
            const bool dead = st[k].y == 0.f;                            // takes no part, whatever it holds
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float xhat = dead ? 0.f : (x[j] - st[k].x) * st[k].y;
                if (dead) v[k][j] = 0.f;
                dg[j] = fmaf(v[k][j], xhat, dg[j]);
                db[j] += v[k][j];
                const float t = v[k][j] * gamma[j];
                sum += t;
                dot = fmaf(t, xhat, dot);
            }
            sum = warp_sum(sum);
            dot = warp_sum(dot);
            if (lane == 0) red[turn][k][warp] = make_float2(sum, dot);
        }
        if (!a.dh) continue;
        __syncthreads();                                                 // `red` of two turns ago is read before anyone writes it again
#pragma unroll
        for (int k = 0; k < kBackRows; ++k) {
            const int row = base + group * kBackRows + k;
            float c1 = 0.f, c2 = 0.f;
            for (int w = 0; w < a.warps; ++w) {
                const float2 o = red[turn][k][group * a.warps + w];
                c1 += o.x;
                c2 += o.y;
            }
            c1 *= inv_d;
            c2 *= inv_d;
            const float f = scale * st[k].y;
            if (on && row < r1) {
                float x[8];
                unpack8(xw[k], x);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float xhat = st[k].y != 0.f ? (x[j] - st[k].x) * st[k].y : 0.f;
                    v[k][j] = f * (v[k][j] * gamma[j] - c1 - xhat * c2);
                }
                *(reinterpret_cast<uint4*>(a.dh + (size_t)row * a.ld_dh) + c) =
                    make_uint4(pack_bf16(v[k][0], v[k][1]), pack_bf16(v[k][2], v[k][3]), pack_bf16(v[k][4], v[k][5]), pack_bf16(v[k][6], v[k][7]));
            }
        }
    }
    if (a.cols && on) {
        float4* out = reinterpret_cast<float4*>(a.cols + ((size_t)blockIdx.x * a.groups + group) * 2 * a.d + c * 8);
        out[0] = make_float4(dg[0], dg[1], dg[2], dg[3]);
        out[1] = make_float4(dg[4], dg[5], dg[6], dg[7]);
        out = reinterpret_cast<float4*>(a.cols + (((size_t)blockIdx.x * a.groups + group) * 2 + 1) * a.d + c * 8);
        out[0] = make_float4(db[0], db[1], db[2], db[3]);
        out[1] = make_float4(db[4], db[5], db[6], db[7]);
    }
}

// The strips' column sums: 32 columns per CTA, 32 groups of strips, joined in order.
__global__ void __launch_bounds__(1024) ce_colsum_kernel(const float* part, int strips, int d, const float* dce, const float* dloss,
                                                        const float* loss, int add, __nv_bfloat16* dgamma, __nv_bfloat16* dbeta) {
    __shared__ float red[32][32];
    launch_dependents();
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const int i = blockIdx.x * 32 + lane;
    grid_dependency_wait();
    float s = 0.f;
    if (i < 2 * d) {
#pragma unroll 8
        for (int k = group; k < strips; k += 32) s += ld_dep(part + (size_t)k * 2 * d + i);
    }
    red[group][lane] = s;
    __syncthreads();
    if (group != 0 || i >= 2 * d) return;
#pragma unroll 8
    for (int k = 1; k < 32; ++k) s += red[k][lane];
    __nv_bfloat16* out = i < d ? dgamma + i : dbeta + (i - d);
    s *= grad_scale(dce, dloss, loss);
    if (add) s += __bfloat162float(*out);
    *out = __float2bfloat16_rn(s);
}

// ---------------------------------------------------------------------------------------------------- host

bool make_map(CUtensorMap* map, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides,
              const cuuint32_t* box, CUtensorMapL2promotion promo = CU_TENSOR_MAP_L2_PROMOTION_L2_128B) {
    EncodeTiledFn fn = encode_tiled_fn();
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn && fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, promo, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// bf16 [rows, cols] with row stride ld, boxes of box_rows x 64 columns.
bool map_2d(CUtensorMap* map, const void* base, int rows, int cols, int ld, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {64u, (cuuint32_t)box_rows};
    return make_map(map, 2, base, dims, strides, box);
}
// The same as blocks of 64 columns (whole ones: cols % 64 == 0), box_rows x box_blocks of them with one request.
bool map_blocks(CUtensorMap* map, const void* base, int rows, int cols, int ld, int box_rows, int box_blocks) {
    const cuuint64_t dims[3] = {64u, (cuuint64_t)rows, (cuuint64_t)(cols / 64)}, strides[2] = {(cuuint64_t)ld * 2, 128u};
    const cuuint32_t box[3] = {64u, (cuuint32_t)box_rows, (cuuint32_t)box_blocks};
    return make_map(map, 3, base, dims, strides, box);
}
// A K-major operand: `rows` of it, kbs k-blocks at a time; two with one request where the columns are whole blocks.
bool map_k(CUtensorMap* map, int* three_d, const void* base, int rows, int cols, int ld, int box_rows, int kbs) {
    *three_d = kbs == 2 && cols % 64 == 0;
    return *three_d ? map_blocks(map, base, rows, cols, ld, box_rows, 2) : map_2d(map, base, rows, cols, ld, box_rows);
}
// An MN-major operand: bf16 [rows (contraction), cols], `width` columns of it and kbs blocks of 64 rows at a time; with one
// request where the columns and the width are whole blocks.
bool map_mn(CUtensorMap* map, int* three_d, const void* base, int rows, int cols, int ld, int width, int kbs) {
    *three_d = cols % 64 == 0 && width % 64 == 0;
    return *three_d ? map_blocks(map, base, rows, cols, ld, 64 * kbs, width / 64) : map_2d(map, base, rows, cols, ld, 64 * kbs);
}

int tiles(int n, int t) { return (n + t - 1) / t; }

// Piece of the vocabulary, splits of dy's contraction, tile width of dy and dW, and the layout of the last step (fixed by the
// sizes alone: the workspace is sized with them).
int back_rows(int d) { return d <= 5120 ? 4 : 1; }
struct CePlan {
    int piece, n_pieces, splits, bn;
    int back_warps, back_groups, back_strip, back_ctas;
};
CePlan ce_plan(int M, int d, int V) {
    CePlan c;
    const int rows = M > 0 ? M : 1;
    // the width that computes the fewest columns beyond d; a tile costs about 32 columns more than its own (loads, hand-over)
    c.bn = 256;
    for (int w = 192; w >= 128; w -= 64)
        if (tiles(d, w) * (w + 32) < tiles(d, c.bn) * (c.bn + 32)) c.bn = w;
    const bool pair = M > BM;
    const int m_units = pair ? tiles(M, 2 * BM) : 1, n_tiles = tiles(d, c.bn), vocab_units = tiles(V, 2 * BM);
    const long long workers = pair ? 74 : 148;
    auto rounds = [](long long n, long long w) { return (n + w - 1) / w; };
    // Splits of dy's contraction over `units` blocks of 256: rounds of tiles over the workers, in k-blocks, and a slab's way to memory
    // and back (5 TB/s against 22 TFLOP/s of a pair of SMs on 256 x bn x 64: some 0.0042 k-blocks per row and column / 256).
    const double slab = (double)rows * d * 8.0 / 5e12 / ((pair ? 256.0 : 128.0) * c.bn * 2.0 * BK / (pair ? 22e12 : 11e12));
    auto dy_cost = [&](int units, int s) { return (double)rounds((long long)m_units * n_tiles * s, workers) / s * (units * 4.0) + s * slab; };
    // Pieces of the vocabulary in units of 256 columns, from the most that G may take down to half of that: the ones whose tiles come out
    // at whole rounds over the SMs, counted in k-blocks of a 256-wide tile; a launch costs about 20 of them.
    auto units_in = [&](size_t bytes) { return (long long)(bytes / 2) / rows / (2 * BM); };
    long long cap = tiles(74, n_tiles), most = vocab_units / 4;
    if (cap > units_in(kGradRoundBytes)) cap = units_in(kGradRoundBytes);
    if (cap < units_in(kGradMostBytes)) cap = units_in(kGradMostBytes);
    if (most > cap) most = cap;
    if (most < units_in(kGradPieceBytes)) most = units_in(kGradPieceBytes);
    if (most < 1) most = 1;
    if (most > vocab_units) most = vocab_units;
    double best = 0;
    int best_units = 0;
    const int step = most > 256 ? (int)(most / 128) : 1;
    for (int units = (int)most; units >= 1 && (units * 2 > most || best_units == 0); units -= step) {
        const int full = vocab_units / units, rest = vocab_units - full * units;
        auto piece_cost = [&](int u) {
            return u == 0 ? 0.0 : 60.0 + (double)rounds((long long)m_units * u, workers) * tiles(d, BK) +
                                  (double)rounds((long long)u * n_tiles, 74) * tiles(rows, BK) * (c.bn / 256.0) + dy_cost(u, 1) * (c.bn / 256.0);
        };
        const double cost = full * piece_cost(units) + piece_cost(rest);
        if (best_units == 0 || cost < best) {
            best = cost;
            best_units = units;
        }
    }
    c.piece = best_units * 2 * BM;
    c.n_pieces = tiles(V, c.piece);
    c.splits = 1;
    for (int s = 2; s <= kMaxSplits && s <= best_units && s * 4 <= tiles(c.piece < V ? c.piece : V, BK); ++s)
        if (dy_cost(best_units, s) < dy_cost(best_units, c.splits)) c.splits = s;
    c.back_warps = tiles(d / 8, 32);
    c.back_groups = c.back_warps >= 8 ? 1 : 8 / c.back_warps;
    const int batch = back_rows(d) * c.back_groups;
    c.back_strip = tiles(tiles(rows, batch), 296) * batch;                // two CTAs per SM, whole batches
    c.back_ctas = tiles(rows, c.back_strip);
    return c;
}

struct CeSpace {
    size_t y, stats, parts, z_label, label_rest, g, dy, cols, total;
};
CeSpace ce_space(int M, int d, int V, bool grad) {
    CeSpace s;
    size_t at = kCtrlBytes;
    auto take = [&](size_t n) { const size_t o = at; at = align_up(at + n, 256); return o; };
    s.y = take((size_t)M * tiles(d, 64) * 128);
    s.stats = take((size_t)M * 8);
    const int narrow = M < kNarrowRows ? M : kNarrowRows;                // rows that logit_tile may give tiles narrower than BN
    const size_t wide_parts = (size_t)tiles(V, BN) * M, narrow_parts = (size_t)tiles(V, kMinTile) * narrow;
    s.parts = take((wide_parts > narrow_parts ? wide_parts : narrow_parts) * sizeof(Part));
    s.z_label = take((size_t)M * 4);
    s.label_rest = s.g = s.dy = s.cols = at;
    if (grad) {
        const CePlan c = ce_plan(M, d, V);
        s.label_rest = take((size_t)M * 4);
        s.g = take((size_t)M * c.piece * 2);
        s.dy = take((size_t)c.splits * M * d * 4);
        s.cols = take((size_t)c.back_ctas * c.back_groups * 2 * d * 4);
    }
    s.total = at;
    return s;
}

// Bytes of one k-block of both operands, and the ring slots that fit.
size_t slot_bytes(int kMode, bool pair, int bn, int a_rows) {
    const int b_rows = pair ? bn / 2 : bn;
    return (size_t)a_rows * BK * 2 + (size_t)((kMode == kDy || kMode == kDw) ? (b_rows + 63) / 64 * 64 : b_rows) * BK * 2;
}
constexpr size_t kFixedSmem = kBarBytes + 1024;
int ring_stages(int kMode, bool pair, int bn, int a_rows, int kbs) {
    const size_t n = (kSmemBudget - kFixedSmem) / (slot_bytes(kMode, pair, bn, a_rows) * kbs);
    return (int)(n < (size_t)kMaxStages ? n : (size_t)kMaxStages);
}
// Two k-blocks per slot -- one request per operand where its columns are whole blocks of 64 -- if three such slots fit (tiles of 256 by
// pairs: they do).  EE_GEMM_K2=0 keeps one.
int blocks_per_slot(int kMode, bool pair, int bn, int a_rows) {
    static const bool on = !(getenv("EE_GEMM_K2") && getenv("EE_GEMM_K2")[0] == '0');
    return on && ring_stages(kMode, pair, bn, a_rows, 2) >= 3 ? 2 : 1;
}

// Width of the logits' tiles: 256 for more than four row tiles, else the multiple of 16 from kMinTile on that makes rounds x (width + 16) smallest
// (the CTAs take whole rounds of tiles: 197 tiles of 256 on 148 SMs are two rounds, as are 286 of 176).
int logit_tile(int M, bool pair, int V, int workers) {
    const int m_units = tiles(M, pair ? 2 * BM : BM);
    if (m_units > kNarrowUnits) return BN;
    int best = BN;
    long long best_cost = -1;
    for (int bn = kMinTile; bn <= BN; bn += 16) {
        const long long cost = (((long long)m_units * tiles(V, bn) + workers - 1) / workers) * (bn + 16);
        if (best_cost < 0 || cost <= best_cost) {
            best = bn;
            best_cost = cost;
        }
    }
    return best;
}

// k-blocks of a logit that an accumulator sums, the same for the loss and its gradient, whose logits have to be the same: up to
// kSegment, in parts as equal as pairs of blocks allow.
int logit_segment(int k_blocks) { return (tiles(k_blocks, tiles(k_blocks, kSegment)) + 1) / 2 * 2; }

// Two-CTA clusters the device runs at once; 0 if the query fails or EE_GEMM_PAIRS=0 switches pairs off.
int resident_pairs(int device) {
    static int pairs[kMaxDevices];
    static bool asked[kMaxDevices] = {};
    if (!asked[device]) {
        int n = 0;
        const char* e = getenv("EE_GEMM_PAIRS");
        if (!(e && e[0] == '0') && cudaFuncSetAttribute(ce_gemm_kernel<kGrad, true, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                        (int)kSmemBudget) == cudaSuccess) {
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute attr[2];
            pair_launch_config(cfg, attr, dim3(2), kThreads, kSmemBudget, nullptr);
            if (cudaOccupancyMaxActiveClusters(&n, ce_gemm_kernel<kGrad, true, false>, &cfg) != cudaSuccess) {
                n = 0;
                (void)cudaGetLastError();
            }
        }
        pairs[device] = n;
        asked[device] = true;
    }
    return pairs[device];
}

template <int kMode, bool kPair, bool kSegmented>
ee_status launch_mode(const CeMaps& maps, CeParams p, int workers, int device, cudaStream_t stream) {
    static bool configured[kMaxDevices] = {};
    if (!configured[device]) {
        if (cudaFuncSetAttribute(ce_gemm_kernel<kMode, kPair, kSegmented>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBudget) != cudaSuccess)
            return EE_ERR_CUDA;
        configured[device] = true;
    }
    p.n_stages = ring_stages(kMode, kPair, p.bn, p.a_rows, p.kbs);
    const size_t smem = p.n_stages * p.kbs * slot_bytes(kMode, kPair, p.bn, p.a_rows) + kFixedSmem;
    const long long total = (long long)(kPair ? (p.m_tiles + 1) / 2 : p.m_tiles) * p.n_tiles * p.splits;
    const int grid = (int)(total < workers ? total : workers);
    const cudaError_t e = kPair ? launch_pdl_pairs(ce_gemm_kernel<kMode, kPair, kSegmented>, 2 * grid, kThreads, smem, stream, maps, p)
                                : launch_pdl(ce_gemm_kernel<kMode, kPair, kSegmented>, grid, kThreads, smem, stream, maps, p);
    return e == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

// Pairs of CTAs on 256-row tiles when the output has more than 128 rows and the device can run them: with and without them a step
// takes 1527 and 1768 us on 4096 rows of 1024, 211 and 231 us on 1003 of 520; the loss of 1003 rows of 1024 87 and 99 us.
bool use_pairs(int rows, int device) { return rows > BM && resident_pairs(device) > 0; }
template <int kMode, bool kSegmented>
ee_status launch_part(const CeMaps& maps, const CeParams& p, bool pair, const CeArgs& a) {
    return pair ? launch_mode<kMode, true, kSegmented>(maps, p, resident_pairs(a.device), a.device, a.stream)
                : launch_mode<kMode, false, kSegmented>(maps, p, a.num_sms, a.device, a.stream);
}
template <int kMode>
ee_status launch_product(const CeMaps& maps, const CeParams& p, bool pair, const CeArgs& a) {
    if constexpr (kMode == kStats || kMode == kGrad)
        if (p.seg_blocks < p.k_blocks) return launch_part<kMode, true>(maps, p, pair, a);
    return launch_part<kMode, false>(maps, p, pair, a);
}

CeLnArgs ln_args(const CeArgs& a, const CeSpace& s, bool grad) {
    unsigned char* ws = static_cast<unsigned char*>(a.workspace);
    CeLnArgs l;
    l.h = static_cast<const __nv_bfloat16*>(a.h);
    l.ld_h = a.ld_h; l.gamma = a.gamma; l.beta = a.beta; l.ln_eps = a.ln_eps;
    l.labels = a.labels; l.dce = a.dce; l.V = a.V;
    l.y = reinterpret_cast<__nv_bfloat16*>(ws + s.y);
    l.ld_y = tiles(a.d, 64) * 64;
    l.permuted = 0;
    l.stats = grad ? reinterpret_cast<float2*>(ws + s.stats) : nullptr;
    l.M = a.M; l.d = a.d;
    return l;
}

CeParams base_params(const CeArgs& a) {
    CeParams p{};
    p.M = a.M; p.d = a.d; p.V = a.V;
    p.splits = 1;
    p.bn = BN;
    p.a_rows = BM;
    p.labels = a.labels; p.lse = a.lse; p.ce = a.ce_in; p.dce = a.dce; p.dloss = a.dloss; p.loss = a.loss;
    p.dW = static_cast<__nv_bfloat16*>(a.dW);
    p.ctrl = reinterpret_cast<Control*>(a.workspace);
    return p;
}

}  // namespace

// A CTA per row up to kLnCtaRows rows, above that a warp per row: the loss takes 31.0 us with a CTA and 32.9 with a warp per row on 64
// rows of 1024 (V = 50304), 86.8 and 87.0 on 1003, 107.3 and 106.2 on 2048 (V = 32003).
constexpr int kLnCtaRows = 1024;
static ee_status ln_launch(const CeLnArgs& l, cudaStream_t stream) {
    if (l.M <= kLnCtaRows) {
        const int warps = (l.d / 8 + 31) / 32;
        return launch_pdl(ce_layer_norm_cta_kernel, dim3(l.M), 32 * (warps < 8 ? warps : 8), 0, stream, l) == cudaSuccess ? EE_OK : EE_ERR_CUDA;
    }
    ce_layer_norm_kernel<<<(l.M + 7) / 8, 256, 0, stream>>>(l);
    return cudaGetLastError() == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

ee_status layer_norm_permuted_launch(const void* h, long long ld_h, const float* gamma, const float* beta, float ln_eps, void* y, int ld_y,
                                     int M, int d, cudaStream_t stream) {
    CeLnArgs l{};
    l.h = static_cast<const __nv_bfloat16*>(h);
    l.ld_h = ld_h; l.gamma = gamma; l.beta = beta; l.ln_eps = ln_eps;
    l.y = static_cast<__nv_bfloat16*>(y);
    l.ld_y = ld_y;
    l.permuted = 1;
    l.M = M; l.d = d;
    return ln_launch(l, stream);
}

size_t ce_workspace_bytes(int M, int d, int V, bool grad) { return ce_space(M, d, V, grad).total; }

ee_status ce_launch(const CeArgs& a) {
    unsigned char* ws = static_cast<unsigned char*>(a.workspace);
    const CeSpace s = ce_space(a.M, a.d, a.V, false);
    const CeLnArgs l = ln_args(a, s, false);
    const ee_status ln = ln_launch(l, a.stream);
    if (ln != EE_OK) return ln;
    const bool pair = use_pairs(a.M, a.device);
    CeMaps maps;
    CeParams p = base_params(a);
    p.bn = logit_tile(a.M, pair, a.V, pair ? resident_pairs(a.device) : a.num_sms);
    p.a_rows = a.M <= 64 ? 64 : BM;
    p.kbs = blocks_per_slot(kStats, pair, p.bn, p.a_rows);
    if (!map_k(&maps.a, &p.a_3d, l.y, a.M, l.ld_y, l.ld_y, p.a_rows, p.kbs) || !map_k(&maps.b, &p.b_3d, a.W, a.V, a.d, a.d, pair ? p.bn / 2 : p.bn, p.kbs)) return EE_ERR_CUDA;
    p.m_tiles = tiles(a.M, BM);
    p.n_tiles = tiles(a.V, p.bn);
    p.k_blocks = tiles(a.d, BK);
    p.seg_blocks = logit_segment(p.k_blocks);
    p.n_cols = a.V;
    p.m_rows = a.M;
    p.parts = reinterpret_cast<Part*>(ws + s.parts);
    p.z_label = reinterpret_cast<float*>(ws + s.z_label);
    const ee_status st = launch_product<kStats>(maps, p, pair, a);
    if (st != EE_OK) return st;
    const int n_parts = p.n_tiles;
    if (launch_pdl(ce_merge_kernel, (a.M + 31) / 32, kMergeThreads, 0, a.stream, (const Part*)p.parts, n_parts, (const float*)p.z_label, a.labels,
                   a.M, a.V, a.ce, a.lse_out, a.loss_out, p.ctrl) != cudaSuccess)
        return EE_ERR_CUDA;
    return EE_OK;
}

ee_status ce_grad_launch(const CeArgs& a) {
    unsigned char* ws = static_cast<unsigned char*>(a.workspace);
    const CeSpace s = ce_space(a.M, a.d, a.V, true);
    const CePlan c = ce_plan(a.M, a.d, a.V);
    const CeLnArgs l = ln_args(a, s, true);
    const ee_status ln = ln_launch(l, a.stream);
    if (ln != EE_OK) return ln;
    const bool pair = use_pairs(a.M, a.device);
    const bool need_dy = a.dh || a.dgamma;
    const int ld_g = c.piece;
    __nv_bfloat16* G = reinterpret_cast<__nv_bfloat16*>(ws + s.g);
    float* dy = reinterpret_cast<float*>(ws + s.dy);

    for (int i = 0; i < c.n_pieces; ++i) {
        const int v0 = i * c.piece, nv = a.V - v0 < c.piece ? a.V - v0 : c.piece;
        const int nv_pad = (nv + 63) / 64 * 64;                          // the columns of G that are written, tiles enough for all (zeros beyond nv)
        CeMaps maps;
        CeParams p = base_params(a);
        p.v0 = v0;
        {
            p.bn = logit_tile(a.M, pair, nv, pair ? resident_pairs(a.device) : a.num_sms);
            p.a_rows = a.M <= 64 ? 64 : BM;
            p.kbs = blocks_per_slot(kGrad, pair, p.bn, p.a_rows);
            if (!map_k(&maps.a, &p.a_3d, l.y, a.M, l.ld_y, l.ld_y, p.a_rows, p.kbs) || !map_k(&maps.b, &p.b_3d, a.W, a.V, a.d, a.d, pair ? p.bn / 2 : p.bn, p.kbs))
                return EE_ERR_CUDA;
            p.G = G; p.ld_g = ld_g;
            p.label_rest = reinterpret_cast<float*>(ws + s.label_rest);
            p.m_tiles = tiles(a.M, BM); p.n_tiles = tiles(nv_pad, p.bn); p.k_blocks = tiles(a.d, BK);
            p.seg_blocks = logit_segment(p.k_blocks);
            p.n_cols = nv; p.m_rows = a.M;
            const ee_status st = launch_product<kGrad>(maps, p, pair, a);
            if (st != EE_OK) return st;
        }
        if (need_dy) {
            CeParams q = p;
            q.bn = c.bn;
            q.kbs = blocks_per_slot(kDy, pair, q.bn, q.a_rows);
            if (!map_k(&maps.a, &q.a_3d, G, a.M, nv_pad, ld_g, q.a_rows, q.kbs) || !map_mn(&maps.b, &q.b_3d, a.W, a.V, a.d, a.d, pair ? q.bn / 2 : q.bn, q.kbs))
                return EE_ERR_CUDA;
            q.dy = dy;
            q.m_tiles = tiles(a.M, BM); q.n_tiles = tiles(a.d, q.bn); q.k_blocks = q.seg_blocks = tiles(nv, BK);
            q.splits = c.splits;
            q.n_cols = a.d; q.m_rows = a.M;
            q.add = i > 0;
            const ee_status st = launch_product<kDy>(maps, q, pair, a);
            if (st != EE_OK) return st;
        }
        if (a.dW) {
            CeParams q = p;
            const bool pair_w = use_pairs(nv, a.device);
            q.bn = c.bn;
            q.a_rows = BM;
            q.kbs = blocks_per_slot(kDw, pair_w, q.bn, BM);
            if (!map_mn(&maps.a, &q.a_3d, G, a.M, nv_pad, ld_g, BM, q.kbs) ||
                !map_mn(&maps.b, &q.b_3d, l.y, a.M, l.ld_y, l.ld_y, pair_w ? q.bn / 2 : q.bn, q.kbs))
                return EE_ERR_CUDA;
            q.sectors = a.d % 16 == 0 && reinterpret_cast<uintptr_t>(a.dW) % 32 == 0;
            q.m_tiles = tiles(nv, BM); q.n_tiles = tiles(a.d, q.bn); q.k_blocks = q.seg_blocks = tiles(a.M, BK);
            q.n_cols = a.d; q.m_rows = nv;
            q.add = a.accumulate;
            const ee_status st = launch_product<kDw>(maps, q, pair_w, a);
            if (st != EE_OK) return st;
        }
    }
    if (!need_dy) return EE_OK;
    CeBackArgs b;
    b.h = l.h; b.ld_h = a.ld_h; b.gamma = a.gamma; b.stats = l.stats;
    b.dy = dy; b.splits = c.splits;
    b.labels = a.labels; b.label_rest = reinterpret_cast<const float*>(ws + s.label_rest);
    b.W = static_cast<const __nv_bfloat16*>(a.W); b.V = a.V;
    b.dce = a.dce; b.dloss = a.dloss; b.loss = a.loss;
    b.dh = static_cast<__nv_bfloat16*>(a.dh); b.ld_dh = a.ld_dh;
    b.M = a.M; b.d = a.d;
    b.cols = a.dgamma ? reinterpret_cast<float*>(ws + s.cols) : nullptr;
    b.warps = c.back_warps; b.groups = c.back_groups; b.strip = c.back_strip;
    if (launch_pdl(back_rows(a.d) == 4 ? ce_back_kernel<4, 640> : ce_back_kernel<1, 1024>, dim3(c.back_ctas), 32 * c.back_warps * c.back_groups, 0,
                   a.stream, b) != cudaSuccess)
        return EE_ERR_CUDA;
    if (a.dgamma &&
        launch_pdl(ce_colsum_kernel, dim3(tiles(2 * a.d, 32)), 1024, 0, a.stream, (const float*)b.cols, c.back_ctas * c.back_groups, a.d, a.dce,
                   a.dloss, a.loss, a.accumulate, static_cast<__nv_bfloat16*>(a.dgamma), static_cast<__nv_bfloat16*>(a.dbeta)) != cudaSuccess)
        return EE_ERR_CUDA;
    return EE_OK;
}

}  // namespace ee
