// Cross-entropy of a head over the whole vocabulary and its gradient (the supervised objective of paper section 3.3,
// "Losses", as a training step needs it), without keeping the M x V logits.
//
//   y = bf16(LN(h)),  z = y W^T,  lse_i = ln sum_v e^{z_iv},  ce_i = lse_i - z_i,label_i
//   G_iv = w_i (e^{z_iv - lse_i} - [v = label_i]),  dy = G W,  dW = G^T y,  and dy through the LayerNorm:
//   t = dy gamma,  dh = rstd (t - mean t - xhat mean(t xhat)),  dgamma = sum_i dy xhat,  dbeta = sum_i dy
//
// Four matrix products of 2 M V d operations each (the logits twice: they are recomputed in the backward pass), all by
// one persistent TMA + tcgen05 kernel whose mode decides which operand runs which way and what its epilogue does:
//   kStats  A = y, B = W (both K-major): per row and 64-column group of the tile the running maximum and sum, and
//           the logit at the label; nothing else leaves the chip
//   kGrad   the same product for a piece of the vocabulary; the epilogue turns it into G, rounded to bf16
//   kDy     A = G, B = W with the contraction over the vocabulary: W is read as it lies, as an MN-major operand; fp32
//           results are stored (first piece) or added (later ones, one launch after the other, so in a fixed order)
//           into one slab per split of the contraction
//   kDw     A = G, B = y with the contraction over the rows: both MN-major as they lie
// The pieces keep G at kGradPieceBytes at most, which the L2 holds in part; all of it is one piece for small batches.
// G is rounded to bf16 because the tensor cores take dW and dy from it: each of its elements is off by at most 2^-9
// of itself, independently, which leaves dy and dW off by about as much as their own rounding to bf16.  G is held
// without the mean's 1 / n, which is applied to the fp32 results.  Rows whose label is outside [0, V) take no part: their
// row of G and of y is zero, whatever their hidden state holds.
#include "common.cuh"
#include "layer_norm.cuh"
#include "kernels.h"
#include "sm100_ptx.cuh"
#include "gemm_roles.cuh"
#include "tensor_map.h"

namespace ee {

namespace {

constexpr int BM = 128;
constexpr int BK = kRoleBK;
constexpr int BN = 256;
constexpr int kThreads = 320;                   // producer warp, MMA warp, eight epilogue warps
constexpr int kATileBytes = BM * BK * 2;
constexpr int kBarBytes = 512;
constexpr int kStageWarpBytes = 4096;           // an epilogue warp's 32 rows x 128 bytes on their way to memory
constexpr size_t kSmemBudget = 226 * 1024;
constexpr int kMaxStages = 12;
constexpr int kAccStride = 256;
constexpr int kTmemCols = 512;
constexpr int kMaxSplits = 32;
constexpr size_t kGradPieceBytes = (size_t)128 << 20;

enum CeMode { kStats, kGrad, kDy, kDw };
template <int kMode> struct Layout {
    static constexpr bool a_mn = kMode == kDw;
    static constexpr bool b_mn = kMode == kDy || kMode == kDw;
};

struct CeMaps {
    CUtensorMap a, b, out;
};

struct CeParams {
    int M, d;              // token rows, width
    int m_tiles;           // 128-row tiles of the output (tokens, or vocabulary rows of dW)
    int n_tiles;           // 256-column tiles of the output
    int splits;            // kDy: parts of the contraction, each with a slab of its own
    int k_blocks;          // contraction in blocks of 64
    int n_cols;            // columns of the output that exist (vocabulary of the piece, or d)
    int m_rows;            // rows of the output that exist
    int v0;                // first vocabulary row of the piece
    int n_stages;
    int a_3d, b_3d;        // an MN-major operand's 64-wide blocks come with one request
    int add;               // kDy: add into the slab; kDw: add to what dW holds
    float2* parts;         // kStats: [4 * n_tiles][M] maximum and sum
    float* z_label;        // kStats: [M]
    const int* labels;
    const float* lse;      // kGrad
    const float* dce;      // row weights, or NULL: every counted row 1, and `scale` at the end
    const float* dloss;    // fp32 [1] or NULL (one)
    const float* loss;     // loss[1] = number of counted rows
    __nv_bfloat16* dW;
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

// An operand tile of `rows` elements of its M or N dimension from mn0 on, 64 of the contraction from k0 on.
template <bool kMn, bool kPair>
__device__ __forceinline__ void load_operand(uint32_t dst, const CUtensorMap* m, int k0, int mn0, int rows, int three_d, uint32_t bar) {
    if (!kMn) {
        if (kPair) ptx::tma_load_2d_pair(dst, m, k0, mn0, bar);
        else ptx::tma_load_2d(dst, m, k0, mn0, bar);
    } else if (three_d) {
        if (kPair) ptx::tma_load_3d_pair(dst, m, 0, k0, mn0 >> 6, bar);
        else ptx::tma_load_3d(dst, m, 0, k0, mn0 >> 6, bar);
    } else {
        for (int c = 0; c < rows; c += 64) {
            if (kPair) ptx::tma_load_2d_pair(dst + c * 128, m, mn0 + c, k0, bar);
            else ptx::tma_load_2d(dst + c * 128, m, mn0 + c, k0, bar);
        }
    }
}

template <int kMode, bool kPair>
__global__ void __launch_bounds__(kThreads, 1) ce_gemm_kernel(const __grid_constant__ CeMaps maps, const CeParams p) {
    constexpr bool a_mn = Layout<kMode>::a_mn, b_mn = Layout<kMode>::b_mn;
    constexpr int b_rows = kPair ? BN / 2 : BN;
    constexpr int b_tile_bytes = b_rows * BK * 2;
    const int S = p.n_stages;
    const uint32_t rank = kPair ? ptx::cluster_cta_rank() : 0u;
    const int worker = kPair ? (int)(blockIdx.x >> 1) : (int)blockIdx.x;
    const int n_workers = kPair ? (int)(gridDim.x >> 1) : (int)gridDim.x;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw_addr = ptx::smem_addr(smem_raw);
    unsigned char* smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
    const uint32_t a_base = ptx::smem_addr(smem);
    const uint32_t b_base = a_base + S * kATileBytes;
    unsigned char* staging = smem + S * (kATileBytes + b_tile_bytes);
    unsigned char* bar_mem = staging + (kMode == kStats ? 0 : 8 * kStageWarpBytes);
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
            ptx::mbar_init(tempty_bar(b), kPair ? 16 : 8);
        }
        ptx::mbar_init(drain_bar, 1);
        *abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&maps.a);
        ptx::prefetch_tensormap(&maps.b);
        if (kMode != kStats) ptx::prefetch_tensormap(&maps.out);
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
        split = tile / mn_tiles;
        tile_coords(tile - split * mn_tiles, m_units, p.n_tiles, m_tile, n_tile);
        if (kPair) m_tile = 2 * m_tile + (int)rank;
        kb0 = (int)((long long)split * p.k_blocks / p.splits);
        kb1 = (int)((long long)(split + 1) * p.k_blocks / p.splits);
    };
    auto load_full_bar = [&](int s) { return kPair ? ptx::map_to_cta(full_bar(s), 0) : full_bar(s); };
    constexpr uint32_t arm_bytes = (uint32_t)(kATileBytes + b_tile_bytes) * (kPair ? 2u : 1u);
    // where the piece of the vocabulary lies in W: rows of B for the logits, the contraction for dy
    const int b_mn_off = (kMode == kStats || kMode == kGrad) ? p.v0 : 0;
    const int b_k_off = kMode == kDy ? p.v0 : 0;

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, armed = 0, armed_parity = 0;
            bool ok = true;
            grid_dependency_wait();
            for (int tile = worker; ok && tile < total_tiles; tile += n_workers) {
                int m_tile, n_tile, split, kb0, kb1;
                locate(tile, m_tile, n_tile, split, kb0, kb1);
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!ptx::mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) {
                        record_failure(p.ctrl, abort_flag, 1, stage, tile);
                        ok = false;
                        break;
                    }
                    if (rank == 0) ptx::mbar_arrive_expect_tx(full_bar(stage), arm_bytes);
                    load_operand<a_mn, kPair>(a_base + stage * kATileBytes, &maps.a, kb * BK, m_tile * BM, BM, p.a_3d, load_full_bar(stage));
                    load_operand<b_mn, kPair>(b_base + stage * b_tile_bytes, &maps.b, b_k_off + kb * BK,
                                              b_mn_off + n_tile * BN + (int)rank * b_rows, b_rows, p.b_3d, load_full_bar(stage));
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
            const uint32_t idesc = ptx::idesc_bf16_f32(kPair ? 2 * BM : BM, BN) | (a_mn ? ptx::kIdescAMnMajor : 0u) |
                                   (b_mn ? ptx::kIdescBMnMajor : 0u);
            constexpr uint32_t a_step = a_mn ? 2048 >> 4 : 32 >> 4, b_step = b_mn ? 2048 >> 4 : 32 >> 4;   // per K = 16
            int stage = 0;
            uint32_t phase = 0;
            int local = 0;
            bool ok = true;
            for (int tile = worker; ok && tile < total_tiles; tile += n_workers) {
                int m_tile, n_tile, split, kb0, kb1;
                locate(tile, m_tile, n_tile, split, kb0, kb1);
                if (kb0 == kb1) continue;
                const int buf = local & 1;
                const uint32_t acc_phase = (uint32_t)(local >> 1) & 1u;
                ++local;
                if (!ptx::mbar_wait(tempty_bar(buf), acc_phase ^ 1u, abort_flag)) {
                    record_failure(p.ctrl, abort_flag, 2, 0x80 | buf, tile);
                    break;
                }
                ptx::tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + (uint32_t)(buf * kAccStride);
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!ptx::mbar_wait(full_bar(stage), phase, abort_flag)) {
                        record_failure(p.ctrl, abort_flag, 2, stage, tile);
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after_sync();
                    const uint32_t a_addr = a_base + stage * kATileBytes, b_addr = b_base + stage * b_tile_bytes;
                    const uint64_t adesc = a_mn ? ptx::smem_desc_mn128(a_addr) : ptx::smem_desc_k128(a_addr);
                    const uint64_t bdesc = b_mn ? ptx::smem_desc_mn128(b_addr) : ptx::smem_desc_k128(b_addr);
#pragma unroll
                    for (int k = 0; k < BK / 16; ++k) {
                        const uint32_t accumulate = (kb == kb0 && k == 0) ? 0u : 1u;
                        if (kPair) ptx::mma_bf16_ss_pair(d_tmem, adesc + a_step * k, bdesc + b_step * k, idesc, accumulate);
                        else ptx::mma_bf16_ss(d_tmem, adesc + a_step * k, bdesc + b_step * k, idesc, accumulate);
                    }
                    mma_commit_all<kPair>(empty_bar(stage));
                    if (++stage == S) { stage = 0; phase ^= 1u; }
                }
                if (ok) mma_commit_all<kPair>(tfull_bar(buf));
            }
            if (*abort_flag) mma_drain<kPair>(drain_bar);
        }
    } else {
        // ------------------------------------------------------------------ epilogue (warps 2..9)
        const int quarter = warp & 3;
        const int half = (warp - 2) >> 2;                   // even / odd groups of 64 columns
        unsigned char* mine = staging + (warp - 2) * kStageWarpBytes;
        const uint32_t mine_addr = ptx::smem_addr(mine);
        int local = 0;
        grid_dependency_wait();
        const float scale = kMode == kDw ? grad_scale(p.dce, p.dloss, p.loss) : 1.f;
        for (int tile = worker; tile < total_tiles; tile += n_workers) {
            int m_tile, n_tile, split, kb0, kb1;
            locate(tile, m_tile, n_tile, split, kb0, kb1);
            if (kb0 == kb1) continue;
            const int buf = local & 1;
            const uint32_t acc_phase = (uint32_t)(local >> 1) & 1u;
            ++local;
            const int row0 = m_tile * BM + quarter * 32, row = row0 + lane;
            const bool live = row < p.m_rows;
            float weight = 0.f, lse = 0.f;
            int label = -1;
            if ((kMode == kStats || kMode == kGrad) && live) {
                label = p.labels ? ld_dep(p.labels + row) - p.v0 : -1;
                if (kMode == kGrad) {
                    weight = row_weight(p.labels, p.dce, p.V, row);
                    lse = ld_dep(p.lse + row);
                }
            }
            if (!__all_sync(0xffffffffu, ptx::mbar_wait(tfull_bar(buf), acc_phase, abort_flag))) {
                if (lane == 0) record_failure(p.ctrl, abort_flag, 3, buf, tile);
                break;
            }
            ptx::tc_fence_after_sync();
            const int n0 = n_tile * BN;
            const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * kAccStride);
            if (row0 < p.m_rows) {
                for (int g = half; g < BN / 64; g += 2) {
                    const int col0 = n0 + g * 64;
                    if (col0 >= p.n_cols) break;
                    if (kMode == kStats) {
                        float m = -CUDART_INF_F, s = 0.f;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float z[32];
                            ptx::tmem_ld_32x32(taddr + g * 64 + c * 32, z);
                            ptx::tmem_ld_wait();
                            const int base = col0 + c * 32;
                            const int nvalid = min(p.n_cols - base, 32);
                            if (nvalid <= 0) break;
                            float cm = z[0];
#pragma unroll
                            for (int j = 1; j < 32; ++j)
                                if (j < nvalid) cm = fmaxf(cm, z[j]);
                            if (cm > m) {
                                s *= ex2((m - cm) * kLog2e);              // an empty state: 0 times 0
                                m = cm;
                            }
                            float add = 0.f;
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (j < nvalid) add += ex2((z[j] - m) * kLog2e);
                            s += add;
                            if ((unsigned)(label - base) < (unsigned)nvalid) {
                                float zl = 0.f;
#pragma unroll
                                for (int j = 0; j < 32; ++j) zl = (base + j == label) ? z[j] : zl;
                                p.z_label[row] = zl;
                            }
                        }
                        if (live) p.parts[(size_t)(n_tile * 4 + g) * p.M + row] = make_float2(m, s);
                    } else {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float z[32];
                            ptx::tmem_ld_32x32(taddr + g * 64 + c * 32, z);
                            ptx::tmem_ld_wait();
                            const int base = col0 + c * 32;
                            if (kMode == kGrad) {
#pragma unroll
                                for (int j = 0; j < 32; ++j) {
                                    const float pr = ex2((z[j] - lse) * kLog2e);
                                    const float gr = weight * ((base + j == label) ? pr - 1.f : pr);
                                    z[j] = (weight == 0.f || base + j >= p.n_cols) ? 0.f : gr;
                                }
                            }
                            if (kMode == kDw) {
#pragma unroll
                                for (int j = 0; j < 32; ++j) z[j] *= scale;
                                if (p.add && live) {
                                    const uint4* old = reinterpret_cast<const uint4*>(p.dW + (size_t)(p.v0 + row) * p.d + base);
#pragma unroll
                                    for (int q = 0; q < 4; ++q) {
                                        if (base + q * 8 < p.n_cols) {
                                            const uint4 o = ld_dep(old + q);
                                            z[q * 8 + 0] += bf16_lo(o.x); z[q * 8 + 1] += bf16_hi(o.x);
                                            z[q * 8 + 2] += bf16_lo(o.y); z[q * 8 + 3] += bf16_hi(o.y);
                                            z[q * 8 + 4] += bf16_lo(o.z); z[q * 8 + 5] += bf16_hi(o.z);
                                            z[q * 8 + 6] += bf16_lo(o.w); z[q * 8 + 7] += bf16_hi(o.w);
                                        }
                                    }
                                }
                            }
                            if (kMode == kDy || c == 0) {                 // the warp's staging area is free again
                                if (lane == 0) ptx::bulk_wait_read();
                                __syncwarp();
                            }
                            // 128-byte rows in the swizzle the tensor map names: 16-byte piece q of row r lies at q ^ (r & 7)
                            if (kMode == kDy) {
#pragma unroll
                                for (int q = 0; q < 8; ++q)
                                    *reinterpret_cast<float4*>(mine + lane * 128 + ((q ^ (lane & 7)) << 4)) =
                                        make_float4(z[q * 4], z[q * 4 + 1], z[q * 4 + 2], z[q * 4 + 3]);
                            } else {
#pragma unroll
                                for (int q = 0; q < 4; ++q)
                                    *reinterpret_cast<uint4*>(mine + lane * 128 + (((c * 4 + q) ^ (lane & 7)) << 4)) =
                                        make_uint4(pack_bf16(z[q * 8], z[q * 8 + 1]), pack_bf16(z[q * 8 + 2], z[q * 8 + 3]),
                                                   pack_bf16(z[q * 8 + 4], z[q * 8 + 5]), pack_bf16(z[q * 8 + 6], z[q * 8 + 7]));
                            }
                            if (kMode == kDy || c == 1) {
                                ptx::fence_proxy_async();
                                __syncwarp();
                                if (lane == 0) {
                                    if (kMode == kDy) {
                                        if (base < p.n_cols) {
                                            if (p.add) ptx::tma_add_3d(&maps.out, mine_addr, base, row0, split);
                                            else ptx::tma_store_3d(&maps.out, mine_addr, base, row0, split);
                                        }
                                    } else {
                                        ptx::tma_store_2d(&maps.out, mine_addr, col0, (kMode == kDw ? p.v0 : 0) + row0);
                                    }
                                    ptx::bulk_commit();
                                }
                            }
                        }
                    }
                }
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (kPair) ptx::mbar_arrive_remote(ptx::map_to_cta(tempty_bar(buf), 0));
                else ptx::mbar_arrive(tempty_bar(buf));
            }
        }
        if (kMode != kStats && lane == 0) ptx::bulk_wait_all();
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

// LayerNorm of the rows into y, a warp per row.  In the backward pass (`stats` given) it also leaves each row's mean
// and 1/sigma for the way back, and a row that takes no part in the gradient becomes zeros with 1/sigma = 0.
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
    float2* stats;
    int M, d;
};

__global__ void __launch_bounds__(256) ce_layer_norm_kernel(const __grid_constant__ CeLnArgs a) {
    launch_dependents();
    const int row = blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= a.M) return;
    const int nvec = a.d >> 3;
    uint4* yrow = reinterpret_cast<uint4*>(a.y + (size_t)row * a.d);
    grid_dependency_wait();
    if (a.stats && row_weight(a.labels, a.dce, a.V, row) == 0.f) {
        for (int c = lane; c < nvec; c += 32) yrow[c] = make_uint4(0, 0, 0, 0);
        if (lane == 0) a.stats[row] = make_float2(0.f, 0.f);
        return;
    }
    const uint4* hrow = reinterpret_cast<const uint4*>(a.h + (size_t)row * a.ld_h);
    const RowStats st = row_stats_strided([&](int c) { return ld_dep(hrow + c); }, nvec, a.ln_eps, lane);
    for (int c = lane; c < nvec; c += 32) yrow[c] = layer_norm_vec8(ld_dep(hrow + c), st, a.gamma, a.beta, c);
    if (a.stats && lane == 0) a.stats[row] = make_float2(st.mu_f, st.rstd_f);
}

// Sum of v over the 256 threads of a CTA, in a fixed order.
__device__ __forceinline__ double cta_sum_d(double v, double* part) {
    part[threadIdx.x] = v;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
        if ((int)threadIdx.x < o) part[threadIdx.x] += part[threadIdx.x + o];
        __syncthreads();
    }
    const double r = part[0];
    __syncthreads();
    return r;
}

// 32 rows per CTA, lane = row, the warps stride over the column groups; then the CTA that finishes last adds up the
// mean over the counted rows, in a fixed order whichever CTA that is.
__global__ void __launch_bounds__(256) ce_merge_kernel(const float2* parts, int n_parts, const float* z_label, const int* labels, int M,
                                                       int V, float* ce, float* lse, float* loss, Control* ctrl) {
    __shared__ float2 part[8][32];
    __shared__ double sums[256];
    __shared__ int is_last;
    launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.x * 32 + lane;
    grid_dependency_wait();
    float m = -CUDART_INF_F, s = 0.f;
    auto fold = [&](float2 o) {
        const float nm = fmaxf(m, o.x);
        s = (s == 0.f ? 0.f : s * ex2((m - nm) * kLog2e)) + (o.y == 0.f ? 0.f : o.y * ex2((o.x - nm) * kLog2e));
        m = nm;
    };
    if (row < M)
        for (int n = warp; n < n_parts; n += 8) fold(__ldcg(parts + (size_t)n * M + row));
    part[warp][lane] = make_float2(m, s);
    __syncthreads();
    if (warp == 0 && row < M) {
#pragma unroll
        for (int w = 1; w < 8; ++w) fold(part[w][lane]);
        const float l = m + logf(s);
        lse[row] = l;
        const bool counted = (unsigned)ld_dep(labels + row) < (unsigned)V;
        ce[row] = counted ? l - ld_dep(z_label + row) : 0.f;
    }
    __syncthreads();
    if (threadIdx.x == 0) is_last = ticket_arrive_is_last(&ctrl->head_ticket[0], gridDim.x) ? 1 : 0;
    __syncthreads();
    if (!is_last) return;
    double total = 0.0, n = 0.0;
    for (int i = threadIdx.x; i < M; i += 256)
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

// dy (the sum of its slabs) back through the LayerNorm, a warp per row; the summed dy is left in the first slab.
struct CeBackArgs {
    const __nv_bfloat16* h;
    long long ld_h;
    const float* gamma;
    const float2* stats;
    float* dy;             // [splits][M][d]
    int splits;
    const float* dce;
    const float* dloss;
    const float* loss;
    __nv_bfloat16* dh;     // or NULL
    long long ld_dh;
    int M, d;
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

__global__ void __launch_bounds__(256) ce_dh_kernel(const __grid_constant__ CeBackArgs a) {
    launch_dependents();
    const int row = blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    grid_dependency_wait();
    if (row >= a.M) return;
    const int nvec = a.d >> 3;
    const float2 st = __ldcg(a.stats + row);
    float* dyrow = a.dy + (size_t)row * a.d;
    const uint4* hrow = reinterpret_cast<const uint4*>(a.h + (size_t)row * a.ld_h);
    const bool dead = st.y == 0.f;                                       // takes no part
    float sum = 0.f, dot = 0.f;
    for (int c = lane; c < nvec; c += 32) {
        float v[8] = {};
        for (int k = 0; k < a.splits; ++k) add8(v, dyrow + (size_t)k * a.M * a.d + c * 8);
        if (a.splits > 1) {
            reinterpret_cast<float4*>(dyrow + c * 8)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(dyrow + c * 8)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
        if (!a.dh || dead) continue;
        float x[8];
        unpack8(ld_dep(hrow + c), x);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = v[j] * __ldg(a.gamma + c * 8 + j);
            sum += t;
            dot = fmaf(t, (x[j] - st.x) * st.y, dot);
        }
    }
    if (!a.dh) return;
    uint4* out = reinterpret_cast<uint4*>(a.dh + (size_t)row * a.ld_dh);
    if (dead) {
        for (int c = lane; c < nvec; c += 32) out[c] = make_uint4(0, 0, 0, 0);
        return;
    }
    const float inv_d = 1.f / (float)a.d;
    const float c1 = warp_sum(sum) * inv_d, c2 = warp_sum(dot) * inv_d;
    const float scale = grad_scale(a.dce, a.dloss, a.loss) * st.y;
    for (int c = lane; c < nvec; c += 32) {
        float v[8] = {}, x[8];
        add8(v, dyrow + c * 8);                                          // this lane's own store when there were several slabs
        unpack8(ld_dep(hrow + c), x);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = scale * (v[j] * __ldg(a.gamma + c * 8 + j) - c1 - (x[j] - st.x) * st.y * c2);
        out[c] = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
}

// Column sums of dy xhat and of dy over a strip of rows: 64 columns per CTA, two per thread, eight rows at a time.
constexpr int kStripRows = 128;
__global__ void __launch_bounds__(256) ce_colsum_kernel(const float* dy, const __nv_bfloat16* h, long long ld_h, const float2* stats,
                                                        int M, int d, float* part) {
    __shared__ float4 red[256];
    launch_dependents();
    const int col = blockIdx.x * 64 + (threadIdx.x & 31) * 2, group = threadIdx.x >> 5;
    const int r0 = blockIdx.y * kStripRows, r1 = min(M, r0 + kStripRows);
    grid_dependency_wait();
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);                        // dgamma of two columns, dbeta of two columns
    if (col < d) {
        for (int r = r0 + group; r < r1; r += 8) {
            const float2 st = __ldcg(stats + r);
            if (st.y == 0.f) continue;
            const float2 g = __ldcg(reinterpret_cast<const float2*>(dy + (size_t)r * d + col));
            const uint32_t x = ld_dep(reinterpret_cast<const uint32_t*>(h + (size_t)r * ld_h + col));
            acc.x = fmaf(g.x, (bf16_lo(x) - st.x) * st.y, acc.x);
            acc.y = fmaf(g.y, (bf16_hi(x) - st.x) * st.y, acc.y);
            acc.z += g.x;
            acc.w += g.y;
        }
    }
    red[threadIdx.x] = acc;
    __syncthreads();
    if (group == 0 && col < d) {
        for (int k = 1; k < 8; ++k) {
            const float4 o = red[threadIdx.x + 32 * k];
            acc.x += o.x; acc.y += o.y; acc.z += o.z; acc.w += o.w;
        }
        float* mine = part + (size_t)blockIdx.y * 2 * d;
        *reinterpret_cast<float2*>(mine + col) = make_float2(acc.x, acc.y);
        *reinterpret_cast<float2*>(mine + d + col) = make_float2(acc.z, acc.w);
    }
}

__global__ void __launch_bounds__(256) ce_colsum_final_kernel(const float* part, int strips, int d, const float* dce, const float* dloss,
                                                              const float* loss, int add, __nv_bfloat16* dgamma, __nv_bfloat16* dbeta) {
    launch_dependents();
    const int i = blockIdx.x * 256 + threadIdx.x;
    grid_dependency_wait();
    if (i >= 2 * d) return;
    float s = 0.f;
    for (int k = 0; k < strips; ++k) s += ld_dep(part + (size_t)k * 2 * d + i);
    __nv_bfloat16* out = i < d ? dgamma + i : dbeta + (i - d);
    s *= grad_scale(dce, dloss, loss);
    if (add) s += __bfloat162float(*out);
    *out = __float2bfloat16_rn(s);
}

// ---------------------------------------------------------------------------------------------------- host

bool make_map(CUtensorMap* map, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides,
              const cuuint32_t* box, CUtensorMapL2promotion promo = CU_TENSOR_MAP_L2_PROMOTION_L2_128B) {
    EncodeTiledFn fn = encode_tiled_fn();
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn && fn(map, type, rank, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, promo, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// bf16 [rows, cols] with row stride ld, boxes of box_rows x 64 columns.
bool map_2d(CUtensorMap* map, const void* base, int rows, int cols, int ld, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {64u, (cuuint32_t)box_rows};
    return make_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box);
}
// An MN-major operand: bf16 [rows (contraction), cols] with row stride ld, read as blocks of 64 x 64; `blocks` of them with
// one request where the columns are whole blocks.
bool map_mn(CUtensorMap* map, int* three_d, const void* base, int rows, int cols, int ld, int blocks) {
    *three_d = cols % 64 == 0;
    if (!*three_d) return map_2d(map, base, rows, cols, ld, 64);
    const cuuint64_t dims[3] = {64u, (cuuint64_t)rows, (cuuint64_t)(cols / 64)}, strides[2] = {(cuuint64_t)ld * 2, 128u};
    const cuuint32_t box[3] = {64u, 64u, (cuuint32_t)blocks};
    return make_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, base, dims, strides, box);
}

int tiles(int n, int t) { return (n + t - 1) / t; }

// Piece of the vocabulary and splits of dy's contraction for a batch (fixed by the sizes alone: the workspace is sized
// with them).
struct CePlan {
    int piece, n_pieces, splits, strips;
};
CePlan ce_plan(int M, int d, int V) {
    CePlan c;
    long long most = (long long)(kGradPieceBytes / 2) / (M > 0 ? M : 1) / BN * BN;
    if (most < BN) most = BN;
    if (most > V) most = (V + BN - 1LL) / BN * BN;
    c.n_pieces = (int)((V + most - 1) / most);
    c.piece = (int)((((long long)V + c.n_pieces - 1) / c.n_pieces + BN - 1) / BN * BN);
    c.n_pieces = tiles(V, c.piece);
    // as many splits as make the workers' rounds shortest; a split costs its slab's way to memory and back
    const bool pair = M > BM;
    const long long workers = pair ? 74 : 148, t = (long long)(pair ? tiles(M, 2 * BM) : 1) * tiles(d, BN);
    const int k_blocks = tiles(c.piece < V ? c.piece : V, BK);
    double best = 0;
    c.splits = 1;
    for (int s = 1; s <= kMaxSplits && s * 4 <= k_blocks; ++s) {
        const double cost = (double)((t * s + workers - 1) / workers) / s + 0.004 * s;
        if (s == 1 || cost < best) {
            best = cost;
            c.splits = s;
        }
    }
    c.strips = tiles(M, kStripRows);
    return c;
}

struct CeSpace {
    size_t y, stats, parts, z_label, g, dy, cols, total;
};
CeSpace ce_space(int M, int d, int V, bool grad) {
    CeSpace s;
    size_t at = kCtrlBytes;
    auto take = [&](size_t n) { const size_t o = at; at = align_up(at + n, 256); return o; };
    s.y = take((size_t)M * d * 2);
    s.stats = take((size_t)M * 8);
    s.parts = take((size_t)4 * tiles(V, BN) * M * 8);
    s.z_label = take((size_t)M * 4);
    s.g = s.dy = s.cols = at;
    if (grad) {
        const CePlan c = ce_plan(M, d, V);
        s.g = take((size_t)M * c.piece * 2);
        s.dy = take((size_t)c.splits * M * d * 4);
        s.cols = take((size_t)c.strips * 2 * d * 4);
    }
    s.total = at;
    return s;
}

template <int kMode, bool kPair>
constexpr int ring_stages() {
    const size_t stage = kATileBytes + (size_t)(kPair ? BN / 2 : BN) * BK * 2;
    const size_t n = (kSmemBudget - 1024 - kBarBytes - (kMode == kStats ? 0 : 8 * kStageWarpBytes)) / stage;
    return (int)(n < (size_t)kMaxStages ? n : (size_t)kMaxStages);
}
template <int kMode, bool kPair>
constexpr size_t ring_smem() {
    return (size_t)ring_stages<kMode, kPair>() * (kATileBytes + (size_t)(kPair ? BN / 2 : BN) * BK * 2) +
           (kMode == kStats ? 0 : 8 * kStageWarpBytes) + kBarBytes + 1024;
}

// Two-CTA clusters the device runs at once; 0 if the query fails or EE_GEMM_PAIRS=0 switches pairs off.
int resident_pairs(int device) {
    static int pairs[kMaxDevices];
    static bool asked[kMaxDevices] = {};
    if (!asked[device]) {
        int n = 0;
        const char* e = getenv("EE_GEMM_PAIRS");
        if (!(e && e[0] == '0') && cudaFuncSetAttribute(ce_gemm_kernel<kGrad, true>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                        (int)kSmemBudget) == cudaSuccess) {
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute attr[2];
            pair_launch_config(cfg, attr, dim3(2), kThreads, kSmemBudget, nullptr);
            if (cudaOccupancyMaxActiveClusters(&n, ce_gemm_kernel<kGrad, true>, &cfg) != cudaSuccess) {
                n = 0;
                (void)cudaGetLastError();
            }
        }
        pairs[device] = n;
        asked[device] = true;
    }
    return pairs[device];
}

template <int kMode, bool kPair>
ee_status launch_mode(const CeMaps& maps, CeParams p, int workers, int device, cudaStream_t stream) {
    static bool configured[kMaxDevices] = {};
    if (!configured[device]) {
        if (cudaFuncSetAttribute(ce_gemm_kernel<kMode, kPair>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)ring_smem<kMode, kPair>()) != cudaSuccess)
            return EE_ERR_CUDA;
        configured[device] = true;
    }
    p.n_stages = ring_stages<kMode, kPair>();
    const long long total = (long long)(kPair ? (p.m_tiles + 1) / 2 : p.m_tiles) * p.n_tiles * p.splits;
    const int grid = (int)(total < workers ? total : workers);
    const cudaError_t e = kPair ? launch_pdl_pairs(ce_gemm_kernel<kMode, kPair>, 2 * grid, kThreads, ring_smem<kMode, kPair>(), stream, maps, p)
                                : launch_pdl(ce_gemm_kernel<kMode, kPair>, grid, kThreads, ring_smem<kMode, kPair>(), stream, maps, p);
    return e == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

// Pairs of CTAs on 256-row tiles when the output has more than 128 rows and the device can run them.
bool use_pairs(int rows, int device) { return rows > BM && resident_pairs(device) > 0; }
template <int kMode>
ee_status launch_product(const CeMaps& maps, const CeParams& p, bool pair, const CeArgs& a) {
    return pair ? launch_mode<kMode, true>(maps, p, resident_pairs(a.device), a.device, a.stream)
                : launch_mode<kMode, false>(maps, p, a.num_sms, a.device, a.stream);
}

CeLnArgs ln_args(const CeArgs& a, const CeSpace& s, bool grad) {
    unsigned char* ws = static_cast<unsigned char*>(a.workspace);
    CeLnArgs l;
    l.h = static_cast<const __nv_bfloat16*>(a.h);
    l.ld_h = a.ld_h; l.gamma = a.gamma; l.beta = a.beta; l.ln_eps = a.ln_eps;
    l.labels = a.labels; l.dce = a.dce; l.V = a.V;
    l.y = reinterpret_cast<__nv_bfloat16*>(ws + s.y);
    l.stats = grad ? reinterpret_cast<float2*>(ws + s.stats) : nullptr;
    l.M = a.M; l.d = a.d;
    return l;
}

CeParams base_params(const CeArgs& a) {
    CeParams p{};
    p.M = a.M; p.d = a.d; p.V = a.V;
    p.splits = 1;
    p.labels = a.labels; p.lse = a.lse; p.dce = a.dce; p.dloss = a.dloss; p.loss = a.loss;
    p.dW = static_cast<__nv_bfloat16*>(a.dW);
    p.ctrl = reinterpret_cast<Control*>(a.workspace);
    return p;
}

}  // namespace

ee_status layer_norm_launch(const void* h, long long ld_h, const float* gamma, const float* beta, float ln_eps, void* y, int M, int d,
                            cudaStream_t stream) {
    CeLnArgs l{};
    l.h = static_cast<const __nv_bfloat16*>(h);
    l.ld_h = ld_h; l.gamma = gamma; l.beta = beta; l.ln_eps = ln_eps;
    l.y = static_cast<__nv_bfloat16*>(y);
    l.M = M; l.d = d;
    return launch_pdl(ce_layer_norm_kernel, dim3((M + 7) / 8), 256, 0, stream, l) == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

size_t ce_workspace_bytes(int M, int d, int V, bool grad) { return ce_space(M, d, V, grad).total; }

ee_status ce_launch(const CeArgs& a) {
    unsigned char* ws = static_cast<unsigned char*>(a.workspace);
    const CeSpace s = ce_space(a.M, a.d, a.V, false);
    const CeLnArgs l = ln_args(a, s, false);
    if (launch_pdl(ce_layer_norm_kernel, dim3((a.M + 7) / 8), 256, 0, a.stream, l) != cudaSuccess) return EE_ERR_CUDA;
    const bool pair = use_pairs(a.M, a.device);
    CeMaps maps;
    if (!map_2d(&maps.a, l.y, a.M, a.d, a.d, BM) || !map_2d(&maps.b, a.W, a.V, a.d, a.d, pair ? BN / 2 : BN)) return EE_ERR_CUDA;
    maps.out = maps.a;                                                   // not used
    CeParams p = base_params(a);
    p.m_tiles = tiles(a.M, BM);
    p.n_tiles = tiles(a.V, BN);
    p.k_blocks = tiles(a.d, BK);
    p.n_cols = a.V;
    p.m_rows = a.M;
    p.parts = reinterpret_cast<float2*>(ws + s.parts);
    p.z_label = reinterpret_cast<float*>(ws + s.z_label);
    const ee_status st = launch_product<kStats>(maps, p, pair, a);
    if (st != EE_OK) return st;
    // the last tile's groups of 64 columns beyond the vocabulary are not written
    const int n_parts = tiles(a.V, 64);
    if (launch_pdl(ce_merge_kernel, (a.M + 31) / 32, 256, 0, a.stream, (const float2*)p.parts, n_parts, (const float*)p.z_label, a.labels,
                   a.M, a.V, a.ce, a.lse_out, a.loss_out, p.ctrl) != cudaSuccess)
        return EE_ERR_CUDA;
    return EE_OK;
}

ee_status ce_grad_launch(const CeArgs& a) {
    unsigned char* ws = static_cast<unsigned char*>(a.workspace);
    const CeSpace s = ce_space(a.M, a.d, a.V, true);
    const CePlan c = ce_plan(a.M, a.d, a.V);
    const CeLnArgs l = ln_args(a, s, true);
    if (launch_pdl(ce_layer_norm_kernel, dim3((a.M + 7) / 8), 256, 0, a.stream, l) != cudaSuccess) return EE_ERR_CUDA;
    const bool pair = use_pairs(a.M, a.device);
    const bool need_dy = a.dh || a.dgamma;
    const int ld_g = c.piece;
    __nv_bfloat16* G = reinterpret_cast<__nv_bfloat16*>(ws + s.g);
    float* dy = reinterpret_cast<float*>(ws + s.dy);

    for (int i = 0; i < c.n_pieces; ++i) {
        const int v0 = i * c.piece, nv = a.V - v0 < c.piece ? a.V - v0 : c.piece;
        const int nv_pad = (nv + 63) / 64 * 64;                          // the columns of G that are written (zeros beyond nv)
        CeMaps maps;
        CeParams p = base_params(a);
        p.v0 = v0;
        {
            if (!map_2d(&maps.a, l.y, a.M, a.d, a.d, BM) || !map_2d(&maps.b, a.W, a.V, a.d, a.d, pair ? BN / 2 : BN) ||
                !map_2d(&maps.out, G, a.M, nv_pad, ld_g, 32))
                return EE_ERR_CUDA;
            p.m_tiles = tiles(a.M, BM); p.n_tiles = tiles(nv, BN); p.k_blocks = tiles(a.d, BK);
            p.n_cols = nv; p.m_rows = a.M;
            const ee_status st = launch_product<kGrad>(maps, p, pair, a);
            if (st != EE_OK) return st;
        }
        if (need_dy) {
            CeParams q = p;
            const cuuint64_t dims[3] = {(cuuint64_t)a.d, (cuuint64_t)a.M, (cuuint64_t)c.splits};
            const cuuint64_t strides[2] = {(cuuint64_t)a.d * 4, (cuuint64_t)a.M * a.d * 4};
            const cuuint32_t box[3] = {32u, 32u, 1u};
            if (!map_2d(&maps.a, G, a.M, nv_pad, ld_g, BM) || !map_mn(&maps.b, &q.b_3d, a.W, a.V, a.d, a.d, (pair ? BN / 2 : BN) / 64) ||
                !make_map(&maps.out, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, dy, dims, strides, box))
                return EE_ERR_CUDA;
            q.m_tiles = tiles(a.M, BM); q.n_tiles = tiles(a.d, BN); q.k_blocks = tiles(nv, BK);
            q.splits = c.splits;
            q.n_cols = a.d; q.m_rows = a.M;
            q.add = i > 0;
            const ee_status st = launch_product<kDy>(maps, q, pair, a);
            if (st != EE_OK) return st;
        }
        if (a.dW) {
            CeParams q = p;
            const bool pair_w = use_pairs(nv, a.device);
            if (!map_mn(&maps.a, &q.a_3d, G, a.M, nv_pad, ld_g, BM / 64) ||
                !map_mn(&maps.b, &q.b_3d, l.y, a.M, a.d, a.d, (pair_w ? BN / 2 : BN) / 64) || !map_2d(&maps.out, a.dW, a.V, a.d, a.d, 32))
                return EE_ERR_CUDA;
            q.m_tiles = tiles(nv, BM); q.n_tiles = tiles(a.d, BN); q.k_blocks = tiles(a.M, BK);
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
    b.dce = a.dce; b.dloss = a.dloss; b.loss = a.loss;
    b.dh = static_cast<__nv_bfloat16*>(a.dh); b.ld_dh = a.ld_dh;
    b.M = a.M; b.d = a.d;
    if (launch_pdl(ce_dh_kernel, dim3((a.M + 7) / 8), 256, 0, a.stream, b) != cudaSuccess) return EE_ERR_CUDA;
    if (a.dgamma) {
        float* part = reinterpret_cast<float*>(ws + s.cols);
        if (launch_pdl(ce_colsum_kernel, dim3(tiles(a.d, 64), c.strips), 256, 0, a.stream, (const float*)dy, l.h, a.ld_h,
                       (const float2*)l.stats, a.M, a.d, part) != cudaSuccess ||
            launch_pdl(ce_colsum_final_kernel, dim3(tiles(2 * a.d, 256)), 256, 0, a.stream, (const float*)part, c.strips, a.d, a.dce, a.dloss,
                       a.loss, a.accumulate, static_cast<__nv_bfloat16*>(a.dgamma), static_cast<__nv_bfloat16*>(a.dbeta)) != cudaSuccess)
            return EE_ERR_CUDA;
    }
    return EE_OK;
}

}  // namespace ee
