// A head in microscaled 4-bit floating point for many rows.
//
// Persistent CTAs; the activations (128 rows to a tile) are the M operand of the products, the weight tiles of 128 rows the N operand.  The
// tiles of the M x V plane are numbered row tile by row tile and every CTA takes an equal run of them, so that it stays with a row tile and its
// epilogue keeps the rows' softmax states in registers from weight tile to weight tile: a state leaves the chip only where a run or a row tile
// ends, and the weights, which all CTAs walk at the same time, stay in L2.
//   warp 0 (one lane)  producer      warp 1 (one lane)  scale copies and products      warps 2 .. 9  states
// Two warps share a quarter of the accumulator's lanes (thread = row), each half of its columns.
#include "q4_common.cuh"
#include "fp4_common.cuh"
#include "gemm_roles.cuh"
#include "kernels.h"
#include "sm100_fp4.cuh"
#include "sm100_operands.cuh"

namespace ee {

namespace {

constexpr int kThreads = 320;
constexpr int kFoldWarps = 8;
constexpr int kUnits = 2;                        // units per stage and operand
constexpr int kTmemCols = 512;
constexpr int kAccCols = 128;
constexpr int kMaxWorkers = 256;
constexpr int kMergeThreads = 256;
constexpr int kBarBytes = 256;

struct GemmParams {
    Fp4Head q;
    RestState* parts;              // [row][slot][half of the columns]
    int m_tiles, n_tiles, slots;
};

template <int kGroup>
struct Shape {
    static constexpr int kUnit = fp4_unit_bytes(kGroup, kFp4Rows);
    static constexpr int kOperandBytes = kUnits * kUnit;
    static constexpr int kStageBytes = (2 * kOperandBytes + 1023) / 1024 * 1024;
    static constexpr int kScaleCols = kUnits * fp4_scale_bytes(kGroup) / 512 * 8;
    static constexpr int kStages = 6;
    static constexpr size_t kSmem = (size_t)kStages * kStageBytes + kBarBytes + 1024;
    static_assert(2 * kAccCols + kStages * kScaleCols <= kTmemCols && kSmem <= 227 * 1024, "fits");
};

// The run of tiles of worker w of n, and the worker that has tile t.
__host__ __device__ inline long long run_begin(int w, int n, long long total) { return (long long)w * total / n; }
__host__ __device__ inline int worker_of(long long t, int n, long long total) { return (int)(((t + 1) * n - 1) / total); }
// Workers that share a row tile, at most.
int max_slots(int m_tiles, int n_tiles, int workers) {
    const long long total = (long long)m_tiles * n_tiles, each = total / workers > 0 ? total / workers : 1;
    return (int)((n_tiles + each - 1) / each) + 1;
}

// Adds 32 logits' terms, all but those of columns j0 and from nvalid on, to a state whose maximum is at least theirs.  The order of the sums is
// the same in either form, so that a row's result does not depend on which one its warp takes.
template <bool kAll>
__device__ __forceinline__ void add_terms(RestState& st, const float (&v)[32], float c, int j0, int nvalid) {
    const unsigned long long minus_m = ptx::pack_f32x2(-st.m, -st.m), cc = ptx::pack_f32x2(c, c);
    unsigned long long s[2] = {0, 0}, t[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
        const unsigned long long dz = ptx::add_f32x2(ptx::pack_f32x2(v[j], v[j + 1]), minus_m);
        const float2 a = ptx::unpack_f32x2(ptx::mul_f32x2(dz, cc));
        float2 x = make_float2(ex2(a.x), ex2(a.y));
        if (!kAll) {
            if (j == j0 || j >= nvalid) x.x = 0.f;
            if (j + 1 == j0 || j + 1 >= nvalid) x.y = 0.f;
        }
        const unsigned long long e = ptx::pack_f32x2(x.x, x.y);
        s[(j >> 1) & 1] = ptx::add_f32x2(s[(j >> 1) & 1], e);
        t[(j >> 1) & 1] = ptx::fma_f32x2(e, dz, t[(j >> 1) & 1]);
    }
    const float2 ss = ptx::unpack_f32x2(ptx::add_f32x2(s[0], s[1])), tt = ptx::unpack_f32x2(ptx::add_f32x2(t[0], t[1]));
    st.s += ss.x + ss.y;
    st.t += tt.x + tt.y;
}

// 32 consecutive logits of a row, before the power of two they have in common (`c` is that times log2 e), into its state, which is in the same
// units.  A new maximum, which leaves its term out of the sum, is rare: some ten of a row's thousand chunks bring one.
__device__ __forceinline__ void fold_chunk(RestState& st, const float (&v)[32], float c, int col0, int nvalid) {
    float cm[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
    if (nvalid >= 32) {
#pragma unroll
        for (int j = 0; j < 32; j += 2) cm[(j >> 1) & 3] = ptx::max3(cm[(j >> 1) & 3], v[j], v[j + 1]);
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < nvalid) cm[j & 3] = fmaxf(cm[j & 3], v[j]);
    }
    const float top = fmaxf(ptx::max3(cm[0], cm[1], cm[2]), cm[3]);
    if (nvalid >= 32 && !__any_sync(0xffffffffu, top > st.m)) {
        add_terms<true>(st, v, c, 0, 32);
        return;
    }
    int j0 = -1;
    if (top > st.m) {
#pragma unroll
        for (int j = 31; j >= 0; --j)
            if (j < nvalid && v[j] == top) j0 = j;
        const bool none = st.s == -1.f;
        const float dl = st.m - top, al = none ? 0.f : ex2(dl * c), n = 1.f + st.s;
        st.t = none ? 0.f : al * fmaf(dl, n, st.t);
        st.s = none ? 0.f : al * n;
        st.m = top;
        st.idx = col0 + j0;
    }
    add_terms<false>(st, v, c, j0, nvalid);
}

template <int kGroup>
__global__ void __launch_bounds__(kThreads, 1) fp4_gemm_kernel(const GemmParams p) {
    using S = Shape<kGroup>;
    const Fp4Head& q = p.q;
    const int blocks = fp4_blocks(q.d), steps = (blocks + kUnits - 1) / kUnits;
    const long long total = (long long)p.m_tiles * p.n_tiles;
    const long long begin = run_begin(blockIdx.x, gridDim.x, total), end = run_begin(blockIdx.x + 1, gridDim.x, total);
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw_addr = ptx::smem_addr(smem_raw);
    unsigned char* smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
    const uint32_t ring = ptx::smem_addr(smem);
    unsigned char* bar_mem = smem + S::kStages * S::kStageBytes;
    const uint32_t bar_base = ptx::smem_addr(bar_mem);
    auto full_bar = [&](int s) { return bar_base + 8u * s; };
    auto empty_bar = [&](int s) { return bar_base + 8u * (S::kStages + s); };
    auto accfull_bar = [&](int b) { return bar_base + 8u * (2 * S::kStages + b); };
    auto accfree_bar = [&](int b) { return bar_base + 8u * (2 * S::kStages + 2 + b); };
    const uint32_t drain_bar = bar_base + 8u * (2 * S::kStages + 4);
    volatile uint32_t* tmem_holder = reinterpret_cast<volatile uint32_t*>(bar_mem + 8 * (2 * S::kStages + 5));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            ptx::mbar_init(full_bar(s), 1);
            ptx::mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(accfull_bar(b), 1);
            ptx::mbar_init(accfree_bar(b), kFoldWarps);
        }
        ptx::mbar_init(drain_bar, 1);
        *abort_flag = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 1) {
        ptx::tmem_alloc(ptx::smem_addr(const_cast<uint32_t*>(tmem_holder)), kTmemCols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_holder, scales_base = tmem_base + 2 * kAccCols;

    if (warp == 0) {
        // ---------------------------------------------------------------- producer
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, armed = 0, armed_parity = 0;
            bool ok = true;
            grid_dependency_wait();
            for (long long t = begin; ok && t < end; ++t) {
                if (t + 1 == end) launch_dependents();
                const size_t m_tile = (size_t)(t / p.n_tiles), n_tile = (size_t)(t - (long long)m_tile * p.n_tiles);
                for (int step = 0; step < steps; ++step) {
                    if (!ptx::mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) {
                        record_failure(q.ctrl, abort_flag, 1, stage, (unsigned)t);
                        ok = false;
                        break;
                    }
                    const uint32_t bytes = (uint32_t)min(kUnits, blocks - step * kUnits) * S::kUnit, to = ring + stage * S::kStageBytes;
                    ptx::mbar_arrive_expect_tx(full_bar(stage), 2 * bytes);
                    ptx::bulk_load(to, q.acts + (m_tile * blocks + step * kUnits) * S::kUnit, bytes, full_bar(stage));
                    ptx::bulk_load(to + S::kOperandBytes, q.weights + (n_tile * blocks + step * kUnits) * S::kUnit, bytes, full_bar(stage));
                    armed |= 1u << stage;
                    armed_parity = (armed_parity & ~(1u << stage)) | (phase << stage);
                    if (++stage == S::kStages) { stage = 0; phase ^= 1u; }
                }
            }
            if (*abort_flag) producer_drain(0, S::kStages, full_bar(0), armed, armed_parity);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------------- products
        if (lane == 0) {
            constexpr uint32_t idesc = ptx::idesc_fp4<kGroup>(kFp4Rows, kFp4Rows);
            constexpr int kAtoms = fp4_scale_bytes(kGroup) / 512;
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (long long t = begin; ok && t < end; ++t) {
                const int local = (int)(t - begin), buf = local & 1;
                if (!ptx::mbar_wait(accfree_bar(buf), ((uint32_t)(local >> 1) & 1u) ^ 1u, abort_flag)) {
                    record_failure(q.ctrl, abort_flag, 2, 0x80 | buf, (unsigned)t);
                    break;
                }
                ptx::tc_fence_after_sync();
                const uint32_t acc = tmem_base + buf * kAccCols;
                for (int step = 0; step < steps; ++step) {
                    if (!ptx::mbar_wait(full_bar(stage), phase, abort_flag)) {
                        record_failure(q.ctrl, abort_flag, 2, stage, (unsigned)t);
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after_sync();
                    const uint32_t x = ring + stage * S::kStageBytes, w = x + S::kOperandBytes;
                    const uint32_t scales = scales_base + stage * S::kScaleCols;
#pragma unroll
                    for (int u = 0; u < kUnits; ++u) {
                        if (step * kUnits + u < blocks) {
                            const uint32_t xu = x + u * S::kUnit, wu = w + u * S::kUnit, su = scales + u * kAtoms * 8;
#pragma unroll
                            for (int k = 0; k < kAtoms; ++k) {
                                ptx::tmem_cp_scales(su + 8 * k, ptx::smem_desc_scales(xu + 512 * k));
                                ptx::tmem_cp_scales(su + 8 * k + 4, ptx::smem_desc_scales(wu + 512 * k));
                            }
                            const uint64_t a = ptx::smem_desc_k64(xu + fp4_scale_bytes(kGroup)), b = ptx::smem_desc_k64(wu + fp4_scale_bytes(kGroup));
#pragma unroll
                            for (int k = 0; k < 2; ++k) {                // 64 columns are 32 bytes, 2 descriptor units
                                const uint32_t sk = su + (kGroup == 16 ? 8 * k : 0);
                                const uint32_t which = kGroup == 32 && k == 1 ? ptx::kIdescFp4SecondHalf : 0u;
                                ptx::mma_fp4<kGroup>(acc, a + 2u * k, b + 2u * k, idesc | which, sk, sk + 4, step > 0 || u > 0 || k > 0 ? 1u : 0u);
                            }
                        }
                    }
                    ptx::mma_commit(empty_bar(stage));
                    if (++stage == S::kStages) { stage = 0; phase ^= 1u; }
                }
                if (ok) ptx::mma_commit(accfull_bar(buf));
            }
            if (*abort_flag) mma_drain<false>(drain_bar);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- states
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        RestState st = rest_empty();
        grid_dependency_wait();
        const float weight_factor = ld_dep(q.weight_factor);
        float factor = 0.f, c = 0.f;
        int m_before = -1;
        auto flush = [&](int m_tile) {
            const long long row = (long long)m_tile * kFp4Rows + quarter * 32 + lane;
            const int slot = (int)blockIdx.x - worker_of((long long)m_tile * p.n_tiles, gridDim.x, total);
            if (row < q.M) p.parts[(row * p.slots + slot) * 2 + half] = RestState{st.m * factor, st.s, st.t * factor, st.idx};
            st = rest_empty();
        };
        for (long long t = begin; t < end; ++t) {
            const int local = (int)(t - begin), buf = local & 1;
            const int m_tile = (int)(t / p.n_tiles), n_tile = (int)(t - (long long)m_tile * p.n_tiles);
            if (m_tile != m_before) {
                if (m_before >= 0) flush(m_before);
                m_before = m_tile;
                const long long row = (long long)m_tile * kFp4Rows + quarter * 32 + lane;
                factor = row < q.M ? ld_dep(q.factor + row) * weight_factor : 1.f;
                c = factor * kLog2e;
            }
            const bool landed = ptx::mbar_wait(accfull_bar(buf), (uint32_t)(local >> 1) & 1u, abort_flag);
            if (!__all_sync(0xffffffffu, landed)) {
                if (lane == 0) record_failure(q.ctrl, abort_flag, 3, buf, (unsigned)t);
                break;
            }
            ptx::tc_fence_after_sync();
            const uint32_t from = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * kAccCols + half * 64;
            const int col0 = n_tile * kFp4Rows + half * 64;
#pragma unroll 1
            for (int k = 0; k < 2; ++k) {
                float v[32];
                ptx::tmem_ld_32x32(from + 32 * k, v);
                ptx::tmem_ld_wait();
                if (k == 1) {
                    ptx::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(accfree_bar(buf));
                }
                const int nvalid = q.V - (col0 + 32 * k);
                if (nvalid > 0) fold_chunk(st, v, c, col0 + 32 * k, nvalid);
            }
        }
        if (m_before >= 0) flush(m_before);
    }
    if (warp < 2) grid_dependency_wait();
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem_base, kTmemCols);
    }
}

// A warp per row: the states of the workers that shared its tile.
__global__ void __launch_bounds__(kMergeThreads) fp4_merge_kernel(const GemmParams p, int workers) {
    launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * (kMergeThreads / 32) + (threadIdx.x >> 5);
    if (row >= p.q.M) return;
    const long long total = (long long)p.m_tiles * p.n_tiles, first = row / kFp4Rows * p.n_tiles;
    const int n = 2 * (worker_of(first + p.n_tiles - 1, workers, total) - worker_of(first, workers, total) + 1);
    const RestState* parts = p.parts + row * p.slots * 2;
    RestState mine = rest_empty();
    for (int k = lane; k < n; k += 32) rest_merge(mine, rest_load_cg(parts + k));
    const RestState all = rest_reduce_lanes<1>(mine);
    if (lane == 0) rest_finish(all, p.q, (int)row);
}

template <int kGroup>
ee_status launch_group(GemmParams p, int workers, int device, cudaStream_t stream) {
    using S = Shape<kGroup>;
    static bool configured[kMaxDevices] = {};
    if (!configured[device]) {
        if (cudaFuncSetAttribute(fp4_gemm_kernel<kGroup>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem) != cudaSuccess) return EE_ERR_CUDA;
        configured[device] = true;
    }
    if (launch_pdl(fp4_gemm_kernel<kGroup>, dim3(workers), kThreads, S::kSmem, stream, p) != cudaSuccess) return EE_ERR_CUDA;
    const int rows = kMergeThreads / 32;
    return launch_pdl(fp4_merge_kernel, dim3((p.q.M + rows - 1) / rows), kMergeThreads, 0, stream, p, workers) == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

int workers_of(long long total, int num_sms) {
    const int most = num_sms < kMaxWorkers ? num_sms : kMaxWorkers;
    return total < most ? (int)total : most;
}

}  // namespace

size_t fp4_gemm_parts_bytes(int M, int V) {      // for any number of SMs
    const int m_tiles = fp4_tiles(M, kFp4Rows), n_tiles = fp4_tiles(V, kFp4Rows);
    return (size_t)M * max_slots(m_tiles, n_tiles, workers_of((long long)m_tiles * n_tiles, kMaxWorkers)) * 2 * sizeof(RestState);
}

ee_status fp4_gemm_launch(const Fp4Head& q, int group, void* parts, int num_sms, int device, cudaStream_t stream) {
    GemmParams p;
    p.q = q;
    p.parts = static_cast<RestState*>(parts);
    p.m_tiles = fp4_tiles(q.M, kFp4Rows);
    p.n_tiles = fp4_tiles(q.V, kFp4Rows);
    const int workers = workers_of((long long)p.m_tiles * p.n_tiles, num_sms);
    p.slots = max_slots(p.m_tiles, p.n_tiles, workers);
    return group == 16 ? launch_group<16>(p, workers, device, stream) : launch_group<32>(p, workers, device, stream);
}

}  // namespace ee
