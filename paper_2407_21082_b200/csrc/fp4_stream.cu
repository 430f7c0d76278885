// A head in microscaled 4-bit floating point for few rows (up to 64): what counts is the read of the weights.
//
// One persistent CTA per SM takes every so-manieth weight tile of 128 rows.  The weights are the M operand of the products and the
// activations, padded to 8, 16, 32 or 64 rows, the N operand; both arrive by plain bulk copies in the layout that the tensor core reads, so no
// thread touches a weight.  A stage of the ring holds two units (256 columns) of either operand: their scales go to tensor memory by
// tcgen05.cp, into columns of the stage's own, then the four products of 64 columns are issued behind them.
//   warp 0 (one lane)  producer      warp 1 (one lane)  scale copies and products      warps 2 .. 9  logits
// The accumulators (lanes: the tile's rows, columns: the tokens) are double-buffered.  The eight epilogue warps move a tile of logits to
// shared memory, token by token, and then a warp takes every eighth token: a lane four of the tile's rows, folded into states in its registers,
// which it keeps from tile to tile.  The lanes' states are merged once, and the CTAs' by the CTA that finishes last (up to 8 rows, a warp
// for each) or by a kernel of their own.
//
// The weights' first stages are requested before the wait for the kernel that writes the activations: at d = 1024 the ring of all SMs
// together holds most of the head.
//
// V = 50304: 10.4 us for a row of 1024 (29.6 MB packed, 4.5 us at the copy rate), 15.7 for one of 2560, 15.6 for 64 of 1024, 22 for 64 of 2560 (74 MB,
// 3.3 TB/s).  Start, LayerNorm and merge are some 6 us of that.  The issuing threads bound the rest: a single thread takes four to five cycles
// for an instruction (a hundred for one to the tensor core, as long as the compiler keeps its operands out of uniform registers, which it does under
// `lane == 0` but not under elect.sync: one row of 1024 took 13.7 us), and a stage of 21 KB takes it some 500.
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
constexpr int kUnits = 2;                        // units per stage
constexpr int kMaxStages = 12;
// Rows up to which the CTA that finishes last merges the states; more are a kernel of their own.  Device times at V = 50304, merged here / there: 4 rows of
// 512 9.2 / 9.3 us, of 2560 16.5 / 16.7, 8 rows of 1024 11.5 / 11.0, of 2560 17.2 / 16.7, 16 rows of 512 11.8 / 9.7, of 1024 13.8 / 11.6, 64 of 512 24.4 / 14.8.
// Up to 8 rows what the launch saves on the device it costs on the host, 2 us, which eager calls of this size wait for.
constexpr int kMergeHere = 8;
constexpr int kMergeThreads = 128;
constexpr int kTmemCols = 512;
constexpr size_t kSmemBudget = 226 * 1024;
constexpr int kBarBytes = 8 * (2 * kMaxStages + 5) + 64;

struct StreamParams {
    Fp4Head q;
    RestState* parts;              // [CTAs][N]
};

constexpr int scale_cols(int group) { return kUnits * fp4_scale_bytes(group) / 512 * 8; }          // of a stage in tensor memory: A's and B's
__host__ __device__ constexpr int acc_cols(int n) { return n < 32 ? 32 : n; }

template <int kGroup, int N>
struct Shape {
    static constexpr int kWUnit = fp4_unit_bytes(kGroup, kFp4Rows), kXUnit = fp4_unit_bytes(kGroup, N);
    static constexpr int kStageBytes = (kUnits * (kWUnit + kXUnit) + 1023) / 1024 * 1024;
    static constexpr int kZBytes = N * (kFp4Rows + 4) * 4;
    static constexpr int kTail = kZBytes + kBarBytes + 1024;
    static constexpr int kScaleCols = scale_cols(kGroup);
    static constexpr int kByTmem = (kTmemCols - 2 * acc_cols(N)) / kScaleCols;
    static constexpr int kBySmem = (int)(kSmemBudget - kTail) / kStageBytes;
    static constexpr int kFit = kByTmem < kBySmem ? kByTmem : kBySmem;
    static constexpr int kStages = kFit < kMaxStages ? kFit : kMaxStages;
    static constexpr size_t kSmem = (size_t)kStages * kStageBytes + kTail;
};

// Four more logits of a row into its state, in increasing order of their indices from idx on; without branches, so that the tokens of a warp overlap.
__device__ __forceinline__ void push4(RestState& a, float4 z, int idx) {
    const float top = fmaxf(fmaxf(z.x, z.y), fmaxf(z.z, z.w));
    const bool up = top > a.m;
    const bool at0 = z.x == top, at1 = !at0 && z.y == top, at2 = !at0 && !at1 && z.z == top, at3 = !at0 && !at1 && !at2;
    const float m = up ? top : a.m;
    const float d0 = z.x - m, d1 = z.y - m, d2 = z.z - m, d3 = z.w - m;
    // a new maximum leaves its term out of the sum, the old one's comes in
    const float e0 = up && at0 ? 0.f : ex2(d0 * kLog2e), e1 = up && at1 ? 0.f : ex2(d1 * kLog2e);
    const float e2 = up && at2 ? 0.f : ex2(d2 * kLog2e), e3 = up && at3 ? 0.f : ex2(d3 * kLog2e);
    const bool fresh = a.s == -1.f;
    const float dl = up && !fresh ? a.m - m : 0.f, al = ex2(dl * kLog2e);
    const float n = up ? 1.f + a.s : a.s;                                // 0 for a new state
    const float t = up ? al * fmaf(dl, n, a.t) : a.t;
    a.s = fmaf(al, n, (e0 + e1) + (e2 + e3));
    a.t = t + (fmaf(e0, d0, e1 * d1) + fmaf(e2, d2, e3 * d3));
    a.m = m;
    a.idx = up ? idx + (at0 ? 0 : at1 ? 1 : at2 ? 2 : 3) : a.idx;
}

// A warp: the CTAs' states of a token, a lane every 32nd CTA's.
__device__ __forceinline__ void merge_token(const StreamParams& p, int padded, int ctas, int tok, int lane) {
    RestState v[kStreamMaxCtas / 32];
#pragma unroll
    for (int i = 0; i < kStreamMaxCtas / 32; ++i) {
        const int b = lane + 32 * i;
        v[i] = b < ctas ? rest_load_cg(p.parts + (size_t)b * padded + tok) : rest_empty();
    }
    const RestState all = rest_reduce_lanes<1>(rest_combine(kStreamMaxCtas / 32, [&](int k) -> const RestState& { return v[k]; }));
    if (lane == 0) rest_finish(all, p.q, tok);
}

// Barrier of the eight epilogue warps; whether any of their threads says so.
__device__ __forceinline__ bool fold_barrier_any(bool mine) {
    uint32_t any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(any) : "r"(mine ? 1u : 0u) : "memory");
    return any != 0;
}

template <int kGroup, int N>
__global__ void __launch_bounds__(kThreads, 1) fp4_stream_kernel(const StreamParams p) {
    using S = Shape<kGroup, N>;
    constexpr int kTokens = (N + kFoldWarps - 1) / kFoldWarps;           // of an epilogue warp
    const Fp4Head& q = p.q;
    const int tiles = fp4_tiles(q.V, kFp4Rows), blocks = fp4_blocks(q.d), steps = (blocks + kUnits - 1) / kUnits;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw_addr = ptx::smem_addr(smem_raw);
    unsigned char* smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
    const uint32_t ring = ptx::smem_addr(smem);
    float* z_mem = reinterpret_cast<float*>(smem + S::kStages * S::kStageBytes);         // [N][128 + 4]
    unsigned char* bar_mem = reinterpret_cast<unsigned char*>(z_mem) + S::kZBytes;
    const uint32_t bar_base = ptx::smem_addr(bar_mem);
    auto full_bar = [&](int s) { return bar_base + 8u * s; };
    auto empty_bar = [&](int s) { return bar_base + 8u * (kMaxStages + s); };
    auto accfull_bar = [&](int b) { return bar_base + 8u * (2 * kMaxStages + b); };
    auto accfree_bar = [&](int b) { return bar_base + 8u * (2 * kMaxStages + 2 + b); };
    const uint32_t drain_bar = bar_base + 8u * (2 * kMaxStages + 4);
    volatile uint32_t* tmem_holder = reinterpret_cast<volatile uint32_t*>(bar_mem + 8 * (2 * kMaxStages + 5));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
    volatile int* is_last = abort_flag + 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    launch_dependents();
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
    const uint32_t tmem_base = *tmem_holder;
    const uint32_t scales_base = tmem_base + 2 * acc_cols(N);

    RestState st[kTokens];
#pragma unroll
    for (int i = 0; i < kTokens; ++i) st[i] = rest_empty();
    const float weight_factor = ld_dep(q.weight_factor);

    if (warp == 0) {
        // ---------------------------------------------------------------- producer
        if (ptx::elect_one()) {
            int stage = 0, issued = 0;
            uint32_t phase = 1, armed = 0, armed_parity = 0;
            bool ok = true;
            const unsigned char* x0 = q.acts;
            const int last_units = blocks - (steps - 1) * kUnits;
            auto load_w = [&](int s, const unsigned char* w, int units) { ptx::bulk_load(ring + s * S::kStageBytes, w, units * S::kWUnit, full_bar(s)); };
            auto load_x = [&](int s, const unsigned char* x, int units) {
                ptx::bulk_load(ring + s * S::kStageBytes + kUnits * S::kWUnit, x, units * S::kXUnit, full_bar(s));
            };
            const int n_pre = (int)blockIdx.x < tiles ? min(S::kStages, steps) : 0;
            for (int step = 0; step < n_pre; ++step) {
                const int units = step + 1 < steps ? kUnits : last_units;
                ptx::mbar_arrive_expect_tx(full_bar(step), units * (S::kWUnit + S::kXUnit));
                load_w(step, q.weights + ((size_t)blockIdx.x * blocks + step * kUnits) * S::kWUnit, units);
                armed |= 1u << step;
            }
            grid_dependency_wait();
            for (int tile = blockIdx.x; ok && tile < tiles; tile += gridDim.x) {
                const unsigned char* w = q.weights + (size_t)tile * blocks * S::kWUnit;
                const unsigned char* x = x0;
                for (int step = 0; step < steps; ++step, ++issued) {
                    const int units = step + 1 < steps ? kUnits : last_units;
                    if (issued >= n_pre) {
                        if (!ptx::mbar_wait(empty_bar(stage), phase, abort_flag)) {
                            record_failure(q.ctrl, abort_flag, 1, stage, tile);
                            ok = false;
                            break;
                        }
                        ptx::mbar_arrive_expect_tx(full_bar(stage), units * (S::kWUnit + S::kXUnit));
                        load_w(stage, w, units);
                        armed |= 1u << stage;
                        armed_parity = (armed_parity & ~(1u << stage)) | ((phase ^ 1u) << stage);
                    }
                    load_x(stage, x, units);
                    w += kUnits * S::kWUnit;
                    x += kUnits * S::kXUnit;
                    if (++stage == S::kStages) { stage = 0; phase ^= 1u; }
                }
            }
            if (*abort_flag) producer_drain(0, S::kStages, full_bar(0), armed, armed_parity);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------------- products (positions by addition: a single thread takes four to five
        // cycles for an instruction)
        if (ptx::elect_one()) {
            constexpr uint32_t idesc = ptx::idesc_fp4<kGroup>(kFp4Rows, N);
            constexpr int kAtoms = fp4_scale_bytes(kGroup) / 512;        // copies of scales per unit and operand
            const uint32_t low0 = ptx::desc_low(ring);
            uint32_t low = low0, cols = scales_base, full = full_bar(0), empty = empty_bar(0), phase = 0, acc_phase = 1;
            int stage = 0, buf = 0;
            bool ok = true;
            for (int tile = blockIdx.x; ok && tile < tiles; tile += gridDim.x) {
                if (!ptx::mbar_wait(accfree_bar(buf), acc_phase, abort_flag)) {
                    record_failure(q.ctrl, abort_flag, 2, 0x80 | buf, tile);
                    break;
                }
                ptx::tc_fence_after_sync();
                const uint32_t acc = tmem_base + buf * acc_cols(N);
                uint32_t accumulate = 0;
                int left = blocks;
                for (int step = 0; step < steps; ++step, left -= kUnits) {
                    if (!ptx::mbar_wait(full, phase, abort_flag)) {
                        record_failure(q.ctrl, abort_flag, 2, stage, tile);
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after_sync();
#pragma unroll
                    for (int u = 0; u < kUnits; ++u) {
                        if (u < left) {
                            const uint32_t wu = low + u * (S::kWUnit / 16), xu = low + (kUnits * S::kWUnit + u * S::kXUnit) / 16, su = cols + u * kAtoms * 8;
#pragma unroll
                            for (int k = 0; k < kAtoms; ++k) {
                                ptx::tmem_cp_scales(su + 8 * k, wu + 32 * k);
                                ptx::tmem_cp_scales(su + 8 * k + 4, xu + 32 * k);
                            }
                            constexpr uint32_t at = fp4_scale_bytes(kGroup) / 16, kSecond = kGroup == 16 ? 8 : 0;
                            // 64 columns are 32 bytes: two steps of the descriptor
                            ptx::mma_fp4<kGroup>(acc, wu + at, xu + at, idesc, su, su + 4, accumulate);
                            ptx::mma_fp4<kGroup>(acc, wu + at + 2, xu + at + 2, idesc | (kGroup == 32 ? ptx::kIdescFp4SecondHalf : 0u), su + kSecond,
                                                 su + kSecond + 4, 1u);
                            accumulate = 1;
                        }
                    }
                    ptx::mma_commit(empty);
                    low += S::kStageBytes / 16;
                    cols += S::kScaleCols;
                    full += 8;
                    empty += 8;
                    if (++stage == S::kStages) {
                        stage = 0;
                        low = low0;
                        cols = scales_base;
                        full = full_bar(0);
                        empty = empty_bar(0);
                        phase ^= 1u;
                    }
                }
                if (ok) ptx::mma_commit(accfull_bar(buf));
                buf ^= 1;
                acc_phase ^= buf == 0 ? 1u : 0u;
            }
            if (*abort_flag) mma_drain<false>(drain_bar);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- logits
        const int e = warp - 2, quarter = warp & 3, half = e >> 2;       // 32 rows, half of the tokens (all of them if there are eight)
        constexpr int kCols = N >= 16 ? N / 2 : N;
        grid_dependency_wait();
        float factor[kTokens];
#pragma unroll
        for (int i = 0; i < kTokens; ++i) factor[i] = e + i * kFoldWarps < q.M ? ld_dep(q.factor + e + i * kFoldWarps) * weight_factor : 0.f;
        int local = 0;
        for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, ++local) {
            const int buf = local & 1;
            const bool landed = warp_wait(accfull_bar(buf), (uint32_t)(local >> 1) & 1u, abort_flag);
            if (!landed && lane == 0) record_failure(q.ctrl, abort_flag, 3, buf, tile);
            if (fold_barrier_any(!landed)) break;                        // all eight warps or none; the tile before has been read
            ptx::tc_fence_after_sync();
            if (N >= 16 || half == 0) {
                const uint32_t from = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * acc_cols(N) + half * kCols;
                float* to = z_mem + half * kCols * (kFp4Rows + 4) + quarter * 32 + lane;
#pragma unroll
                for (int b = 0; b < kCols; b += 8) {
                    float v[8];
                    ptx::tmem_ld_32x8(from + b, v);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 8; ++j) to[(b + j) * (kFp4Rows + 4)] = v[j];
                }
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(accfree_bar(buf));
            fold_barrier_any(false);
            const int first = tile * kFp4Rows + lane * 4, valid = q.V - first;
#pragma unroll
            for (int i = 0; i < kTokens; ++i) {
                const int tok = e + i * kFoldWarps;
                if (valid > 0) {                                         // padding tokens too: the tokens of a warp overlap without a test between them
                    const float4 v = *reinterpret_cast<const float4*>(z_mem + tok * (kFp4Rows + 4) + lane * 4);
                    const float4 z = make_float4(v.x * factor[i], v.y * factor[i], v.z * factor[i], v.w * factor[i]);
                    if (valid >= 4) {
                        push4(st[i], z, first);
                    } else {
                        rest_push(st[i], z.x, first);
                        if (valid > 1) rest_push(st[i], z.y, first + 1);
                        if (valid > 2) rest_push(st[i], z.z, first + 2);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kTokens; ++i) st[i] = rest_reduce_lanes<1>(st[i]);
#pragma unroll
        for (int i = 0; i < kTokens; ++i)
            if (lane == 0 && e + i * kFoldWarps < q.M) p.parts[(size_t)blockIdx.x * N + e + i * kFoldWarps] = st[i];
    }
    if (warp < 2) grid_dependency_wait();
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem_base, kTmemCols);
    }
    if (N > kMergeHere) return;
    if (threadIdx.x == 0) *is_last = ticket_arrive_is_last(&q.ctrl->head_ticket[0], gridDim.x) ? 1 : 0;
    __syncthreads();
    if (!*is_last) return;
    for (int tok = warp; tok < q.M; tok += kThreads / 32) merge_token(p, N, (int)gridDim.x, tok, lane);
    if (threadIdx.x == 0) q.ctrl->head_ticket[0] = 0;                    // ready for the next launch
}

__global__ void __launch_bounds__(kMergeThreads) fp4_stream_merge_kernel(const StreamParams p, int padded, int ctas) {
    launch_dependents();
    grid_dependency_wait();
    const int tok = blockIdx.x * (kMergeThreads / 32) + (threadIdx.x >> 5);
    if (tok < p.q.M) merge_token(p, padded, ctas, tok, threadIdx.x & 31);
}

template <int kGroup, int N>
ee_status launch_tokens(const Fp4Head& q, void* parts, int num_sms, int device, cudaStream_t stream) {
    using S = Shape<kGroup, N>;
    static_assert(S::kStages >= 3, "ring");
    static bool configured[kMaxDevices] = {};
    if (!configured[device]) {
        if (cudaFuncSetAttribute(fp4_stream_kernel<kGroup, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem) != cudaSuccess) return EE_ERR_CUDA;
        configured[device] = true;
    }
    StreamParams p;
    p.q = q;
    p.parts = static_cast<RestState*>(parts);
    const int tiles = fp4_tiles(q.V, kFp4Rows);
    int grid = tiles < num_sms ? tiles : num_sms;
    if (grid > kStreamMaxCtas) grid = kStreamMaxCtas;
    if (launch_pdl(fp4_stream_kernel<kGroup, N>, dim3(grid), kThreads, S::kSmem, stream, p) != cudaSuccess) return EE_ERR_CUDA;
    if (N <= kMergeHere) return EE_OK;
    const int rows = kMergeThreads / 32;
    return launch_pdl(fp4_stream_merge_kernel, dim3((q.M + rows - 1) / rows), kMergeThreads, 0, stream, p, N, grid) == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}
template <int kGroup>
ee_status launch_group(const Fp4Head& q, void* parts, int num_sms, int device, cudaStream_t stream) {
    switch (fp4_stream_padded(q.M)) {
        case 8: return launch_tokens<kGroup, 8>(q, parts, num_sms, device, stream);
        case 16: return launch_tokens<kGroup, 16>(q, parts, num_sms, device, stream);
        case 32: return launch_tokens<kGroup, 32>(q, parts, num_sms, device, stream);
        default: return launch_tokens<kGroup, 64>(q, parts, num_sms, device, stream);
    }
}

}  // namespace

int fp4_stream_padded(int M) { return M <= 8 ? 8 : M <= 16 ? 16 : M <= 32 ? 32 : 64; }
size_t fp4_stream_parts_bytes(int M) { return (size_t)kStreamMaxCtas * fp4_stream_padded(M) * sizeof(RestState); }

ee_status fp4_stream_launch(const Fp4Head& q, int group, void* parts, int num_sms, int device, cudaStream_t stream) {
    return group == 16 ? launch_group<16>(q, parts, num_sms, device, stream) : launch_group<32>(q, parts, num_sms, device, stream);
}

}  // namespace ee
