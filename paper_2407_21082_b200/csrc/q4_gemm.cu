// A head in 4 bits on the 5th-generation tensor cores.
//
// One CTA per SM takes an equal share of W's 16-row tiles -- at V = 50304 on 148 SMs 21 or 22 of them -- and walks the width
// once, 64 columns at a time.  The weights are the M operand, in tensor memory: 24 warps unpack one tile each, from registers
// straight into the rows of three 128-row operands (tcgen05.st in the order of a matrix fragment, which is the order the
// packed form is laid out in), so unpacked weights touch neither shared memory nor its bandwidth.  The tokens are the N
// operand, in shared memory (TMA, up to 64 rows; a stage is read by three products).  (With the tokens as M and the weights
// written to shared memory as N, a stage of 64 columns took 0.89 us: the products read 78 KB of shared memory for it and waited
// for that, not for the tensor cores.)  The fragment order permutes the columns of every 64; y is written in the same order.
//
// Accumulators: three operands x N tokens (16, 32 or 64), in as many sets as 192 columns hold; k-block b goes to set b mod
// sets, and the sets are added up in fp32.  The tensor core truncates rather than rounds what falls below the last bit of its
// accumulator, which adds up over a row; with four sets (up to 16 tokens) a quarter as much.
//
// Then the CTA's logits go through shared memory, so that a thread has one token and some of the rows, and its states to the
// CTA that finishes last.  A share of more than 24 tiles goes in several passes; more than 64 tokens in several launches.
#include "q4_common.cuh"
#include "kernels.h"
#include "sm100_ptx.cuh"
#include "gemm_roles.cuh"
#include "tensor_map.h"

namespace ee {

namespace {

constexpr int kUnpackWarps = 24;                 // warp w: rows 16 (w / 4 % 2) + 32 (w % 4) of operand w / 8
constexpr int kOperands = 3;                     // of 128 rows, each with eight unpacking warps and a product warp
constexpr int kTmaWarp = kUnpackWarps, kProductWarp = kUnpackWarps + 1;
constexpr int kThreads = (kUnpackWarps + 1 + kOperands) * 32;
constexpr int kWorkers = kUnpackWarps * 32;      // threads of the softmax
constexpr int kAhead = 4;                        // packed blocks in flight per warp
constexpr int kMaxTiles = 24;
constexpr int kWStages = 3;                      // of 3 x 32 columns of tensor memory
constexpr int kYStages = 8;                      // of N x 128 bytes of shared memory
constexpr int kAccCols = 192;
constexpr int kTmemCols = 512;
constexpr int kBarBytes = 512;
constexpr size_t kSmemBudget = 226 * 1024;

struct GemmParams {
    Q4Params q;
    int passes;                                  // of every CTA
    int n;                                       // tokens, padded: 16, 32 or 64
    int sets;                                    // of accumulators
    int group_shift;                             // log2 of the scales' group
};

size_t z_bytes(int n) { return (size_t)kMaxTiles * 16 * (n + 4) * sizeof(float); }

// n states of a token, `stride` apart in shared memory: the maximum first, then the sums, so that no step waits for the one before.
__device__ __forceinline__ State combine_column(const State* s, int n, int stride) {
    float m = -CUDART_INF_F;
    for (int k = 0; k < n; ++k) m = fmaxf(m, s[k * stride].m);
    State r{m, 0.f, 0.f, 0x7fffffff};
    for (int k = 0; k < n; ++k) {
        const State o = s[k * stride];
        const bool live = !(o.s == 0.f);
        const float dl = o.m - m, al = live ? ex2(dl * kLog2e) : 0.f;
        r.s += live ? al * o.s : 0.f;
        r.t += live ? al * fmaf(dl, o.s, o.t) : 0.f;
        r.idx = (live && o.m == m) ? min(r.idx, o.idx) : r.idx;
    }
    if (r.s == 0.f) r.m = -CUDART_INF_F;
    return r;
}

__global__ void __launch_bounds__(kThreads, 1) q4_gemm_kernel(const __grid_constant__ CUtensorMap map_y, const GemmParams p) {
    const Q4Params& q = p.q;
    const Q4Layout l = q4_layout(q.V, q.d, q.group);
    const int t_begin = (int)((long long)blockIdx.x * l.tiles / gridDim.x), t_end = (int)((long long)(blockIdx.x + 1) * l.tiles / gridDim.x);
    const int nt = (t_end - t_begin + p.passes - 1) / p.passes;          // tiles of a pass (the last of several may have fewer)
    const int operands = (nt + 7) / 8;
    const int N = p.n, y_bytes = N * 128;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw_addr = ptx::smem_addr(smem_raw);
    unsigned char* smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
    const uint32_t y_base = ptx::smem_addr(smem);
    float* z_mem = reinterpret_cast<float*>(smem + kYStages * y_bytes);  // [rows][N + 4]
    State* states = reinterpret_cast<State*>(smem + kYStages * y_bytes + (size_t)kMaxTiles * 16 * (N + 4) * sizeof(float));   // [kWorkers / N][N]
    unsigned char* bar_mem = reinterpret_cast<unsigned char*>(states + kWorkers);
    const uint32_t bar_base = ptx::smem_addr(bar_mem);
    constexpr int kWBars = kOperands * kWStages;
    auto wfull_bar = [&](int o, int s) { return bar_base + 8u * (o * kWStages + s); };
    auto wempty_bar = [&](int o, int s) { return bar_base + 8u * (kWBars + o * kWStages + s); };
    auto yfull_bar = [&](int s) { return bar_base + 8u * (2 * kWBars + s); };
    auto yempty_bar = [&](int s) { return bar_base + 8u * (2 * kWBars + kYStages + s); };
    const uint32_t tfull_bar = bar_base + 8u * (2 * kWBars + 2 * kYStages);
    auto drain_bar = [&](int o) { return tfull_bar + 8u * (1 + o); };
    volatile uint32_t* tmem_holder = reinterpret_cast<volatile uint32_t*>(bar_mem + 8 * (2 * kWBars + 2 * kYStages + 1 + kOperands));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
    volatile int* is_last = abort_flag + 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    launch_dependents();

    // An unpacking warp keeps its tile of a pass from k-block to k-block; the first blocks are requested here, weights being
    // constants of the stream.
    const int quarter = warp & 3;
    const int slot = warp < kUnpackWarps ? (warp >> 3) * 8 + 2 * quarter + ((warp >> 2) & 1) : kMaxTiles;       // which of the pass's tiles
    const bool unpacks = slot < nt;
    const int g = lane >> 2, c = lane & 3;
    uint4 wq[kAhead];
    uint32_t sc[kAhead];
    const uint4* my_weights = nullptr;
    const uint32_t* my_scales = nullptr;
    auto fetch = [&](int i, int kb) {
        if (kb < l.blocks) {
            wq[i] = __ldg(my_weights + kb * 32);
            sc[i] = __ldg(my_scales + ((kb * 64 + c * 16) >> p.group_shift) * 8);
        }
    };
    auto begin_pass = [&](int pass) {
        const int tile = min(t_begin + pass * nt + slot, t_end - 1);
        my_weights = q.weights + (size_t)tile * l.blocks * 32 + lane;
        my_scales = q.scales + (size_t)tile * l.groups * 8 + g;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fetch(i, i);
    };
    if (unpacks) begin_pass(0);
    if (threadIdx.x == 0) {
        for (int o = 0; o < kOperands; ++o) {
            for (int s = 0; s < kWStages; ++s) {
                ptx::mbar_init(wfull_bar(o, s), max(1, min(8, nt - 8 * o)));
                ptx::mbar_init(wempty_bar(o, s), 1);
            }
            ptx::mbar_init(drain_bar(o), 1);
        }
        for (int s = 0; s < kYStages; ++s) {
            ptx::mbar_init(yfull_bar(s), 1);
            ptx::mbar_init(yempty_bar(s), operands);
        }
        ptx::mbar_init(tfull_bar, operands);
        *abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&map_y);
    }
    if (warp == kProductWarp) {
        ptx::tmem_alloc(ptx::smem_addr(const_cast<uint32_t*>(tmem_holder)), kTmemCols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_holder, ring = tmem_base + kAccCols;

    // softmax: thread = one token and every `shares`-th row
    const int tok = threadIdx.x & (N - 1), share = threadIdx.x / N, shares = kWorkers / N;
    State st = state_empty();
    bool ok = true;                                                      // of this warp's role
    int ws = 0, ys = 0;                                                  // ring positions
    uint32_t wp = 0, yp = 0;
    uint32_t armed = 0, armed_parity = 0;
    for (int pass = 0; pass < p.passes; ++pass) {
        if (warp == kTmaWarp) {
            // ---------------------------------------------------------------- y
            if (lane == 0) {
                if (pass == 0) grid_dependency_wait();
                for (int kb = 0; ok && kb < l.blocks; ++kb) {
                    if (!ptx::mbar_wait(yempty_bar(ys), yp ^ 1u, abort_flag)) {
                        record_failure(q.ctrl, abort_flag, 1, ys, kb);
                        ok = false;
                        break;
                    }
                    ptx::mbar_arrive_expect_tx(yfull_bar(ys), (uint32_t)y_bytes);
                    ptx::tma_load_2d(y_base + ys * y_bytes, &map_y, kb * 64, 0, yfull_bar(ys));
                    armed |= 1u << ys;
                    armed_parity = (armed_parity & ~(1u << ys)) | (yp << ys);
                    if (++ys == kYStages) { ys = 0; yp ^= 1u; }
                }
                if (*abort_flag) producer_drain(0, kYStages, yfull_bar(0), armed, armed_parity);
            }
            __syncwarp();
        } else if (warp >= kProductWarp) {
            // ---------------------------------------------------------------- products: a warp per operand (one thread issues a product in
            // about 75 cycles, whatever its size; twelve of them a stage by one thread were what the kernel waited for)
            const int o = warp - kProductWarp;
            if (lane == 0 && o < operands) {
                const uint32_t idesc = ptx::idesc_bf16_f32(128, N);
                int set = 0;
                for (int kb = 0; ok && kb < l.blocks; ++kb) {
                    if (!ptx::mbar_wait(yfull_bar(ys), yp, abort_flag) || !ptx::mbar_wait(wfull_bar(o, ws), wp, abort_flag)) {
                        record_failure(q.ctrl, abort_flag, 2, ws, kb);
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after_sync();
                    const uint64_t bdesc = ptx::smem_desc_k128(y_base + ys * y_bytes);
                    const uint32_t acc = tmem_base + (set * 3 + o) * N, a = ring + ws * 96 + o * 32;
#pragma unroll
                    for (int k = 0; k < 4; ++k) ptx::mma_bf16_ts(acc, a + k * 8, bdesc + 2u * k, idesc, (kb >= p.sets || k > 0) ? 1u : 0u);
                    ptx::mma_commit(wempty_bar(o, ws));
                    ptx::mma_commit(yempty_bar(ys));
                    if (++ws == kWStages) { ws = 0; wp ^= 1u; }
                    if (++ys == kYStages) { ys = 0; yp ^= 1u; }
                    if (++set == p.sets) set = 0;
                }
                if (ok) ptx::mma_commit(tfull_bar);
                if (*abort_flag) mma_drain<false>(drain_bar(o));
            }
            __syncwarp();
        } else if (unpacks) {
            // ---------------------------------------------------------------- unpacking
            if (pass > 0) begin_pass(pass);
            const int o = warp >> 3;
            const uint32_t to = ring + (uint32_t)o * 32u + ((uint32_t)(quarter * 32 + ((warp >> 2) & 1) * 16) << 16);
            for (int kb0 = 0; ok && kb0 < l.blocks; kb0 += kAhead) {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    if (kb0 + i >= l.blocks) break;
                    const uint32_t sl = low_twice(sc[i]), sh = high_twice(sc[i]);
                    uint32_t v[16];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {                        // pair k of the lane's eight, rows g and g + 8
                        v[(k >> 1) * 4 + (k & 1)] = q4_pair(k < 4 ? wq[i].x : wq[i].y, k & 3, sl);
                        v[(k >> 1) * 4 + 2 + (k & 1)] = q4_pair(k < 4 ? wq[i].z : wq[i].w, k & 3, sh);
                    }
                    fetch(i, kb0 + i + kAhead);
                    if (!__all_sync(0xffffffffu, ptx::mbar_wait(wempty_bar(o, ws), wp ^ 1u, abort_flag))) {
                        if (lane == 0) record_failure(q.ctrl, abort_flag, 4, ws, kb0 + i);
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after_sync();
                    ptx::tmem_st_16x64bf16(to + ws * 96, v);
                    ptx::tmem_st_wait();
                    ptx::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(wfull_bar(o, ws));
                    if (++ws == kWStages) { ws = 0; wp ^= 1u; }
                }
            }
        }
        // -------------------------------------------------------------------- logits to shared memory: rows x tokens
        if (pass == 0 && warp != kTmaWarp) grid_dependency_wait();
        if (!__all_sync(0xffffffffu, ptx::mbar_wait(tfull_bar, (uint32_t)pass & 1u, abort_flag))) {
            if (lane == 0) record_failure(q.ctrl, abort_flag, 3, 0, pass);
            ok = false;
        }
        ptx::tc_fence_after_sync();
        const int first = t_begin + pass * nt;
        const int rows = min(min(nt, t_end - first) * 16, q.V - first * 16);      // of this pass that exist
        if (warp < kUnpackWarps && ok) {
            // warp = a quarter of the lanes, operand (warp / 4) % 3, half (warp / 12) of the tokens
            const int o = (warp >> 2) % 3, half = warp / 12, r0 = o * 128 + quarter * 32;
            const int sets = min(p.sets, l.blocks);
            if (r0 < rows) {
                const uint32_t from = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(o * N + half * (N / 2));
                float* to = z_mem + (size_t)(r0 + lane) * (N + 4) + half * (N / 2);
                for (int b = 0; b < N / 2; b += 8) {
                    float z[8] = {};
                    for (int s = 0; s < sets; ++s) {
                        float x[8];
                        ptx::tmem_ld_32x8(from + s * 3 * N + b, x);
                        ptx::tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 8; ++j) z[j] += x[j];
                    }
                    *reinterpret_cast<float4*>(to + b) = make_float4(z[0], z[1], z[2], z[3]);
                    *reinterpret_cast<float4*>(to + b + 4) = make_float4(z[4], z[5], z[6], z[7]);
                }
            }
        }
        ptx::tc_fence_before_sync();
        __syncthreads();
        ptx::tc_fence_after_sync();
        if (threadIdx.x < kWorkers && tok < q.M && share < rows) {
            const float* z = z_mem + tok;
            float m = -CUDART_INF_F;
#pragma unroll 8
            for (int r = share; r < rows; r += shares) m = fmaxf(m, z[(size_t)r * (N + 4)]);
            float s = 0.f, t = 0.f;
            int idx = 0x7fffffff;
#pragma unroll 8
            for (int r = share; r < rows; r += shares) {
                const float x = z[(size_t)r * (N + 4)], dz = x - m, e = ex2(dz * kLog2e);
                s += e;
                t = fmaf(e, dz, t);
                idx = (x == m && idx == 0x7fffffff) ? r : idx;
            }
            state_merge(st, State{m, s, t, first * 16 + idx});
        }
        if (pass + 1 < p.passes) __syncthreads();                        // z is read before the next pass writes it
    }

    if (threadIdx.x < kWorkers) states[share * N + tok] = st;
    __syncthreads();
    if (warp == kProductWarp) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem_base, kTmemCols);
    }
    if ((int)threadIdx.x < q.M) q.parts[(size_t)blockIdx.x * N + threadIdx.x] = combine_column(states + threadIdx.x, shares, N);
    __syncthreads();
    if (threadIdx.x == 0) *is_last = ticket_arrive_is_last(&q.ctrl->head_ticket[0], gridDim.x) ? 1 : 0;
    __syncthreads();
    if (!*is_last) return;
    // the CTAs' states: lane = token, eight CTAs at a time in flight per thread, then as above
    if (threadIdx.x < kWorkers) {
        State s = state_empty();
        if (tok < q.M)
            for (int b0 = share; b0 < (int)gridDim.x; b0 += 8 * shares) {
                State v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int b = b0 + i * shares;
                    v[i] = b < (int)gridDim.x ? state_load_cg(q.parts + (size_t)b * N + tok) : state_empty();
                }
                state_merge(s, state_combine<8>(v));
            }
        states[share * N + tok] = s;
    }
    __syncthreads();
    if ((int)threadIdx.x < q.M)
        state_finish(combine_column(states + threadIdx.x, shares, N), q.tau_per_row ? ld_dep(q.tau_per_row + threadIdx.x) : q.tau, q.argmax,
                     q.entropy, q.maxprob, q.exit_mask, threadIdx.x);
    if (threadIdx.x == 0) q.ctrl->head_ticket[0] = 0;                    // ready for the next launch
}

}  // namespace

ee_status q4_gemm_launch(const Q4Params& q, int num_sms, int device, cudaStream_t stream) {
    static bool configured[kMaxDevices] = {};
    if (!configured[device]) {
        if (cudaFuncSetAttribute(q4_gemm_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBudget) != cudaSuccess) return EE_ERR_CUDA;
        configured[device] = true;
    }
    const Q4Layout l = q4_layout(q.V, q.d, q.group);
    GemmParams p;
    p.q = q;
    int grid = l.tiles < num_sms ? l.tiles : num_sms;
    if (grid > kStreamMaxCtas) grid = kStreamMaxCtas;
    const int most = (l.tiles + grid - 1) / grid;                        // tiles of the largest share
    p.passes = (most + kMaxTiles - 1) / kMaxTiles;
    p.n = q.M <= 16 ? 16 : q.M <= 32 ? 32 : 64;
    p.sets = kAccCols / (3 * p.n);
    p.group_shift = q.group == 32 ? 5 : q.group == 64 ? 6 : 7;
    const size_t smem = (size_t)kYStages * p.n * 128 + z_bytes(p.n) + kWorkers * sizeof(State) + kBarBytes + 1024;
    CUtensorMap map;
    if (!make_tile_map(&map, q.y, q.M, l.blocks * 64, p.n)) return EE_ERR_CUDA;
    return launch_pdl(q4_gemm_kernel, dim3(grid), kThreads, smem, stream, map, p) == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

}  // namespace ee
