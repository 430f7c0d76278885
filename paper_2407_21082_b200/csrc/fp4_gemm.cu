// A head in microscaled 4-bit floating point for many rows.
//
// Persistent pairs of CTAs; the activations (256 rows to a pair, 128 to a CTA) are the M operand of the products, the weight tiles of 128 rows the
// N operand, half of each staged by either CTA.  The tiles of the M x V plane are numbered row tile by row tile and every pair takes an equal run
// of them, so that it stays with its rows: in long runs their elements (up to d = 2560) stay in shared memory, and their scales in tensor memory, while the
// weights pass by (40 bytes per cycle and SM instead of 112; L2 gave 63), and the epilogue keeps the rows' softmax states in registers from
// tile to tile.  A state leaves the chip only where a run or a row tile ends.
//   warp 0 (one lane)  producer      warp 1 (one lane)  products      warps 2 .. 17  states      warp 18 (one lane)  scales to tensor memory
// Two warps share a quarter of an accumulator's lanes (thread = row), each half of its columns; of the two accumulators each has eight such warps.
//
// What it measured on the way, 16384 rows against V = 50304 (d = 2560 / 1024): 2.30 ms / - with one CTA per 128 x 128 tile, 1.37 with the tensor core's
// instructions issued under elect.sync instead of lane == 0, 1.32 as pairs with resident activations and one unit per stage, 0.93 / 0.69 with four
// (taking and giving a stage costs an issuing thread 250 cycles), 0.94 / 0.53 with sixteen epilogue warps instead of eight, each set with its own
// accumulator (a warp alone needs 1500 cycles for 32 columns: the terms depend on one another; eight warps could not hide that).
// Now 0.97 / 0.51 (narrow rows streamed); 4096 x 512 takes 124 us, 203 x 1056 24 us.
//
// What bounds it: at d = 2560 the products, some 200 cycles per 128 columns where 128 would be the tensor core's rate (with the loads left
// out of a copy 0.80 instead of 0.95 ms): a product of 256 x 128 reads 6 KB of operands per SM for 64 cycles of work.  256 weight rows at a
// time would halve that, but two such accumulators fill tensor memory, scales beside them do not fit.  At d <= 1024 the epilogue: a third of the chunks of a
// short run bring some row of the warp a new maximum, which costs three more instructions per logit, and 32 powers per chunk take 256 cycles.
#include "q4_common.cuh"
#include "fp4_common.cuh"
#include "gemm_roles.cuh"
#include "kernels.h"
#include "sm100_fp4.cuh"
#include "sm100_operands.cuh"
#include "tensor_map.h"

namespace ee {

namespace {

constexpr int kFoldWarps = 16, kParts = kFoldWarps / 4, kScaleWarp = 2 + kFoldWarps;
constexpr int kThreads = (3 + kFoldWarps) * 32;
constexpr int kTmemCols = 512;
constexpr int kAccCols = 128;
constexpr int kMaxPairs = 128;
constexpr int kMergeThreads = 256, kMergeLoads = 8;
constexpr int kBarBytes = 1024;
constexpr size_t kSmemBudget = 226 * 1024;
constexpr int kResidentBlocks = 20;              // units of a row tile that may stay on the chip
constexpr int kMaxStages = 12;
constexpr int kChunk = 32;                       // columns folded at a time
constexpr int kWarpCols = kAccCols / 2;          // ... of a tile, by a warp
constexpr int kUnits = 4;                        // units per stage: taking and giving one costs each issuing thread some 250 cycles

struct GemmMaps {
    // boxes: the scales of kUnits weight units, the halves of their elements that a CTA loads; the same of one unit; a unit of activations (or its
    // elements alone), the scales of several
    CUtensorMap scales, weights, scales_one, weights_one, acts, act_scales;
};
struct GemmParams {
    Fp4Head q;
    RestState* parts;              // [row][slot][part of the columns]
    int m_pairs, n_tiles, slots, n_stages;
};

// A stage of the ring holds kUnits halves of weight units, all those units' scales, and, unless they are resident, as many units of activations.
// kResident: the elements of a row tile's activations stay in shared memory, and their scales, which come through the ring as well, in tensor
// memory, while the weights pass by.
template <int kGroup, bool kResident>
struct Shape {
    static constexpr int kUnit = fp4_unit_bytes(kGroup, kFp4Rows), kScales = fp4_scale_bytes(kGroup), kElements = kUnit - kScales, kHalf = kElements / 2;
    static constexpr int kPartBytes = kHalf + kScales + (kResident ? 0 : kUnit), kStageBytes = kUnits * kPartBytes;
    static constexpr int kAtoms = kScales / 512;
    static constexpr int kUnitCols = kAtoms * 4;                               // of a unit's scales in tensor memory
    static constexpr int kPartCols = kResident ? kUnitCols : 2 * kUnitCols, kStageCols = kUnits * kPartCols;
    static constexpr int kScaleUnits = kStageBytes / kScales;                  // whose scales one stage brings
    static int resident_bytes(int blocks) { return kResident ? blocks * kElements : 0; }
    static int stages(int blocks) {
        const int by_smem = (int)(kSmemBudget - kBarBytes - 1024 - resident_bytes(blocks)) / kStageBytes;
        const int by_tmem = (kTmemCols - 2 * kAccCols - (kResident ? blocks * kUnitCols : 0)) / kStageCols;
        const int fit = by_smem < by_tmem ? by_smem : by_tmem;
        return fit < kMaxStages ? fit : kMaxStages;
    }
    static size_t smem(int blocks) { return (size_t)stages(blocks) * kStageBytes + resident_bytes(blocks) + kBarBytes + 1024; }
};

// The run of tiles of worker w of n, and the worker that has tile t.
__host__ __device__ inline long long run_begin(int w, int n, long long total) { return (long long)w * total / n; }
__host__ __device__ inline int worker_of(long long t, int n, long long total) { return (int)(((t + 1) * n - 1) / total); }
// Workers that share a row tile, at most.
int max_slots(int m_pairs, int n_tiles, int workers) {
    const long long total = (long long)m_pairs * n_tiles, each = total / workers > 0 ? total / workers : 1;
    return (int)((n_tiles + each - 1) / each) + 1;
}

// The state of a row while its logits v (before the power of two they have in common; `c` is that times log2 e) pass by: the largest, m, and sums of
// the others' 2^(v c - R) and 2^(v c - R) (v c - R) for R = round(m c), so that a term is one multiplication and addition, one power and two
// additions.  The maximum's own term, left out, is 2^d with d = m c - R, which is as good as exact and taken out at the end.
__device__ __forceinline__ float reference(float m, float c) { return __fmul_rn(m, c); }
__device__ __forceinline__ float beside_reference(float m, float c) { return fmaf(m, c, -__fmul_rn(m, c)); }

// Adds a chunk's terms.  In the plain form all of them; otherwise the first nvalid, and where the maximum is new (`up`) all but those that equal
// it, whose columns come back as bits.  The order of the sums is the same, so that a row's result does not depend on which form its warp takes.
template <bool kPlain, bool kFull>
__device__ __forceinline__ uint32_t add_terms(RestState& st, const float (&v)[kChunk], float c, bool up, int nvalid) {
    const float r = -reference(st.m, c);
    const unsigned long long minus_r = ptx::pack_f32x2(r, r), cc = ptx::pack_f32x2(c, c);
    unsigned long long s[2] = {0, 0}, t[2] = {0, 0};
    uint32_t tops = 0;
#pragma unroll
    for (int j = 0; j < kChunk; j += 2) {
        const unsigned long long a2 = ptx::fma_f32x2(ptx::pack_f32x2(v[j], v[j + 1]), cc, minus_r);
        const float2 a = ptx::unpack_f32x2(a2);
        float2 x = make_float2(ex2(a.x), ex2(a.y));
        if (!kPlain) {
            const bool top0 = up && v[j] == st.m, top1 = up && v[j + 1] == st.m;
            const bool in0 = kFull || j < nvalid, in1 = kFull || j + 1 < nvalid;
            if (top0 || !in0) x.x = 0.f;
            if (top1 || !in1) x.y = 0.f;
            if (top0 && in0) tops |= 1u << j;
            if (top1 && in1) tops |= 2u << j;
        }
        const unsigned long long e = ptx::pack_f32x2(x.x, x.y);
        s[(j >> 1) & 1] = ptx::add_f32x2(s[(j >> 1) & 1], e);
        t[(j >> 1) & 1] = ptx::fma_f32x2(e, a2, t[(j >> 1) & 1]);
    }
    const float2 ss = ptx::unpack_f32x2(ptx::add_f32x2(s[0], s[1])), tt = ptx::unpack_f32x2(ptx::add_f32x2(t[0], t[1]));
    st.s += ss.x + ss.y;
    st.t += tt.x + tt.y;
    return tops;
}

// A chunk of consecutive logits.  A new maximum is rare in a long row: some ten of a thousand chunks bring one.
__device__ __forceinline__ void fold_chunk(RestState& st, const float (&v)[kChunk], float c, int col0, int nvalid) {
    float cm[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
    if (nvalid >= kChunk) {
#pragma unroll
        for (int j = 0; j < kChunk; j += 2) cm[(j >> 1) & 3] = ptx::max3(cm[(j >> 1) & 3], v[j], v[j + 1]);
    } else {
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
            if (j < nvalid) cm[j & 3] = fmaxf(cm[j & 3], v[j]);
    }
    const float top = fmaxf(ptx::max3(cm[0], cm[1], cm[2]), cm[3]);
    const bool up = top > st.m;
    if (nvalid >= kChunk && !__any_sync(0xffffffffu, up)) {
        add_terms<true, true>(st, v, c, false, kChunk);
        return;
    }
    if (up) {
        if (st.s == -1.f) {
            st.s = st.t = 0.f;
        } else {                                                         // the old maximum's term comes in, all of them go to the new reference
            const float d = beside_reference(st.m, c), w = ex2(d), n = st.s + w;
            const float dl = reference(st.m, c) - reference(top, c), al = ex2(dl);
            st.t = al * fmaf(dl, n, fmaf(w, d, st.t));
            st.s = al * n;
        }
        st.m = top;
    }
    const uint32_t tops = nvalid >= kChunk ? add_terms<false, true>(st, v, c, up, kChunk) : add_terms<false, false>(st, v, c, up, nvalid);
    if (up) {
        const float more = (float)(__popc(tops) - 1), d = beside_reference(top, c), w = ex2(d);
        st.idx = col0 + __ffs(tops) - 1;
        st.s = fmaf(more, w, st.s);
        st.t = fmaf(more, w * d, st.t);
    }
}

// ... as a state in nats beside its own maximum.
__device__ __forceinline__ RestState finished(const RestState& st, float factor, float c) {
    if (st.s == -1.f) return st;
    const float d = beside_reference(st.m, c), w = ex2(-d);
    return RestState{st.m * factor, st.s * w, kLn2 * w * fmaf(-d, st.s, st.t), st.idx};
}

template <int kGroup, bool kResident>
__global__ void __launch_bounds__(kThreads, 1) fp4_gemm_kernel(const __grid_constant__ GemmMaps maps, const GemmParams p) {
    using S = Shape<kGroup, kResident>;
    const Fp4Head& q = p.q;
    const int rank = (int)ptx::cluster_cta_rank(), pair = (int)(blockIdx.x >> 1), pairs = (int)(gridDim.x >> 1);
    const int n_stages = p.n_stages, blocks = fp4_blocks(q.d);
    const long long total = (long long)p.m_pairs * p.n_tiles;
    const long long begin = run_begin(pair, pairs, total), end = run_begin(pair + 1, pairs, total);
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw_addr = ptx::smem_addr(smem_raw);
    unsigned char* smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
    const uint32_t ring = ptx::smem_addr(smem), resident = ring + n_stages * S::kStageBytes;
    unsigned char* bar_mem = smem + n_stages * S::kStageBytes + (kResident ? blocks * S::kElements : 0);
    const uint32_t bar_base = ptx::smem_addr(bar_mem);
    auto full_bar = [&](int s) { return bar_base + 8u * s; };                            // in rank 0: both CTAs' loads have landed
    auto empty_bar = [&](int s) { return bar_base + 8u * (kMaxStages + s); };
    auto act_bar = [&](int u) { return bar_base + 8u * (2 * kMaxStages + u); };          // in rank 0, likewise
    const uint32_t act_free = bar_base + 8u * (2 * kMaxStages + kResidentBlocks);
    auto accfull_bar = [&](int b) { return act_free + 8u * (1 + b); };
    auto accfree_bar = [&](int b) { return act_free + 8u * (3 + b); };                   // in rank 0: both CTAs' epilogues
    const uint32_t drain_bar = act_free + 8u * 5;
    auto ready_bar = [&](int s) { return act_free + 8u * (6 + s); };                     // in rank 0: the scales are in tensor memory too
    volatile uint32_t* tmem_holder = reinterpret_cast<volatile uint32_t*>(bar_mem + 8 * (3 * kMaxStages + kResidentBlocks + 6));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
    static_assert(8 * (3 * kMaxStages + kResidentBlocks + 6) + 8 <= kBarBytes, "barriers");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < n_stages; ++s) {
            ptx::mbar_init(full_bar(s), 1);
            ptx::mbar_init(empty_bar(s), 1);
            ptx::mbar_init(ready_bar(s), 1);
        }
        for (int u = 0; u < kResidentBlocks; ++u) ptx::mbar_init(act_bar(u), 1);
        ptx::mbar_init(act_free, 1);
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(accfull_bar(b), 1);
            ptx::mbar_init(accfree_bar(b), kFoldWarps);          // half of the warps, of both CTAs
        }
        ptx::mbar_init(drain_bar, 1);
        *abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&maps.acts);
        ptx::prefetch_tensormap(&maps.weights);
        ptx::prefetch_tensormap(&maps.scales);
        if (kResident) ptx::prefetch_tensormap(&maps.act_scales);
        ptx::prefetch_tensormap(&maps.weights_one);
        ptx::prefetch_tensormap(&maps.scales_one);
    }
    if (warp == 1) {
        ptx::tmem_alloc_pair(ptx::smem_addr(const_cast<uint32_t*>(tmem_holder)), kTmemCols);
        ptx::tmem_relinquish_pair();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::cluster_sync_all();                              // the partner's barriers exist before anything signals them
    ptx::tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_holder, act_cols = tmem_base + 2 * kAccCols, stage_cols = act_cols + (kResident ? blocks * S::kUnitCols : 0);

    // The two issuing threads have some hundred cycles per unit, at four to five per instruction of a single thread: positions in the ring are
    // moved along by additions.
    if (warp == 0) {
        // ---------------------------------------------------------------- producer
        if (ptx::elect_one()) {
            const uint32_t ring_end = ring + n_stages * S::kStageBytes;
            const uint32_t full0 = ptx::map_to_cta(full_bar(0), 0), act0 = ptx::map_to_cta(act_bar(0), 0);         // where loads report
            uint32_t to = ring, full = full0, empty = empty_bar(0), phase = 1;
            int fills = 0;
            bool ok = true;
            auto next_stage = [&](unsigned what) {
                if (ptx::mbar_wait(empty, phase, abort_flag)) return true;
                record_failure(q.ctrl, abort_flag, 1, (to - ring) / S::kStageBytes, what);
                return ok = false;
            };
            auto stage_done = [&]() {
                to += S::kStageBytes;
                full += 8;
                empty += 8;
                if (to == ring_end) {
                    to = ring;
                    full = full0;
                    empty = empty_bar(0);
                    phase ^= 1u;
                }
            };
            long long m_pair = begin / p.n_tiles;
            int n_tile = (int)(begin - m_pair * p.n_tiles);
            bool fresh = kResident;
            // The weights of the first stages do not wait for the kernel that writes the activations.
            constexpr int kScaleStages = kResident ? (kResidentBlocks + S::kScaleUnits - 1) / S::kScaleUnits : 0;
            const int scale_stages = kResident ? (blocks + S::kScaleUnits - 1) / S::kScaleUnits : 0;
            static_assert(kScaleStages < 3, "the first stages");
            int ahead = 0;                                // steps of the first tile whose weights are under way
            if (begin < end) ahead = max(0, min(n_stages - scale_stages, (blocks + kUnits - 1) / kUnits));
            const int half_line = S::kScales / 128 + rank * (S::kHalf / 128);
            auto load_weights = [&](uint32_t at, int unit, int n, uint32_t bar) {        // n units: one request of kUnits, or one by one
                if (n == kUnits) {
                    ptx::tma_load_3d_pair(at, &maps.weights, 0, half_line, unit, bar);
                    ptx::tma_load_3d_pair(at + kUnits * S::kHalf, &maps.scales, 0, 0, unit, bar);
                } else {
                    for (int k = 0; k < n; ++k) {
                        ptx::tma_load_3d_pair(at + k * S::kHalf, &maps.weights_one, 0, half_line, unit + k, bar);
                        ptx::tma_load_3d_pair(at + kUnits * S::kHalf + k * S::kScales, &maps.scales_one, 0, 0, unit + k, bar);
                    }
                }
            };
            for (int step = 0; step < ahead; ++step) {
                const int n = min(kUnits, blocks - step * kUnits), s = scale_stages + step;
                if (rank == 0) ptx::mbar_arrive_expect_tx(full_bar(s), 2 * n * S::kPartBytes);
                load_weights(ring + s * S::kStageBytes, n_tile * blocks + step * kUnits, n, full0 + 8 * s);
            }
            grid_dependency_wait();
            for (long long t = begin; ok && t < end; ++t) {
                if (t + 1 == end) launch_dependents();
                const int act_unit = (int)(2 * m_pair + rank) * blocks;
                if (fresh) {
                    // the products of the row tile before have read their activations
                    if (fills > 0 && !ptx::mbar_wait(act_free, (uint32_t)(fills - 1) & 1u, abort_flag)) {
                        record_failure(q.ctrl, abort_flag, 1, 0x80, (unsigned)t);
                        break;
                    }
                    ++fills;
                    for (int u0 = 0; u0 < blocks && next_stage((unsigned)t); u0 += S::kScaleUnits) {
                        if (rank == 0) ptx::mbar_arrive_expect_tx(full_bar(0) + (full - full0), 2 * S::kScaleUnits * S::kScales);
                        ptx::tma_load_3d_pair(to, &maps.act_scales, 0, 0, act_unit + u0, full);
                        stage_done();
                    }
                }
                const int unit = n_tile * blocks;
                for (int u0 = 0; u0 < blocks && ok && next_stage((unsigned)t); u0 += kUnits) {
                    const int n = min(kUnits, blocks - u0);
                    const bool here = ahead == 0;
                    ahead -= here ? 0 : 1;
                    if (rank == 0 && here) ptx::mbar_arrive_expect_tx(full_bar(0) + (full - full0), 2 * n * S::kPartBytes);
                    if (here) load_weights(to, unit + u0, n, full);
                    for (int u = u0; fresh && u < u0 + n; ++u) {
                        if (rank == 0) ptx::mbar_arrive_expect_tx(act_bar(u), 2 * S::kElements);
                        ptx::tma_load_3d_pair(resident + u * S::kElements, &maps.acts, 0, S::kScales / 128, act_unit + u, act0 + 8 * u);
                    }
                    for (int k = 0; !kResident && k < n; ++k)
                        ptx::tma_load_3d_pair(to + kUnits * (S::kHalf + S::kScales) + k * S::kUnit, &maps.acts, 0, 0, act_unit + u0 + k, full);
                    stage_done();
                }
                fresh = false;
                if (++n_tile == p.n_tiles) {
                    n_tile = 0;
                    ++m_pair;
                    fresh = kResident;
                }
            }
            if (*abort_flag) {                            // copies still in flight: of the stages' last or last but one fill, and of the activations
                if (rank != 0) producer_drain(1, 0, 0, 0, 0);
                else
                    for (int i = 0; i < 10000; ++i) __nanosleep(1000);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------------- products
        if (rank == 0 && ptx::elect_one()) {
            constexpr uint32_t idesc = ptx::idesc_fp4<kGroup>(2 * kFp4Rows, kFp4Rows);
            const int scale_stages = kResident ? (blocks + S::kScaleUnits - 1) / S::kScaleUnits : 0;
            const uint32_t low0 = ptx::desc_low(ring), act_low = ptx::desc_low(resident);
            uint32_t low = low0, cols = stage_cols, ready = ready_bar(0), empty = empty_bar(0), phase = 0;
            uint32_t acc_phase = 1, act_phase = 1;
            int left = n_stages;
            bool ok = true;
            auto landed = [&](uint32_t bar, uint32_t parity, unsigned what) {
                if (ptx::mbar_wait(bar, parity, abort_flag)) return true;
                record_failure(q.ctrl, abort_flag, 2, (bar - bar_base) / 8, what);
                return ok = false;
            };
            auto next_stage = [&]() {
                low += S::kStageBytes / 16;
                cols += S::kStageCols;
                ready += 8;
                empty += 8;
                if (--left == 0) {
                    left = n_stages;
                    low = low0;
                    cols = stage_cols;
                    ready = ready_bar(0);
                    empty = empty_bar(0);
                    phase ^= 1u;
                }
            };
            int n_tile = (int)(begin % p.n_tiles), buf = 0;
            bool fresh = kResident;
            for (long long t = begin; ok && t < end; ++t) {
                if (fresh) {                              // stages of the activations' scales are the scale warp's alone
                    act_phase ^= 1u;
                    for (int i = 0; i < scale_stages; ++i) next_stage();
                }
                if (!landed(accfree_bar(buf), acc_phase, (unsigned)t)) break;
                ptx::tc_fence_after_sync();
                const uint32_t acc = tmem_base + buf * kAccCols;
                uint32_t x_low = act_low, x_cols = act_cols;
                for (int u0 = 0; u0 < blocks && landed(ready, phase, (unsigned)t); u0 += kUnits) {
                    const int n = min(kUnits, blocks - u0);
                    for (int k = 0; fresh && k < n; ++k) landed(act_bar(u0 + k), act_phase, (unsigned)t);
                    ptx::tc_fence_after_sync();
#pragma unroll
                    for (int k = 0; k < kUnits; ++k) {
                        if (k >= n) break;
                        const uint32_t w_low = low + k * (S::kHalf / 16), w_cols = cols + k * S::kUnitCols;
                        const uint32_t a_low = kResident ? x_low + k * (S::kElements / 16) : low + (kUnits * (S::kHalf + S::kScales) + k * S::kUnit + S::kScales) / 16;
                        const uint32_t a_cols = kResident ? x_cols + k * S::kUnitCols : cols + (kUnits + k) * S::kUnitCols;
                        // 64 columns are 32 bytes: two steps of the descriptor
                        constexpr uint32_t kSecond = kGroup == 16 ? 4 : 0;   // the other scales, or the other half of the same ones
                        ptx::mma_fp4<kGroup, true>(acc, a_low, w_low, idesc, a_cols, w_cols, k > 0 || u0 > 0 ? 1u : 0u);
                        ptx::mma_fp4<kGroup, true>(acc, a_low + 2, w_low + 2, idesc | (kGroup == 32 ? ptx::kIdescFp4SecondHalf : 0u), a_cols + kSecond,
                                                   w_cols + kSecond, 1u);
                    }
                    x_low += kUnits * (S::kElements / 16);
                    x_cols += kUnits * S::kUnitCols;
                    ptx::mma_commit_pair(empty, 3);       // frees the stage, in both CTAs, once all products so far have been computed
                    next_stage();
                }
                if (!ok) break;
                ptx::mma_commit_pair(accfull_bar(buf), 3);
                fresh = false;
                if (++n_tile == p.n_tiles) {
                    n_tile = 0;
                    fresh = kResident;
                    if (kResident && t + 1 < end) ptx::mma_commit_pair(act_free, 3);
                }
                buf ^= 1;
                acc_phase ^= buf == 0 ? 1u : 0u;
            }
            if (*abort_flag) mma_drain<true>(drain_bar);
        }
        __syncwarp();
    } else if (warp == kScaleWarp) {
        // ---------------------------------------------------------------- scales to tensor memory, in both CTAs
        if (rank == 0 && ptx::elect_one()) {
            const uint32_t low0 = ptx::desc_low(ring);
            uint32_t low = low0, cols = stage_cols, phase = 0;
            int stage = 0;
            bool ok = true;
            auto landed = [&](unsigned what) {
                if (ptx::mbar_wait(full_bar(stage), phase, abort_flag)) {
                    ptx::tc_fence_after_sync();
                    return true;
                }
                record_failure(q.ctrl, abort_flag, 4, stage, what);
                return ok = false;
            };
            auto next_stage = [&]() {
                low += S::kStageBytes / 16;
                cols += S::kStageCols;
                if (++stage == n_stages) {
                    stage = 0;
                    low = low0;
                    cols = stage_cols;
                    phase ^= 1u;
                }
            };
            int n_tile = (int)(begin % p.n_tiles);
            bool fresh = kResident;
            for (long long t = begin; ok && t < end; ++t) {
                for (int u0 = 0; fresh && u0 < blocks && landed((unsigned)t); u0 += S::kScaleUnits) {
                    for (int k = 0; k < min(S::kScaleUnits, blocks - u0) * S::kAtoms; ++k)
                        ptx::tmem_cp_scales<true>(act_cols + u0 * S::kUnitCols + 4 * k, low + 32 * k);
                    ptx::mma_commit_pair(ready_bar(stage), 1);           // nobody waits for it here, but its phases go with the ring's turns
                    ptx::mma_commit_pair(empty_bar(stage), 3);
                    next_stage();
                }
                for (int u0 = 0; u0 < blocks && ok && landed((unsigned)t); u0 += kUnits) {
                    const int n = min(kUnits, blocks - u0);
#pragma unroll
                    for (int k = 0; k < kUnits * S::kAtoms; ++k)
                        if (k < n * S::kAtoms) ptx::tmem_cp_scales<true>(cols + 4 * k, low + kUnits * S::kHalf / 16 + 32 * k);
                    for (int k = 0; !kResident && k < n * S::kAtoms; ++k)
                        ptx::tmem_cp_scales<true>(cols + kUnits * S::kUnitCols + 4 * k,
                                                  low + (kUnits * (S::kHalf + S::kScales) + k / S::kAtoms * S::kUnit) / 16 + 32 * (k % S::kAtoms));
                    ptx::mma_commit_pair(ready_bar(stage), 1);
                    next_stage();
                }
                fresh = false;
                if (++n_tile == p.n_tiles) {
                    n_tile = 0;
                    fresh = kResident;
                }
            }
            if (*abort_flag)                              // copies still on their way
                for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- states (every second tile: a set of eight warps has an accumulator
        // for itself, so that the way from products to states and back is hidden behind the other set's work)
        const int quarter = warp & 3, part = (warp - 2) >> 2, buf = part >> 1, half = part & 1;
        RestState st = rest_empty();
        grid_dependency_wait();
        const float weight_factor = ld_dep(q.weight_factor);
        float factor = 0.f, c = 0.f;
        int m_pair = (int)(begin / p.n_tiles), n_tile = (int)(begin - (long long)m_pair * p.n_tiles);
        auto row_of = [&](int m) { return (2ll * m + rank) * kFp4Rows + quarter * 32 + lane; };
        auto take = [&]() {                               // the rows of tile pair m_pair
            factor = row_of(m_pair) < q.M ? ld_dep(q.factor + row_of(m_pair)) * weight_factor : 1.f;
            c = factor * kLog2e;
        };
        auto flush = [&]() {
            const long long row = row_of(m_pair);
            const int slot = pair - worker_of((long long)m_pair * p.n_tiles, pairs, total);
            if (row < q.M) p.parts[(row * p.slots + slot) * kParts + part] = finished(st, factor, c);
            st = rest_empty();
        };
        take();
        uint32_t phase = 0;
        for (long long t = begin; t < end; ++t, ++n_tile) {
            if (n_tile == p.n_tiles) {
                flush();
                n_tile = 0;
                ++m_pair;
                take();
            }
            if (((int)(t - begin) & 1) != buf) continue;
            if (!warp_wait(accfull_bar(buf), phase, abort_flag)) {
                if (lane == 0) record_failure(q.ctrl, abort_flag, 3, buf, (unsigned)t);
                break;
            }
            phase ^= 1u;
            ptx::tc_fence_after_sync();
            const uint32_t from = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * kAccCols + half * kWarpCols;
            const int col0 = n_tile * kFp4Rows + half * kWarpCols;
#pragma unroll 1
            for (int k = 0; k < kWarpCols; k += kChunk) {
                float v[kChunk];
                ptx::tmem_ld_32x32(from + k, v);
                ptx::tmem_ld_wait();
                if (k + kChunk == kWarpCols) {
                    ptx::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive_remote(ptx::map_to_cta(accfree_bar(buf), 0));
                }
                const int nvalid = q.V - (col0 + k);
                if (nvalid > 0) fold_chunk(st, v, c, col0 + k, nvalid);
            }
        }
        flush();
    }
    if (warp < 2 || warp == kScaleWarp) grid_dependency_wait();
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::cluster_sync_all();                              // neither CTA leaves while the other may still signal it or write its accumulators
    if (warp == 1) {
        __syncwarp();
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc_pair(tmem_base, kTmemCols);
    }
}

// A warp per row: the states of the pairs that shared its tile.
__global__ void __launch_bounds__(kMergeThreads) fp4_merge_kernel(const GemmParams p, int pairs) {
    launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * (kMergeThreads / 32) + (threadIdx.x >> 5);
    if (row >= p.q.M) return;
    const long long total = (long long)p.m_pairs * p.n_tiles, first = row / (2 * kFp4Rows) * p.n_tiles;
    const int n = kParts * (worker_of(first + p.n_tiles - 1, pairs, total) - worker_of(first, pairs, total) + 1);
    const RestState* parts = p.parts + row * p.slots * kParts;
    RestState mine = rest_empty();
    for (int k0 = lane; k0 < n; k0 += 32 * kMergeLoads) {
        RestState v[kMergeLoads];
#pragma unroll
        for (int i = 0; i < kMergeLoads; ++i) v[i] = k0 + 32 * i < n ? rest_load_cg(parts + k0 + 32 * i) : rest_empty();
        rest_merge(mine, rest_combine(kMergeLoads, [&](int k) -> const RestState& { return v[k]; }));
    }
    const RestState all = rest_reduce_lanes<1>(mine);
    if (lane == 0) rest_finish(all, p.q, (int)row);
}

// Units of 128 rows as [units][lines of 128 bytes], boxes of `lines` of `units` neighbouring units.
bool make_unit_map(CUtensorMap* map, const void* base, int group, long long n_units, int lines, int units) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t unit = fp4_unit_bytes(group, kFp4Rows);
    const cuuint64_t dims[3] = {128u, unit / 128, (cuuint64_t)n_units};
    const cuuint64_t strides[2] = {128u, unit};
    const cuuint32_t box[3] = {128u, (cuuint32_t)lines, (cuuint32_t)units};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Pairs of CTAs the device runs at once; 0 if the query fails.
template <int kGroup, bool kResident>
int resident_pairs(int device) {
    static int pairs[kMaxDevices];
    static bool asked[kMaxDevices] = {};
    if (!asked[device]) {
        int n = 0;
        if (cudaFuncSetAttribute(fp4_gemm_kernel<kGroup, kResident>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBudget) == cudaSuccess) {
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute attr[2];
            pair_launch_config(cfg, attr, dim3(2), kThreads, kSmemBudget, nullptr);
            if (cudaOccupancyMaxActiveClusters(&n, fp4_gemm_kernel<kGroup, kResident>, &cfg) != cudaSuccess) {
                n = 0;
                (void)cudaGetLastError();
            }
        }
        pairs[device] = n < kMaxPairs ? n : kMaxPairs;
        asked[device] = true;
    }
    return pairs[device];
}

int pairs_of(long long total, int most) { return total < most ? (int)total : most; }

template <int kGroup, bool kResident>
ee_status launch_shape(GemmParams p, int device, cudaStream_t stream) {
    using S = Shape<kGroup, kResident>;
    const int most = resident_pairs<kGroup, kResident>(device);
    if (most == 0) return EE_ERR_CUDA;
    const int blocks = fp4_blocks(p.q.d), pairs = pairs_of((long long)p.m_pairs * p.n_tiles, most);
    p.slots = max_slots(p.m_pairs, p.n_tiles, pairs);
    p.n_stages = S::stages(blocks);
    GemmMaps maps;
    const long long act_units = 2ll * p.m_pairs * blocks, weight_units = (long long)p.n_tiles * blocks;
    if (!make_unit_map(&maps.scales, p.q.weights, kGroup, weight_units, S::kScales / 128, kUnits) ||
        !make_unit_map(&maps.weights, p.q.weights, kGroup, weight_units, S::kHalf / 128, kUnits) ||
        !make_unit_map(&maps.scales_one, p.q.weights, kGroup, weight_units, S::kScales / 128, 1) ||
        !make_unit_map(&maps.weights_one, p.q.weights, kGroup, weight_units, S::kHalf / 128, 1) ||
        !make_unit_map(&maps.acts, p.q.acts, kGroup, act_units, (kResident ? S::kElements : S::kUnit) / 128, 1) ||
        !make_unit_map(&maps.act_scales, p.q.acts, kGroup, act_units, S::kScales / 128, kResident ? S::kScaleUnits : 1))
        return EE_ERR_CUDA;
    if (launch_pdl_pairs(fp4_gemm_kernel<kGroup, kResident>, dim3(2 * pairs), kThreads, S::smem(blocks), stream, maps, p) != cudaSuccess) return EE_ERR_CUDA;
    const int rows = kMergeThreads / 32;
    return launch_pdl(fp4_merge_kernel, dim3((p.q.M + rows - 1) / rows), kMergeThreads, 0, stream, p, pairs) == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

// Whether a pair keeps the activations of its row tile.  It saves their loads, which the products of wide rows wait for, and power; it costs a start at
// which a row tile arrives before anything else, and stages, of which three are left at d = 2560.  So: wide rows, long runs.
// Kept / streamed, us, V = 50304, groups of 16; short runs: 300 rows of 1024 34.1 / 31.2, of 2560 51.1 / 43.9, 1000 of 2560 84 / 76, 4096 of 1024 150 / 142, of 1536
// 192 / 187, of 2048 231 / 230, of 2560 273 / 275.  Long runs (medians of calls back to back, under the power cap): 16384 of 1024 568 / 539, of 1536
// 733 / 746, of 2048 878 / 924, of 2560 1175 / 1126, and by themselves, at full clocks, 958 / 1040; 6144 of 2048 334 / 339, of 2560 449 / 426 and 408 / 401.
// Groups of 32: 16384 of 1536 687 / 689, of 2048 817 / 857, of 2560 1084 / 1054 and 898 / 973.
constexpr int kStreamedBlocks = 12;              // up to so many units of a row
constexpr int kLongRun = 128;                    // tiles

template <int kGroup>
ee_status launch_group(const GemmParams& p, int device, cudaStream_t stream) {
    const int blocks = fp4_blocks(p.q.d);
    const bool keep = blocks > kStreamedBlocks && blocks <= kResidentBlocks &&
                      (long long)p.m_pairs * p.n_tiles >= (long long)kLongRun * resident_pairs<kGroup, true>(device);
    return keep ? launch_shape<kGroup, true>(p, device, stream) : launch_shape<kGroup, false>(p, device, stream);
}

}  // namespace

int fp4_gemm_act_tiles(int M) { return (fp4_tiles(M, kFp4Rows) + 1) / 2 * 2; }

// For any number of pairs, and the most that any number of rows up to M takes: fewer rows have shorter runs, and more states to a row.  From
// kMaxPairs pairs of row tiles on a run is a row tile at least, and the states grow with the rows.
size_t fp4_gemm_parts_bytes(int M, int V) {
    const int m_pairs = fp4_gemm_act_tiles(M) / 2, n_tiles = fp4_tiles(V, kFp4Rows);
    size_t most = 0;
    for (int m = m_pairs; m > 0; m = m > kMaxPairs ? kMaxPairs : m - 1) {
        const size_t rows = 2ll * m * kFp4Rows < M ? 2ll * m * kFp4Rows : M;
        const size_t bytes = rows * max_slots(m, n_tiles, pairs_of((long long)m * n_tiles, kMaxPairs)) * kParts * sizeof(RestState);
        most = bytes > most ? bytes : most;
    }
    return most;
}

ee_status fp4_gemm_launch(const Fp4Head& q, int group, void* parts, int device, cudaStream_t stream) {
    GemmParams p;
    p.q = q;
    p.parts = static_cast<RestState*>(parts);
    p.m_pairs = fp4_gemm_act_tiles(q.M) / 2;
    p.n_tiles = fp4_tiles(q.V, kFp4Rows);
    return group == 16 ? launch_group<16>(p, device, stream) : launch_group<32>(p, device, stream);
}

}  // namespace ee
