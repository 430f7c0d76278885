// A head in 4 bits on the 5th-generation tensor cores.
//
// One CTA per SM takes an equal share of W's 16-row tiles -- at V = 50304 on 148 SMs 21 or 22 of them -- and walks the width
// once, 64 columns at a time.  The weights are the M operand, in tensor memory: 24 warps unpack one tile each, straight into the
// rows of three 128-row operands (tcgen05.st in the order of a matrix fragment, which is the order the packed form is laid out
// in), so unpacked weights touch neither shared memory nor its bandwidth.  The tokens are the N operand, in shared memory (TMA,
// up to 64 rows; a stage is read by three products).  (With the tokens as M and the weights written to shared memory as N, the
// products read 78 KB of shared memory per 64 columns and waited for that.)  The fragment order permutes the columns of every 64; y
// is written in the same order.  The packed blocks come in bulk copies, four at a time per warp, into a ring of its own.
//
// The tensor core truncates rather than rounds what falls below the last bit of its accumulator, which adds up over a row: summed
// in one go over d = 2176 an entropy was off by 3e-5 of itself where fp32 is off by 3e-7.  So an accumulator holds 256 columns at a
// time, and the unpacking warps add it to fp32 sums in their registers, two blocks after its last one was unpacked, when its products
// have long ended.
//
// Then the CTA's logits go through shared memory, so that a thread has one token and some of the rows, and its states to the
// CTA that finishes last.  A share of more than 24 tiles -- on 148 SMs, a vocabulary above 56832 -- goes in several passes, each with its
// own walk over y and its own softmax (64 rows of 1024: 29.4 us at V = 56832, 39.8 at 56833, 48.9 at 113664, 62.5 at 128256: a pass
// costs some 10 us beside its weights; more tiles in one would need more rows of tensor memory); more than 64 tokens in several launches.
//
// 28 us for 64 rows of 1024 against V = 50304 (27 MB packed), 50 us for 33 of 2560 (66 MB, 1.3 TB/s), 17 to 64 rows within 10 % of
// each other.  Issue slots bound it: two thirds of all cycles issue an instruction, half of those to unpack (four per two weights), the
// others to hand blocks from one role to the next and to add the segments.  Timed in copies with a part left out, a block of
// 64 columns took 0.73 us without the unpacking arithmetic, 0.82 without the sums, 0.83 with a quarter of the products, 0.56 without
// all three, of 0.9.  Handing two blocks over at a time changed nothing (28.4 us), nor did handing over after the next block's arithmetic (30.9
// where 30.1 was the rule).
#include "q4_common.cuh"
#include "kernels.h"
#include "sm100_operands.cuh"
#include "gemm_roles.cuh"
#include "tensor_map.h"

namespace ee {

namespace {

constexpr int kUnpackWarps = 24;                 // warp w unpacks rows 16 (w / 4 % 2) + 32 (w % 4) of operand w / 8
constexpr int kOperands = 3;                     // of 128 rows, each with eight unpacking warps and a product warp
constexpr int kTmaWarp = kUnpackWarps, kProductWarp = kUnpackWarps + 1;
constexpr int kThreads = (kUnpackWarps + 1 + kOperands) * 32;
constexpr int kWorkers = kUnpackWarps * 32;      // threads of the softmax
constexpr int kMaxTiles = 24;
constexpr int kWStages = 3;                      // of 3 x 32 columns of tensor memory
constexpr int kYStages = 8;                      // of N x 128 bytes of shared memory
constexpr int kSegment = 4;                      // blocks of 64 columns an accumulator sums
constexpr int kLag = 2;                          // blocks unpacked between a segment's last one and its reading: fewer than kWStages, or nobody moves
constexpr int kRawBlocks = 4;                    // packed blocks per bulk copy
static_assert(kRawBlocks == kSegment, "a copy is a segment");
constexpr int kRawBytes = kRawBlocks * 512 + 256;      // ... and their scales, up to eight groups
constexpr int kAccCols = 192;
constexpr int kTmemCols = 512;
constexpr size_t kSmemBudget = 226 * 1024;

struct GemmParams {
    Q4Params q;
    int passes;                                  // of every CTA
    int group_shift;                             // log2 of the scales' group
};

// Barriers: per operand the ring of unpacked weights and the accumulators, the ring of y, per unpacking warp the ring of packed blocks.
constexpr int kWBars = kOperands * kWStages, kAccBars = kOperands * 4, kRawBars = kUnpackWarps * 2;
constexpr int kBarBytes = 8 * (2 * kWBars + 2 * kAccBars + 2 * kYStages + kRawBars + kOperands) + 64;
size_t big_bytes(int n) {                         // the rings of packed blocks, and afterwards the logits
    const size_t z = (size_t)kMaxTiles * 16 * (n + 4) * sizeof(float), raw = (size_t)kUnpackWarps * 2 * kRawBytes;
    return ((z > raw ? z : raw) + 127) / 128 * 128;
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

template <int N>                                  // tokens, padded: 16, 32 or 64
__global__ void __launch_bounds__(kThreads, 1) q4_gemm_kernel(const __grid_constant__ CUtensorMap map_y, const GemmParams p, const int big) {
    constexpr int kSets = kAccCols / (kOperands * N);                    // accumulators: 4, 2 or 1
    constexpr int y_bytes = N * 128;
    const Q4Params& q = p.q;
    const Q4Layout l = q4_layout(q.V, q.d, q.group);
    const int t_begin = (int)((long long)blockIdx.x * l.tiles / gridDim.x), t_end = (int)((long long)(blockIdx.x + 1) * l.tiles / gridDim.x);
    const int nt = (t_end - t_begin + p.passes - 1) / p.passes;          // tiles of a pass (the last of several may have fewer)
    const int operands = (nt + 7) / 8;
    const int segments = (l.blocks + kSegment - 1) / kSegment;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw_addr = ptx::smem_addr(smem_raw);
    unsigned char* smem = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
    const uint32_t y_base = ptx::smem_addr(smem);
    unsigned char* big_mem = smem + kYStages * y_bytes;
    float* z_mem = reinterpret_cast<float*>(big_mem);                    // [rows][N + 4]
    RestState* states = reinterpret_cast<RestState*>(big_mem + big);             // [kWorkers / N][N]
    unsigned char* bar_mem = reinterpret_cast<unsigned char*>(states + kWorkers);
    const uint32_t bar_base = ptx::smem_addr(bar_mem);
    auto wfull_bar = [&](int o, int s) { return bar_base + 8u * (o * kWStages + s); };
    auto wempty_bar = [&](int o, int s) { return bar_base + 8u * (kWBars + o * kWStages + s); };
    auto accfull_bar = [&](int o, int s) { return bar_base + 8u * (2 * kWBars + o * 4 + s); };
    auto accfree_bar = [&](int o, int s) { return bar_base + 8u * (2 * kWBars + kAccBars + o * 4 + s); };
    const uint32_t y_bars = bar_base + 8u * (2 * kWBars + 2 * kAccBars);
    auto yfull_bar = [&](int s) { return y_bars + 8u * s; };
    auto yempty_bar = [&](int s) { return y_bars + 8u * (kYStages + s); };
    auto raw_bar = [&](int w, int s) { return y_bars + 8u * (2 * kYStages + 2 * w + s); };
    auto drain_bar = [&](int o) { return y_bars + 8u * (2 * kYStages + kRawBars + o); };
    volatile uint32_t* tmem_holder = reinterpret_cast<volatile uint32_t*>(bar_mem + kBarBytes - 64);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
    volatile int* is_last = abort_flag + 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    launch_dependents();
    if (threadIdx.x == 0) {
        for (int o = 0; o < kOperands; ++o) {
            for (int s = 0; s < kWStages; ++s) {
                ptx::mbar_init(wfull_bar(o, s), max(1, min(8, nt - 8 * o)));
                ptx::mbar_init(wempty_bar(o, s), 1);
            }
            for (int s = 0; s < 4; ++s) {
                ptx::mbar_init(accfull_bar(o, s), 1);
                ptx::mbar_init(accfree_bar(o, s), 8);
            }
            ptx::mbar_init(drain_bar(o), 1);
        }
        for (int s = 0; s < kYStages; ++s) {
            ptx::mbar_init(yfull_bar(s), 1);
            ptx::mbar_init(yempty_bar(s), operands);
        }
        for (int w = 0; w < kUnpackWarps; ++w)
            for (int s = 0; s < 2; ++s) ptx::mbar_init(raw_bar(w, s), 1);
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

    // unpacking: a warp keeps its tile of a pass from block to block
    const int quarter = warp & 3;
    const int slot = warp < kUnpackWarps ? (warp >> 3) * 8 + 2 * quarter + ((warp >> 2) & 1) : kMaxTiles;       // which of the pass's tiles
    const bool unpacks = slot < nt;
    const int g = lane >> 2, c = lane & 3;
    unsigned char* raw_mem = big_mem + warp * 2 * kRawBytes;             // this warp's two slots
    // four blocks of the warp's tile and their scales from block kb0 on (one lane)
    auto fetch = [&](int tile, int kb0, int s) {
        const int n = min(kRawBlocks, l.blocks - kb0);
        const int g0 = (kb0 * 64) >> p.group_shift, g1 = ((kb0 + n) * 64 - 1) >> p.group_shift;
        const uint32_t dst = ptx::smem_addr(raw_mem + s * kRawBytes), scale_bytes = (uint32_t)(g1 - g0 + 1) * 32u;
        ptx::mbar_arrive_expect_tx(raw_bar(warp, s), n * 512u + scale_bytes);
        bulk_load(dst, q.weights + ((size_t)tile * l.blocks + kb0) * 32, n * 512u, raw_bar(warp, s));
        bulk_load(dst + kRawBlocks * 512, q.scales + ((size_t)tile * l.groups + g0) * 8, scale_bytes, raw_bar(warp, s));
    };
    // sums: warp = 32 rows of operand (w / 4) % 3, half (w / 12) of the tokens
    const int my_op = (warp >> 2) % 3, my_half = warp / 12;
    const bool sums = warp < kUnpackWarps && my_op < operands;
    const uint32_t acc_from = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(my_op * N + my_half * (N / 2));

    // softmax: thread = one token and every `shares`-th row
    constexpr int shares = kWorkers / N;
    const int tok = threadIdx.x & (N - 1), share = threadIdx.x / N;
    if (threadIdx.x < kWorkers) states[share * N + tok] = rest_empty();          // in shared memory: the loop needs its registers
    bool ok = true;                                                      // of this warp's role
    for (int pass = 0; pass < p.passes; ++pass) {
        const int seg0 = pass * segments;                                // segments before this pass, for the accumulators' parities
        int ws = pass * l.blocks % kWStages, ys = pass * l.blocks % kYStages;              // ring positions and their parities
        uint32_t wp = pass * l.blocks / kWStages & 1, yp = pass * l.blocks / kYStages & 1;
        float z[N / 2];
#pragma unroll
        for (int j = 0; j < N / 2; ++j) z[j] = 0.f;
        if (warp == kTmaWarp) {
            // ---------------------------------------------------------------- y
            if (lane == 0) {
                uint32_t armed = 0, armed_parity = 0;                    // of this pass: the loads of the one before were all waited for
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
            // about 75 cycles, whatever its size; twelve of them a block by one thread were what the kernel waited for)
            const int o = warp - kProductWarp;
            if (lane == 0 && o < operands) {
                constexpr uint32_t idesc = ptx::idesc_bf16_f32(128, N);
                for (int seg = 0; ok && seg < segments; ++seg) {
                    const int set = (seg0 + seg) % kSets, use = (seg0 + seg) / kSets;
                    if (use > 0 && !ptx::mbar_wait(accfree_bar(o, set), (uint32_t)(use - 1) & 1u, abort_flag)) {
                        record_failure(q.ctrl, abort_flag, 2, 0x80 | set, seg);
                        ok = false;
                        break;
                    }
                    const uint32_t acc = tmem_base + (set * kOperands + o) * N;
                    for (int kb = seg * kSegment; kb < min(l.blocks, (seg + 1) * kSegment); ++kb) {
                        if (!ptx::mbar_wait(yfull_bar(ys), yp, abort_flag) || !ptx::mbar_wait(wfull_bar(o, ws), wp, abort_flag)) {
                            record_failure(q.ctrl, abort_flag, 2, ws, kb);
                            ok = false;
                            break;
                        }
                        ptx::tc_fence_after_sync();
                        const uint64_t bdesc = ptx::smem_desc_k128(y_base + ys * y_bytes);
                        const uint32_t a = ring + ws * 96 + o * 32;
#pragma unroll
                        for (int k = 0; k < 4; ++k) ptx::mma_bf16_ts(acc, a + k * 8, bdesc + 2u * k, idesc, (kb > seg * kSegment || k > 0) ? 1u : 0u);
                        ptx::mma_commit(wempty_bar(o, ws));
                        ptx::mma_commit(yempty_bar(ys));
                        if (++ws == kWStages) { ws = 0; wp ^= 1u; }
                        if (++ys == kYStages) { ys = 0; yp ^= 1u; }
                    }
                    if (ok) ptx::mma_commit(accfull_bar(o, set));
                }
                if (*abort_flag) mma_drain<false>(drain_bar(o));
            }
            __syncwarp();
        } else {
            // ---------------------------------------------------------------- unpacking and sums
            const int o = warp >> 3;
            const uint32_t to = ring + (uint32_t)o * 32u + ((uint32_t)(quarter * 32 + ((warp >> 2) & 1) * 16) << 16);
            const int tile = min(t_begin + pass * nt + slot, t_end - 1);
            int fetched = 0;                                             // copies issued, four blocks each
            if (unpacks && ok && lane == 0) {
                if (pass > 0) ptx::fence_proxy_async();                  // the logits of the pass before lay here
                fetch(tile, 0, 0);
                if (kRawBlocks < l.blocks) fetch(tile, kRawBlocks, 1);
            }
            if (unpacks && ok) fetched = kRawBlocks < l.blocks ? 2 : 1;
            const uint32_t raw0 = (uint32_t)(pass * ((segments + 1) >> 1)), raw1 = (uint32_t)(pass * (segments >> 1));     // copies before, by slot
            // segments, and one turn more for adding the last; unrolled, so that what depends on a block's place in its segment is constant
            for (int seg = 0; ok && seg <= segments; ++seg) {
#pragma unroll
                for (int i = 0; i < kSegment; ++i) {
                    const int kb = seg * kSegment + i;
                    if (unpacks && kb < l.blocks) {
                        const int s = seg & 1;
                        if (i == 0 && !__all_sync(0xffffffffu, ptx::mbar_wait(raw_bar(warp, s), ((s ? raw1 : raw0) + (uint32_t)(seg >> 1)) & 1u, abort_flag))) {
                            if (lane == 0) record_failure(q.ctrl, abort_flag, 4, s, kb);
                            ok = false;
                            break;
                        }
                        const unsigned char* raw = raw_mem + s * kRawBytes;
                        const uint4 w = *reinterpret_cast<const uint4*>(raw + i * 512 + lane * 16);
                        const int group = (i * 64 + c * 16) >> p.group_shift;                // a copy begins with a group: 256 columns
                        const uint32_t s2 = *reinterpret_cast<const uint32_t*>(raw + kRawBlocks * 512 + group * 32 + g * 4);
                        const uint32_t sl = low_twice(s2), sh = high_twice(s2);
                        uint32_t v[16];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {                        // pair k of the lane's eight, rows g and g + 8
                            v[(k >> 1) * 4 + (k & 1)] = q4_pair(k < 4 ? w.x : w.y, k & 3, sl);
                            v[(k >> 1) * 4 + 2 + (k & 1)] = q4_pair(k < 4 ? w.z : w.w, k & 3, sh);
                        }
                        if (i == kRawBlocks - 1) {                           // the slot is read: the blocks after the next four
                            __syncwarp();
                            const int kb0 = kb + 1 + kRawBlocks;
                            if (kb0 < l.blocks) {
                                if (lane == 0) fetch(tile, kb0, s);
                                ++fetched;
                            }
                        }
                        if (!__all_sync(0xffffffffu, ptx::mbar_wait(wempty_bar(o, ws), wp ^ 1u, abort_flag))) {
                            if (lane == 0) record_failure(q.ctrl, abort_flag, 4, 0x40 | ws, kb);
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
                    if (i == kLag - 1 && seg > 0 && sums) {                  // the segment before
                        const int set = (seg0 + seg - 1) % kSets, use = (seg0 + seg - 1) / kSets;
                        if (!__all_sync(0xffffffffu, ptx::mbar_wait(accfull_bar(my_op, set), (uint32_t)use & 1u, abort_flag))) {
                            if (lane == 0) record_failure(q.ctrl, abort_flag, 3, set, seg - 1);
                            ok = false;
                            break;
                        }
                        ptx::tc_fence_after_sync();
#pragma unroll
                        for (int b = 0; b < N / 2; b += 8) {
                            float x[8];
                            ptx::tmem_ld_32x8(acc_from + set * kOperands * N + b, x);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 8; j += 2) {
                                const float2 sum = ptx::unpack_f32x2(ptx::add_f32x2(ptx::pack_f32x2(z[b + j], z[b + j + 1]), ptx::pack_f32x2(x[j], x[j + 1])));
                                z[b + j] = sum.x;
                                z[b + j + 1] = sum.y;
                            }
                        }
                        ptx::tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(accfree_bar(my_op, set));
                    }
                }
            }
            if (unpacks && !ok && lane == 0) {                           // let the copies in flight land before the CTA ends
                for (int k = max(0, fetched - 2); k < fetched; ++k)
                    for (uint32_t i = 0; i < (1u << 16) && !ptx::mbar_try_wait(raw_bar(warp, k & 1), ((k & 1 ? raw1 : raw0) + (uint32_t)(k >> 1)) & 1u); ++i)
                        __nanosleep(100);
            }
        }
        // -------------------------------------------------------------------- logits to shared memory: rows x tokens
        if (pass == 0 && warp != kTmaWarp) grid_dependency_wait();
        __syncthreads();                                                 // the packed blocks, which lay here, are all read
        const int first = t_begin + pass * nt;
        const int rows = min(min(nt, t_end - first) * 16, q.V - first * 16);      // of this pass that exist
        if (sums) {
            const int r0 = my_op * 128 + quarter * 32;
            float* out = z_mem + (size_t)(r0 + lane) * (N + 4) + my_half * (N / 2);
            if (r0 < rows) {
#pragma unroll
                for (int b = 0; b < N / 2; b += 4) *reinterpret_cast<float4*>(out + b) = make_float4(z[b], z[b + 1], z[b + 2], z[b + 3]);
            }
        }
        __syncthreads();
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
                const bool top = x == m && idx == 0x7fffffff;            // the largest term stays out of the sum
                s += top ? 0.f : e;
                t = fmaf(e, dz, t);
                idx = top ? r : idx;
            }
            RestState st = states[share * N + tok];
            rest_merge(st, RestState{m, s, t, idx == 0x7fffffff ? idx : first * 16 + idx});
            states[share * N + tok] = st;
        }
        if (pass + 1 < p.passes) __syncthreads();                        // z is read before the next pass writes it
    }

    auto column = [&](int token) { return rest_combine(shares, [&](int k) -> const RestState& { return states[k * N + token]; }); };
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == kProductWarp) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem_base, kTmemCols);
    }
    if ((int)threadIdx.x < q.M) q.parts[(size_t)blockIdx.x * N + threadIdx.x] = column(threadIdx.x);
    __syncthreads();
    if (threadIdx.x == 0) *is_last = ticket_arrive_is_last(&q.ctrl->head_ticket[0], gridDim.x) ? 1 : 0;
    __syncthreads();
    if (!*is_last) return;
    // the CTAs' states: lane = token, eight CTAs at a time in flight per thread, then as above
    if (threadIdx.x < kWorkers) {
        RestState s = rest_empty();
        if (tok < q.M)
            for (int b0 = share; b0 < (int)gridDim.x; b0 += 8 * shares) {
                RestState v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int b = b0 + i * shares;
                    v[i] = b < (int)gridDim.x ? rest_load_cg(q.parts + (size_t)b * N + tok) : rest_empty();
                }
                rest_merge(s, rest_combine(8, [&](int k) -> const RestState& { return v[k]; }));
            }
        states[share * N + tok] = s;
    }
    __syncthreads();
    if ((int)threadIdx.x < q.M)
        rest_finish(column(threadIdx.x), q, threadIdx.x);
    if (threadIdx.x == 0) q.ctrl->head_ticket[0] = 0;                    // ready for the next launch
}

template <int N>
ee_status launch_tokens(const Q4Params& q, int num_sms, int device, cudaStream_t stream) {
    static bool configured[kMaxDevices] = {};
    if (!configured[device]) {
        if (cudaFuncSetAttribute(q4_gemm_kernel<N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBudget) != cudaSuccess) return EE_ERR_CUDA;
        configured[device] = true;
    }
    const Q4Layout l = q4_layout(q.V, q.d, q.group);
    GemmParams p;
    p.q = q;
    int grid = l.tiles < num_sms ? l.tiles : num_sms;
    if (grid > kStreamMaxCtas) grid = kStreamMaxCtas;
    const int most = (l.tiles + grid - 1) / grid;                        // tiles of the largest share
    p.passes = (most + kMaxTiles - 1) / kMaxTiles;
    p.group_shift = q.group == 32 ? 5 : q.group == 64 ? 6 : 7;
    const size_t smem = (size_t)kYStages * N * 128 + big_bytes(N) + kWorkers * sizeof(RestState) + kBarBytes + 1024;
    CUtensorMap map;
    if (!make_tile_map(&map, q.y, q.M, l.blocks * 64, N)) return EE_ERR_CUDA;
    return launch_pdl(q4_gemm_kernel<N>, dim3(grid), kThreads, smem, stream, map, p, (int)big_bytes(N)) == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

}  // namespace

ee_status q4_gemm_launch(const Q4Params& q, int num_sms, int device, cudaStream_t stream) {
    return q.M <= 16 ? launch_tokens<16>(q, num_sms, device, stream) : q.M <= 32 ? launch_tokens<32>(q, num_sms, device, stream)
                                                                                 : launch_tokens<64>(q, num_sms, device, stream);
}

}  // namespace ee
