// Exit heads whose weights are held in 4 bits: whole numbers q = -8 .. 7 with one bf16 scale s per row and group of 32, 64
// or 128 columns.  What they stand for is w = bf16(s q); the head itself is that of ee_exit_head (LayerNorm, projection,
// entropy, argmax, decision) with these weights.  Drafting reads the whole head for a handful of tokens, so a call's time
// is the time of that read: 4.25 bits per weight at a group of 64 instead of 16.
//
// The product with the scale is rounded to bf16 because the tensor cores take bf16 operands; it is part of the
// definition (ee_head_q4_unpack returns the same values), so nothing is lost between the two.
//
// The packed layout (q4_common.cuh) is the operand of four m16n8k16 products per block of 64 columns if the contraction is walked
// in the order "lane c: columns 16c + 4s .. 16c + 4s + 3 in step s", which costs nothing as long as the other operand is read
// in the same order: a lane's share of y is then 32 consecutive bytes as well.
#include "q4_common.cuh"
#include "layer_norm.cuh"
#include "kernels.h"

namespace ee {

namespace {

constexpr int kWarps = 24;                       // as many as leave a thread 80 registers: a warp's loads are what is in flight
constexpr int kThreads = kWarps * 32;
constexpr int kUnroll = 2;                       // blocks (512 bytes of a tile) in flight per warp, twice
constexpr size_t kSmemBudget = 226 * 1024;

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// ---------------------------------------------------------------------------------------------------- writing and reading

// 32 bytes with one access: the 16 columns a lane owns are a whole sector, where two 16-byte accesses would each move half of
// every sector they touch (packing + unpacking at d = 2048, V = 50304: 242 us with two, 94 us with one: 5.5 TB/s).
struct Sector { uint32_t w[8]; };
__device__ __forceinline__ Sector ld_sector(const void* p) {
    Sector s;
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(s.w[0]), "=r"(s.w[1]), "=r"(s.w[2]), "=r"(s.w[3]), "=r"(s.w[4]), "=r"(s.w[5]), "=r"(s.w[6]), "=r"(s.w[7]) : "l"(p));
    return s;
}
__device__ __forceinline__ void st_sector(void* p, const Sector& s) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(s.w[0]), "r"(s.w[1]), "r"(s.w[2]), "r"(s.w[3]), "r"(s.w[4]), "r"(s.w[5]), "r"(s.w[6]), "r"(s.w[7]) : "memory");
}

__device__ __forceinline__ float amax16(const Sector& v) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fmaxf(fabsf(bf16_lo(v.w[i])), fabsf(bf16_hi(v.w[i]))));
    return m;
}

// q + 8 of one weight, q = nearest whole number of x / s, ties to the even one; r = 1 / s.  A quotient of two numbers of eight
// significant bits and at most 8 in magnitude is either exactly a whole number and a half or at least 2^-11 away from one,
// while x r is off by less than 2^-20: rounded to the grid of 2^-13 first, it is a tie exactly where the quotient is.
__device__ __forceinline__ uint32_t q4_fast(float x, float r) {
    const float snapped = __fadd_rn(__fadd_rn(__fmul_rn(x, r), 1536.f), -1536.f);
    return __float_as_uint(__fadd_rn(snapped, 12582912.f + 8.f)) & 15u;          // 1.5 * 2^23: the low bits are the whole number
}
__device__ __forceinline__ uint32_t q4_slow(float x, float s) {                    // scales next to or below the smallest normal number
    return (uint32_t)(max(-8, min(7, __float2int_rn(__fdiv_rn(x, s)))) + 8);
}
// Words [i] = columns 8i .. 8i + 7 of the lane's sixteen.
__device__ __forceinline__ uint2 q4_words(const Sector& v, float s) {
    if (!(s > 0.f)) return make_uint2(0x88888888u, 0x88888888u);
    uint32_t w[2] = {0, 0};
    if (s >= 1e-30f) {
        const float r = __frcp_rn(s);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i >> 2] |= (q4_fast(bf16_lo(v.w[i]), r) << (4 * (i & 3))) | (q4_fast(bf16_hi(v.w[i]), r) << (4 * (i & 3) + 16));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i >> 2] |= (q4_slow(bf16_lo(v.w[i]), s) << (4 * (i & 3))) | (q4_slow(bf16_hi(v.w[i]), s) << (4 * (i & 3) + 16));
    }
    return make_uint2(w[0], w[1]);
}

// A warp per 16 rows x 128 columns (two blocks, so that a group of 128 lies inside).  An ordinary launch, here and below: the
// weights may just have been written, and 32-byte loads take the L1.
__global__ void __launch_bounds__(256) q4_pack_kernel(const __nv_bfloat16* W, int V, int d, int group, uint4* weights, uint32_t* scales) {
    const Q4Layout l = q4_layout(V, d, group);
    const int pairs = (l.blocks + 1) / 2;
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (unit >= (long long)l.tiles * pairs) return;
    const int tile = (int)(unit / pairs), b0 = 2 * (int)(unit % pairs);
    Sector v[2][2];                                // [block][row g, row g + 8]
    float m[2][2];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int row = tile * 16 + g + 8 * r, col = (b0 + b) * 64 + c * 16;
            v[b][r] = Sector{};
            if (row < V && col < d) v[b][r] = ld_sector(W + (size_t)row * d + col);      // d is a multiple of 32: a whole sector
        }
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            m[b][r] = amax16(v[b][r]);
            m[b][r] = fmaxf(m[b][r], __shfl_xor_sync(0xffffffffu, m[b][r], 1));
            if (group >= 64) m[b][r] = fmaxf(m[b][r], __shfl_xor_sync(0xffffffffu, m[b][r], 2));
        }
#pragma unroll
    for (int r = 0; r < 2; ++r)
        if (group == 128) m[0][r] = m[1][r] = fmaxf(m[0][r], m[1][r]);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        if (b0 + b >= l.blocks) break;
        const uint32_t s2 = pack_bf16(__fdiv_rn(m[b][0], 7.f), __fdiv_rn(m[b][1], 7.f));
        const uint2 wg = q4_words(v[b][0], bf16_lo(s2)), wh = q4_words(v[b][1], bf16_hi(s2));
        weights[((size_t)tile * l.blocks + b0 + b) * 32 + lane] = make_uint4(wg.x, wg.y, wh.x, wh.y);
        const int col = (b0 + b) * 64 + c * 16;
        if (col % group == 0) scales[((size_t)tile * l.groups + col / group) * 8 + g] = s2;
    }
}

// A warp per 16 rows x 64 columns.
__global__ void __launch_bounds__(256) q4_unpack_kernel(const uint4* weights, const uint32_t* scales, int V, int d, int group, __nv_bfloat16* W) {
    const Q4Layout l = q4_layout(V, d, group);
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (unit >= (long long)l.tiles * l.blocks) return;
    const int tile = (int)(unit / l.blocks), b = (int)(unit % l.blocks);
    const int col = b * 64 + c * 16;
    const uint4 w = weights[unit * 32 + lane];
    const uint32_t s2 = scales[((size_t)tile * l.groups + col / group) * 8 + g];
    const uint32_t words[2][2] = {{w.x, w.y}, {w.z, w.w}};
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = tile * 16 + g + 8 * r;
        const uint32_t s = r ? high_twice(s2) : low_twice(s2);
        Sector o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.w[i] = q4_pair(words[r][i >> 2], i & 3, s);
        if (row < V && col < d) st_sector(W + (size_t)row * d + col, o);
    }
}

// ---------------------------------------------------------------------------------------------------- the head

// Bytes between two rows of y in shared memory: 16 more than a multiple of 128, so that the eight lanes of a 16-byte access
// (two rows, four columns 32 bytes apart) touch every bank once.
__host__ __device__ inline int y_row_bytes(int d) { return (d + 63) / 64 * 128 + 16; }

// Up to NT * 8 rows, one launch: the rows are normalised by every CTA into its shared memory while the first weights are on
// their way; a warp takes a 16-row tile of W at a time, streams it through registers and multiplies it with all rows of y; the
// CTA's tiles are folded into one softmax state per row, and the CTA that finishes last merges the CTAs' states and decides.
//
// V = 50304, group 64, one call after the other: 16.8 us for 1 row of 1024 (27 MB of weights), 17.9 for 8, 21.9 for 16; 12.0 for 8
// rows of 512; 28.8 for 1 and 31.6 for 8 of 2560 (2.2 TB/s); the first weights ahead of the wait for the stream's earlier work,
// which may be what writes them, would take 0.1 to 0.7 us off.  Unpacking bounds it: a 64-column block takes a warp some 110
// instructions, half of them in the pipe that issues every other cycle, 150 cycles of its scheduler; start, LayerNorm and merge are
// 8 us beside that.  A ring of eight blocks per warp in shared memory, filled by asynchronous copies, was no faster (31.7 us
// for 8 rows of 2560, 13.0 for 8 of 512): what is in flight is not what it waits for.
// What one launch takes goes to this kernel, 16 rows or the 8 that fit shared memory at d > 6784, more to the tensor-core one, which
// reads the weights once: 16 rows of 1024 take 21.9 us here and 25.5 there, 17 rows (two
// passes here) 38 and 26.7; at d = 2560 42 and 46, then 77 and 48.5;
// at d = 8192 8 rows 87 and 120, 16 rows (two passes) 173 and 120.
template <int NT>
__global__ void __launch_bounds__(kThreads, 1) q4_head_kernel(const __grid_constant__ Q4Params p) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int is_last;
    __shared__ double2 sums[kWarps];
    const Q4Layout l = q4_layout(p.V, p.d, p.group);
    const int group_shift = 31 - __clz(p.group);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int ld = y_row_bytes(p.d);
    RestState* states = reinterpret_cast<RestState*>(smem + NT * 8 * ld);        // [kWarps][max(NT * 8, 32)]: per warp, then scratch of the merge
    launch_dependents();

    uint4 w[kUnroll];
    uint32_t sc[kUnroll];
    auto load = [&](int tile, int b0) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (b0 + u < l.blocks) {
                w[u] = ld_dep(p.weights + ((size_t)tile * l.blocks + b0 + u) * 32 + lane);
                sc[u] = ld_dep(p.scales + ((size_t)tile * l.groups + (((b0 + u) * 64 + c * 16) >> group_shift)) * 8 + g);
            }
    };
    int tile = blockIdx.x + gridDim.x * warp;
    grid_dependency_wait();                                              // the weights may just have been packed, gamma and beta learned
    if (tile < l.tiles) load(tile, 0);                                   // in flight beside the LayerNorm
    {
        // the LayerNorm, above 1024 columns with every warp taking part, kWarps / M of them to a row (M <= 16): 8 rows of 2560 take
        // 31.5 us instead of 35; up to 1024 a warp per row, without the barriers: 8 rows of 512 take 11.8 us instead of 13.4
        const int nvec = p.d >> 3, width = l.blocks * 8, per_row = nvec > 128 ? kWarps / p.M : 1;
        const int row = warp / per_row, first = (warp - row * per_row) * 32 + lane, step = per_row * 32;
        const bool live = row < p.M;
        const uint4* hrow = reinterpret_cast<const uint4*>(p.h + (size_t)(live ? row : 0) * p.ld_h);
        const double d = (double)p.d, inv_d = 1.0 / d;
        auto row_sum2 = [&](double& s, double& q) {                      // in a fixed order, the same bits in every warp of the row
            warp_sum2_d(s, q);
            if (per_row == 1) return;
            if (lane == 0) sums[warp] = make_double2(s, q);
            __syncthreads();
            s = q = 0.0;
            if (live)
                for (int i = 0; i < per_row; ++i) {
                    const double2 o = sums[row * per_row + i];
                    s += o.x;
                    q += o.y;
                }
        };
        Moments m;
        m.clear();
        if (live)
            for (int k = first, j = 0; k < nvec; k += step, ++j) m.add(ld_dep(hrow + k), j);
        double s = m.sum(), q = m.sum_sq(), mu = 0.0, var = 0.0;
        row_sum2(s, q);
        const bool again = live && !row_variance_one_pass(s, q, d, inv_d, mu, var);
        if (per_row == 1 ? again : __syncthreads_or(again)) {
            double v0 = 0.0, v1 = 0.0;
            if (again)
                for (int k = first; k < nvec; k += step) vec8_sqdev_d(ld_dep(hrow + k), mu, v0, v1);
            double v = v0 + v1, none = 0.0;
            row_sum2(v, none);
            if (again) var = v * inv_d;
        }
        if (live) {
            uint4* yrow = reinterpret_cast<uint4*>(smem + row * ld);
            const RowStats st = row_stats(mu, var, p.ln_eps);
            for (int k = first; k < nvec; k += step) yrow[k] = layer_norm_vec8<true, true>(ld_dep(hrow + k), st, p.gamma, p.beta, k);
            for (int k = nvec + first; k < width; k += step) yrow[k] = make_uint4(0, 0, 0, 0);
        }
        for (int r = p.M + warp; r < NT * 8; r += kWarps)
            for (int k = lane; k < width; k += 32) reinterpret_cast<uint4*>(smem + r * ld)[k] = make_uint4(0, 0, 0, 0);
    }
    RestState* mine = states + warp * (NT * 8);
    for (int i = lane; i < NT * 8; i += 32) mine[i] = rest_empty();
    __syncthreads();

    const unsigned char* ybase = smem + g * ld + c * 32;
    for (; tile < l.tiles; tile += gridDim.x * kWarps) {
        float acc[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.f;
#pragma unroll 1
        for (int b0 = 0; b0 < l.blocks; b0 += kUnroll) {
            uint4 cur[kUnroll];
            uint32_t cs[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) { cur[u] = w[u]; cs[u] = sc[u]; }
            if (b0 + kUnroll < l.blocks) load(tile, b0 + kUnroll);
            else if (tile + gridDim.x * kWarps < l.tiles) load(tile + gridDim.x * kWarps, 0);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (b0 + u < l.blocks) {
                    const uint32_t sg = low_twice(cs[u]), sh = high_twice(cs[u]);
                    const unsigned char* yb = ybase + (b0 + u) * 128;
                    // a block is summed by itself and added in fp32: the tensor core cuts off, rather than rounds, what falls
                    // below the last bit of its accumulator, which over a whole row adds up (M = 1, d = 1024: entropy off by 1.4e-5
                    // of itself when accumulated in one go)
                    float part[NT][4];
#pragma unroll
                    for (int t = 0; t < NT; ++t) part[t][0] = part[t][1] = part[t][2] = part[t][3] = 0.f;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {                        // steps 2e and 2e + 1: eight columns of each lane
                        const uint32_t wg = e ? cur[u].y : cur[u].x, wh = e ? cur[u].w : cur[u].z;
                        uint32_t a[2][4];
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            a[s][0] = q4_pair(wg, 2 * s, sg);
                            a[s][1] = q4_pair(wh, 2 * s, sh);
                            a[s][2] = q4_pair(wg, 2 * s + 1, sg);
                            a[s][3] = q4_pair(wh, 2 * s + 1, sh);
                        }
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            const uint4 y = *reinterpret_cast<const uint4*>(yb + t * 8 * ld + e * 16);
                            mma_16816(part[t], a[0][0], a[0][1], a[0][2], a[0][3], y.x, y.y);
                            mma_16816(part[t], a[1][0], a[1][1], a[1][2], a[1][3], y.z, y.w);
                        }
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[t][j] += part[t][j];
                }
            }
        }
        const int v = tile * 16 + g;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {                                // token 2c + j of the eight: rows g and g + 8, then over g
                RestState s = rest_empty();
                if (v < p.V) rest_push(s, acc[t][j], v);
                if (v + 8 < p.V) rest_push(s, acc[t][2 + j], v + 8);
                s = rest_reduce_lanes<4>(s);
                if (g == 0) {
                    RestState o = mine[t * 8 + 2 * c + j];
                    rest_merge(o, s);
                    mine[t * 8 + 2 * c + j] = o;
                }
            }
    }
    __syncthreads();
    for (int tok = warp; tok < p.M; tok += kWarps) {                      // the warps' states of a row, one per lane
        const RestState s = rest_reduce_lanes<1>(lane < kWarps ? states[lane * (NT * 8) + tok] : rest_empty());
        if (lane == 0) p.parts[(size_t)blockIdx.x * (NT * 8) + tok] = s;
    }
    __syncthreads();
    if (threadIdx.x == 0) is_last = ticket_arrive_is_last(&p.ctrl->head_ticket[0], gridDim.x) ? 1 : 0;
    __syncthreads();
    if (!is_last) return;
    for (int tok = warp; tok < p.M; tok += kWarps) {                      // the CTAs' states, up to eight per lane
        RestState v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = lane + 32 * i < (int)gridDim.x ? rest_load_cg(p.parts + (size_t)(lane + 32 * i) * (NT * 8) + tok) : rest_empty();
        const RestState s = rest_reduce_lanes<1>(rest_combine(8, [&](int k) -> const RestState& { return v[k]; }));
        if (lane == 0) rest_finish(s, p, tok);
    }
    if (threadIdx.x == 0) p.ctrl->head_ticket[0] = 0;                    // ready for the next launch
}

size_t q4_smem(int nt, int d) { return (size_t)nt * 8 * y_row_bytes(d) + (size_t)kWarps * (nt * 8 > 32 ? nt * 8 : 32) * sizeof(RestState); }

// Rows one launch takes: sixteen, or eight where sixteen do not fit shared memory.
int slab_rows(int d) { return q4_smem(2, d) <= kSmemBudget ? 16 : 8; }

template <int NT>
ee_status launch_head(const Q4Params& p, int num_sms, int device, cudaStream_t stream) {
    static bool configured[kMaxDevices] = {};
    if (!configured[device]) {
        if (cudaFuncSetAttribute(q4_head_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBudget) != cudaSuccess) return EE_ERR_CUDA;
        configured[device] = true;
    }
    const int tiles = (p.V + 15) / 16;
    int grid = tiles < num_sms ? tiles : num_sms;
    if (grid > kStreamMaxCtas) grid = kStreamMaxCtas;
    return launch_pdl(q4_head_kernel<NT>, dim3(grid), kThreads, q4_smem(NT, p.d), stream, p) == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

size_t parts_bytes() { return (size_t)kStreamMaxCtas * kQ4GemmRows * sizeof(RestState); }


}  // namespace

size_t q4_weight_bytes(int V, int d, int group) {
    const Q4Layout l = q4_layout(V, d, group);
    return align_up((size_t)l.tiles * l.blocks * 512, 256) + align_up((size_t)l.tiles * l.groups * 32, 256);
}
static const uint32_t* q4_scales(const void* q4, int V, int d, int group) {
    const Q4Layout l = q4_layout(V, d, group);
    return reinterpret_cast<const uint32_t*>(static_cast<const unsigned char*>(q4) + align_up((size_t)l.tiles * l.blocks * 512, 256));
}

ee_status q4_pack_launch(const void* W, int V, int d, int group, void* q4, cudaStream_t stream) {
    const Q4Layout l = q4_layout(V, d, group);
    const long long units = (long long)l.tiles * ((l.blocks + 1) / 2);
    q4_pack_kernel<<<(unsigned)((units + 7) / 8), 256, 0, stream>>>(static_cast<const __nv_bfloat16*>(W), V, d, group, static_cast<uint4*>(q4),
                                                                    const_cast<uint32_t*>(q4_scales(q4, V, d, group)));
    return cudaGetLastError() == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

ee_status q4_unpack_launch(const void* q4, int V, int d, int group, void* W, cudaStream_t stream) {
    const Q4Layout l = q4_layout(V, d, group);
    const long long units = (long long)l.tiles * l.blocks;
    q4_unpack_kernel<<<(unsigned)((units + 7) / 8), 256, 0, stream>>>(static_cast<const uint4*>(q4), q4_scales(q4, V, d, group), V, d, group,
                                                                      static_cast<__nv_bfloat16*>(W));
    return cudaGetLastError() == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

size_t q4_head_workspace_bytes(int M, int d) { return kCtrlBytes + parts_bytes() + align_up((size_t)M * ((d + 63) / 64) * 128, 256); }

ee_status q4_head_launch(const HeadArgs& a, const void* q4, int group) {
    unsigned char* ws = static_cast<unsigned char*>(a.workspace);
    __nv_bfloat16* y = reinterpret_cast<__nv_bfloat16*>(ws + kCtrlBytes + parts_bytes());
    // EE_Q4_KERNEL=stream | gemm forces one of the two kernels (for tests and comparisons)
    const char* force = getenv("EE_Q4_KERNEL");
    const bool gemm = force && force[0] == 'g' ? true : force && force[0] == 's' ? false : a.M > slab_rows(a.d);
    const int slab = gemm ? kQ4GemmRows : slab_rows(a.d);
    const int ld_y = (a.d + 63) / 64 * 64;
    if (gemm) {
        const ee_status st = layer_norm_permuted_launch(a.h, a.ld_h, a.gamma, a.beta, a.ln_eps, y, ld_y, a.M, a.d, a.stream);
        if (st != EE_OK) return st;
    }
    for (int r0 = 0; r0 < a.M; r0 += slab) {
        Q4Params p;
        p.weights = static_cast<const uint4*>(q4);
        p.scales = q4_scales(q4, a.V, a.d, group);
        p.y = y + (size_t)r0 * ld_y;
        p.h = static_cast<const __nv_bfloat16*>(a.h) + (size_t)r0 * a.ld_h;
        p.ld_h = a.ld_h; p.gamma = a.gamma; p.beta = a.beta; p.ln_eps = a.ln_eps;
        p.M = a.M - r0 < slab ? a.M - r0 : slab;
        p.d = a.d; p.V = a.V; p.group = group;
        p.parts = reinterpret_cast<RestState*>(ws + kCtrlBytes);
        p.tau_per_row = a.tau_per_row ? a.tau_per_row + r0 : nullptr;
        p.tau = a.tau;
        p.argmax = a.argmax + r0; p.entropy = a.entropy + r0; p.maxprob = a.maxprob + r0; p.exit_mask = a.exit_mask + r0;
        p.ctrl = reinterpret_cast<Control*>(ws);
        const int nt = (p.M + 7) / 8;
        const ee_status s = gemm ? q4_gemm_launch(p, a.num_sms, a.device, a.stream)
                          : nt <= 1 ? launch_head<1>(p, a.num_sms, a.device, a.stream) : launch_head<2>(p, a.num_sms, a.device, a.stream);
        if (s != EE_OK) return s;
    }
    return EE_OK;
}

}  // namespace ee
