// Writing heads in microscaled 4-bit floating point, reading them back, and the activations of a call in the same form.
//
// Packing reads 2 bytes per weight and writes 0.56 (0.53 for groups of 32).  Groups of 16 need the largest magnitude of the whole matrix
// first, which is a pass of its own over it.  50304 x 2048, groups of 16: 36 us for that pass (5.7 TB/s), 57 for the writing (4.6 TB/s read and
// written; issue slots 72 % busy), 53 for the reading back (4.9 TB/s); 151 us together.  A warp has four pieces of a row in flight: with one, and
// a 64-bit division per vector when reading back, it was 207.
//
// The activations (a LayerNorm in fp64 moments, then the quantisation) are bound by issue slots: 16384 rows of 2560 take 80 us, 1.3 TB/s; left out
// of copies, the normalisation is 30 us of that and the quantisation 20.
#include "fp4_common.cuh"
#include "layer_norm.cuh"
#include "kernels.h"

namespace ee {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kAhead = 4;                        // 512-byte pieces of a row that a warp has in flight

struct Fp4Pack {
    const uint4* W;                // [V][d] bf16
    int V, d;
    unsigned char* fp4;
};

// Largest magnitude of the matrix, into the second word of the header (cleared before).
__global__ void __launch_bounds__(kThreads) fp4_top_kernel(const Fp4Pack p) {
    const long long n = (long long)p.V * p.d / 8;
    uint32_t top = 0;
    const long long stride = (long long)gridDim.x * kThreads;
    long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
    for (; i + 3 * stride < n; i += 4 * stride) {
        uint4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = ld_dep(p.W + i + k * stride);
#pragma unroll
        for (int k = 0; k < 4; ++k) top = max(top, fp4_top8(v[k]));
    }
    for (; i < n; i += stride) top = max(top, fp4_top8(ld_dep(p.W + i)));
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) atomicMax(reinterpret_cast<uint32_t*>(p.fp4) + 1, top);
}

// A warp per row, 256 columns at a time.
template <int kGroup>
__global__ void __launch_bounds__(kThreads) fp4_pack_kernel(const Fp4Pack p) {
    const int blocks = fp4_blocks(p.d), nvec = p.d >> 3, lane = threadIdx.x & 31;
    const long long rows = (long long)fp4_tiles(p.V, kFp4Rows) * kFp4Rows;
    float common = 1.f;
    if (kGroup == 16) {
        const int e = fp4_common_exponent(ld_dep(reinterpret_cast<const uint32_t*>(p.fp4) + 1));
        common = fp4_two_to(-e);
        if (blockIdx.x == 0 && threadIdx.x == 0) *reinterpret_cast<float*>(p.fp4) = fp4_two_to(e);
    } else if (blockIdx.x == 0 && threadIdx.x == 0) {
        *reinterpret_cast<float*>(p.fp4) = 1.f;
    }
    for (long long row = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); row < rows; row += (long long)gridDim.x * kWarps) {
        const int r = (int)(row % kFp4Rows);
        unsigned char* tile = p.fp4 + kFp4Header + (row / kFp4Rows) * blocks * (long long)fp4_unit_bytes(kGroup, kFp4Rows);
        const uint4* src = p.W + row * nvec;
        for (int c0 = 0; c0 < blocks * 16; c0 += 32 * kAhead) {
            uint4 v[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int c = c0 + 32 * k + lane;
                v[k] = row < p.V && c < nvec ? ld_dep(src + c) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (c0 + 32 * k >= blocks * 16) break;                   // the same for the whole warp
                const int c = c0 + 32 * k + lane;
                uint32_t code;
                const uint32_t word = fp4_quantise8<kGroup>(v[k], fp4_group_top<kGroup>(fp4_top8(v[k])), common, code);
                const uint32_t codes = fp4_gather_codes<kGroup>(code);
                if (c < blocks * 16) {
                    unsigned char* unit = tile + (c >> 4) * (long long)fp4_unit_bytes(kGroup, kFp4Rows);
                    *reinterpret_cast<uint32_t*>(unit + fp4_scale_bytes(kGroup) + fp4_word_offset(r, c & 15)) = word;
                    if (kGroup == 16 ? (c & 7) == 0 : (c & 15) == 0)
                        *reinterpret_cast<uint32_t*>(unit + fp4_scales_offset(r, kGroup == 16 ? (c >> 3) & 1 : 0)) = codes;
                }
            }
        }
    }
}

// A warp per row, likewise.
template <int kGroup>
__global__ void __launch_bounds__(kThreads) fp4_unpack_kernel(const unsigned char* fp4, int V, int d, uint4* W) {
    const int blocks = fp4_blocks(d), nvec = d >> 3;
    const float factor = ld_dep(reinterpret_cast<const float*>(fp4));
    const int lane = threadIdx.x & 31;
    for (long long row = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); row < V; row += (long long)gridDim.x * kWarps) {
        const int r = (int)(row % kFp4Rows);
        const unsigned char* tile = fp4 + kFp4Header + (row / kFp4Rows) * blocks * (long long)fp4_unit_bytes(kGroup, kFp4Rows);
        for (int c0 = lane; c0 < nvec; c0 += 32 * kAhead) {
            uint32_t word[kAhead], codes[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int c = c0 + 32 * k;
                const unsigned char* unit = tile + (c >> 4) * (long long)fp4_unit_bytes(kGroup, kFp4Rows);
                word[k] = c < nvec ? ld_dep(reinterpret_cast<const uint32_t*>(unit + fp4_scale_bytes(kGroup) + fp4_word_offset(r, c & 15))) : 0u;
                codes[k] = c < nvec ? ld_dep(reinterpret_cast<const uint32_t*>(unit + fp4_scales_offset(r, kGroup == 16 ? (c >> 3) & 1 : 0))) : 0u;
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int c = c0 + 32 * k, group = (c & 15) * 8 / kGroup;                // of the unit's
                const uint32_t code = (codes[k] >> (8 * (group & 3))) & 0xffu;
                const float s = kGroup == 32 ? fp4_two_to((int)code - 127) : fp4_scale_value(code) * factor;
                uint32_t o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 x = fp4_unpack2(word[k] >> (8 * i));
                    o[i] = pack_bf16(x.x * s, x.y * s);
                }
                if (c < nvec) __stcs(W + row * nvec + c, make_uint4(o[0], o[1], o[2], o[3]));
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------- activations
struct Fp4Acts {
    const __nv_bfloat16* h;
    long long ld_h;
    const float* gamma;
    const float* beta;
    float ln_eps;
    int M, d;
    int rows_per_tile;             // 8, 16, 32, 64 or 128
    unsigned char* acts;
    float* factor;
};

// Vector c of a row, its LayerNorm in `y`, into the row's place.  Whole warps, for their shuffles.
template <int kGroup>
__device__ __forceinline__ void put_act(const Fp4Acts& a, unsigned char* tile, int r, int c, uint4 y, float common, int blocks) {
    uint32_t code;
    const uint32_t word = fp4_quantise8<kGroup>(y, fp4_group_top<kGroup>(fp4_top8(y)), common, code);
    const uint32_t codes = fp4_gather_codes<kGroup>(code);
    if (c >= blocks * 16) return;
    unsigned char* unit = tile + (c >> 4) * (long long)fp4_unit_bytes(kGroup, a.rows_per_tile);
    *reinterpret_cast<uint32_t*>(unit + fp4_scale_bytes(kGroup) + fp4_word_offset(r, c & 15)) = word;
    if (kGroup == 16 ? (c & 7) == 0 : (c & 15) == 0)
        *reinterpret_cast<uint32_t*>(unit + fp4_scales_offset(r, kGroup == 16 ? (c >> 3) & 1 : 0)) = codes;
}

// A row by kRowThreads threads (a warp, or the CTA), kVecs vectors of eight each; the row stays in registers.
// The first kernel of a call: it lets no other start before all earlier work of the stream is done, so that the kernels behind it may
// read the weights as they are.
template <int kGroup, int kRowThreads, int kVecs>
__global__ void __launch_bounds__(kThreads) fp4_acts_kernel(const Fp4Acts a) {
    __shared__ double sums[2][kWarps];
    __shared__ uint32_t tops[kWarps];
    constexpr bool kCta = kRowThreads > 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = kCta ? blockIdx.x : blockIdx.x * kWarps + warp;
    const int at = kCta ? threadIdx.x : lane, step = kCta ? (int)blockDim.x : 32, warps = blockDim.x >> 5;
    const int nvec = a.d >> 3, blocks = fp4_blocks(a.d);
    grid_dependency_wait();
    launch_dependents();
    if (row >= a.M) return;
    const uint4* src = reinterpret_cast<const uint4*>(a.h + (size_t)row * a.ld_h);
    uint4 x[kVecs];
    Moments m;
    m.clear();
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
        x[k] = at + k * step < nvec ? ld_dep(src + at + k * step) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
        if (at + k * step < nvec) m.add(x[k], k);
    auto totals = [&](double& s, double& q) {                            // in a fixed order, the same bits in every thread
        warp_sum2_d(s, q);
        if (!kCta) return;
        if (lane == 0) { sums[0][warp] = s; sums[1][warp] = q; }
        __syncthreads();
        s = q = 0.0;
        for (int w = 0; w < warps; ++w) { s += sums[0][w]; q += sums[1][w]; }
        __syncthreads();
    };
    const double d = (double)a.d, inv_d = 1.0 / d;
    double s = m.sum(), q = m.sum_sq(), mu, var;
    totals(s, q);
    if (!row_variance_one_pass(s, q, d, inv_d, mu, var)) {
        double q0 = 0.0, q1 = 0.0;
#pragma unroll
        for (int k = 0; k < kVecs; ++k)
            if (at + k * step < nvec) vec8_sqdev_d(x[k], mu, q0, q1);
        double v = q0 + q1, none = 0.0;
        totals(v, none);
        var = v * inv_d;
    }
    const RowStats st = row_stats(mu, var, a.ln_eps);
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const int c = at + k * step;
        if (c < nvec) {
            x[k] = layer_norm_vec8<true, true>(x[k], st, a.gamma, a.beta, c);
            top = max(top, fp4_top8(x[k]));
        }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (kCta) {
        if (lane == 0) tops[warp] = top;
        __syncthreads();
        for (int w = 0; w < warps; ++w) top = max(top, tops[w]);
    }
    const bool finite = top < 0x7f80u;
    const int e = kGroup == 16 && finite ? fp4_common_exponent(top) : 0;
    if (at == 0) a.factor[row] = finite ? fp4_two_to(e) : CUDART_NAN_F;
    const float common = fp4_two_to(-e);
    const int r = row % a.rows_per_tile;
    unsigned char* tile = a.acts + (row / a.rows_per_tile) * (size_t)blocks * fp4_unit_bytes(kGroup, a.rows_per_tile);
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        if (k * step >= blocks * 16) break;                              // the same for the whole warp
        put_act<kGroup>(a, tile, r, at + k * step, finite ? x[k] : make_uint4(0, 0, 0, 0), common, blocks);
    }
}

template <int kGroup>
cudaError_t launch_acts(const Fp4Acts& a, cudaStream_t stream) {
    const int padded = fp4_blocks(a.d) * 16;                             // vectors of a row, zeros beyond d among them
    // A CTA per row while there are too few rows to fill the SMs with warps, and where a row does not fit a warp's registers; a warp per row above.
    // The whole call, us, a warp / a CTA per row (V = 50304): 256 rows of 2560 43 / 37, 1024 of 1024 52.9 / 50.7, 2048 of 512 71.0 / 70.6, of 1024 86.5 / 86.4,
    // of 2560 146 / 143, 4096 of 512 124.5 / 125.1, of 1024 151 / 154, of 2560 265 / 264, 16384 of 512 438 / 441, of 1024 535 / 550, of 2560 969 / 1021;
    // rows of 4096 (in a warp 128 registers): 1024 of them 139 / 112, 4096 478 / 426; 2048 of 8192 505 / 417.
    if (a.M <= 2048 || padded > 320) {
        const int warps = (padded + 31) / 32;
        const int threads = 32 * (warps < kWarps ? warps : kWarps);
        return padded <= threads * 2 ? launch_pdl(fp4_acts_kernel<kGroup, kThreads, 2>, dim3(a.M), threads, 0, stream, a)
                                     : launch_pdl(fp4_acts_kernel<kGroup, kThreads, 4>, dim3(a.M), threads, 0, stream, a);
    }
    const dim3 grid((a.M + kWarps - 1) / kWarps);
    return padded <= 128 ? launch_pdl(fp4_acts_kernel<kGroup, 32, 4>, grid, kThreads, 0, stream, a)
                         : launch_pdl(fp4_acts_kernel<kGroup, 32, 10>, grid, kThreads, 0, stream, a);
}

struct HeadSpace {
    size_t factor, acts, parts, total;
};
HeadSpace head_space(int M, int d, int V, int group) {
    HeadSpace s;
    const int rows = M <= kFp4StreamRows ? fp4_stream_padded(M) : kFp4Rows;
    const int tiles = M <= kFp4StreamRows ? 1 : fp4_gemm_act_tiles(M);
    s.factor = kCtrlBytes;
    s.acts = align_up(s.factor + (size_t)M * sizeof(float), 1024);
    s.parts = align_up(s.acts + (size_t)tiles * fp4_blocks(d) * fp4_unit_bytes(group, rows), 256);
    // a workspace for M rows serves fewer as well: what lies in front of the states grows with M, and the states' part is the most of any
    const size_t few = fp4_stream_parts_bytes(M <= kFp4StreamRows ? M : kFp4StreamRows), many = M <= kFp4StreamRows ? 0 : fp4_gemm_parts_bytes(M, V);
    s.total = s.parts + (few > many ? few : many);
    return s;
}

}  // namespace

size_t fp4_weight_bytes(int V, int d, int group) {
    return kFp4Header + (size_t)fp4_tiles(V, kFp4Rows) * fp4_blocks(d) * fp4_unit_bytes(group, kFp4Rows);
}

ee_status fp4_pack_launch(const void* W, int V, int d, int group, void* fp4, int num_sms, cudaStream_t stream) {
    const Fp4Pack p{static_cast<const uint4*>(W), V, d, static_cast<unsigned char*>(fp4)};
    const long long rows = (long long)fp4_tiles(V, kFp4Rows) * kFp4Rows, most = (long long)num_sms * 8;
    const int grid = (int)(rows / kWarps < most ? rows / kWarps : most);
    if (cudaMemsetAsync(fp4, 0, kFp4Header, stream) != cudaSuccess) return EE_ERR_CUDA;
    if (group == 16) {
        fp4_top_kernel<<<(int)most, kThreads, 0, stream>>>(p);
        fp4_pack_kernel<16><<<grid, kThreads, 0, stream>>>(p);
    } else {
        fp4_pack_kernel<32><<<grid, kThreads, 0, stream>>>(p);
    }
    return cudaGetLastError() == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

ee_status fp4_unpack_launch(const void* fp4, int V, int d, int group, void* W, int num_sms, cudaStream_t stream) {
    const unsigned char* src = static_cast<const unsigned char*>(fp4);
    if (group == 16) fp4_unpack_kernel<16><<<num_sms * 8, kThreads, 0, stream>>>(src, V, d, static_cast<uint4*>(W));
    else fp4_unpack_kernel<32><<<num_sms * 8, kThreads, 0, stream>>>(src, V, d, static_cast<uint4*>(W));
    return cudaGetLastError() == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

size_t fp4_head_workspace_bytes(int M, int d, int V, int group) { return head_space(M, d, V, group).total; }

ee_status fp4_head_launch(const HeadArgs& a, const void* fp4, int group) {
    unsigned char* ws = static_cast<unsigned char*>(a.workspace);
    const HeadSpace s = head_space(a.M, a.d, a.V, group);
    const bool few = a.M <= kFp4StreamRows;
    Fp4Acts acts;
    acts.h = static_cast<const __nv_bfloat16*>(a.h);
    acts.ld_h = a.ld_h; acts.gamma = a.gamma; acts.beta = a.beta; acts.ln_eps = a.ln_eps;
    acts.M = a.M; acts.d = a.d;
    acts.rows_per_tile = few ? fp4_stream_padded(a.M) : kFp4Rows;
    acts.acts = ws + s.acts;
    acts.factor = reinterpret_cast<float*>(ws + s.factor);
    if ((group == 16 ? launch_acts<16>(acts, a.stream) : launch_acts<32>(acts, a.stream)) != cudaSuccess) return EE_ERR_CUDA;
    Fp4Head p;
    p.weights = static_cast<const unsigned char*>(fp4) + kFp4Header;
    p.weight_factor = static_cast<const float*>(fp4);
    p.acts = acts.acts;
    p.factor = acts.factor;
    p.M = a.M; p.d = a.d; p.V = a.V;
    p.tau_per_row = a.tau_per_row; p.tau = a.tau;
    p.argmax = a.argmax; p.entropy = a.entropy; p.maxprob = a.maxprob; p.exit_mask = a.exit_mask;
    p.ctrl = reinterpret_cast<Control*>(a.workspace);
    return few ? fp4_stream_launch(p, group, ws + s.parts, a.num_sms, a.device, a.stream)
               : fp4_gemm_launch(p, group, ws + s.parts, a.device, a.stream);
}

}  // namespace ee
