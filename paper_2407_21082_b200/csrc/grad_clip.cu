// The norm over all of a step's gradients, and their scaling where it is too large:
//   norm = sqrt(sum over all tensors of sum g^2),   g <- round(g min(1, max_norm / (norm + 1e-6)))
//
// Both walk the tensors in pieces of 32 KB, many CTAs to an SM, and are bound by memory.  The table of tensors is a kernel parameter, so
// that a call copies nothing to the device and may be captured.  The norm needs one launch (the CTA that finishes last adds the CTAs'
// sums, in a fixed order); the scaling walks the pieces backwards, because what the norm read last is what L2 still holds.
//
// Norm and scaling of 103 MB take 48 us (6.4 TB/s over the 309 MB that are read twice and written once), of 820 MB 390 us (6.3 TB/s; the norm alone
// 6.8).  Pieces of 16 KB take 50 and 447 us, of 64 KB 52 and 390; six CTAs per SM 48 and 419.
#include "common.cuh"
#include "kernels.h"

#include <cuda_fp16.h>

namespace ee {

namespace {

constexpr int kThreads = 256;
constexpr int kPieceBytes = 32768;               // eight 16-byte loads per thread
constexpr int kVecs = kPieceBytes / 16 / kThreads;
constexpr int kFew = 16, kMany = 512;            // tensors of a launch: parameters of 0.5 and 16 KB
constexpr int kMaxCtas = 2048;

struct Entry {
    const void* data;
    void* out;
    long long n;
    unsigned int first;                          // number of its first piece, in the launch
    int type;
};
template <int N>
struct Table {
    Entry e[N];
    int count;
    unsigned int pieces;
};

struct NormSpace {
    Control ctrl;
    double parts[1];                             // of every CTA of every launch
};

__device__ __forceinline__ uint4 ld_stream(const void* p) { return __ldcg(reinterpret_cast<const uint4*>(p)); }

template <int N>
__device__ __forceinline__ int entry_of(const Table<N>& t, unsigned int piece) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.e[mid].first <= piece) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ float half_lo(uint32_t v) { return __half2float(__ushort_as_half((unsigned short)v)); }
__device__ __forceinline__ float half_hi(uint32_t v) { return __half2float(__ushort_as_half((unsigned short)(v >> 16))); }

// Element i of a tensor (the ragged or unaligned part).
__device__ __forceinline__ float load_one(const void* p, long long i, int type) {
    if (type == EE_FLOAT32) return __ldcg(reinterpret_cast<const float*>(p) + i);
    const unsigned short v = __ldcg(reinterpret_cast<const unsigned short*>(p) + i);
    return type == EE_BFLOAT16 ? bf16_lo(v) : __half2float(__ushort_as_half(v));
}
__device__ __forceinline__ void store_one(void* p, long long i, int type, float v) {
    if (type == EE_FLOAT32) reinterpret_cast<float*>(p)[i] = v;
    else if (type == EE_BFLOAT16) reinterpret_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
    else reinterpret_cast<__half*>(p)[i] = __float2half_rn(v);
}

template <int kType>
__device__ __forceinline__ void values(uint4 v, float (&x)[kType == EE_FLOAT32 ? 4 : 8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (kType == EE_FLOAT32) x[i] = __uint_as_float(w[i]);
        else {
            x[2 * i] = kType == EE_BFLOAT16 ? bf16_lo(w[i]) : half_lo(w[i]);
            x[2 * i + 1] = kType == EE_BFLOAT16 ? bf16_hi(w[i]) : half_hi(w[i]);
        }
    }
}

// Sum of the squares of a vector's elements.  In fp32 where that neither overflows nor loses anything below (every square that counts is
// a normal number); otherwise, which gradients of any use are not, in fp64.
template <int kType>
__device__ __forceinline__ double squares(uint4 v) {
    constexpr int n = kType == EE_FLOAT32 ? 4 : 8;
    float x[n];
    values<kType>(v, x);
    float q = x[0] * x[0];
#pragma unroll
    for (int i = 1; i < n; ++i) q = fmaf(x[i], x[i], q);
    if (q > 1e-25f && q < 1e37f) return (double)q;
    double s = 0.0;
    if ((v.x | v.y | v.z | v.w) != 0) {
#pragma unroll
        for (int i = 0; i < n; ++i) s = fma((double)x[i], (double)x[i], s);
    }
    return s;
}

template <int kType>
__device__ __forceinline__ double piece_squares(const Entry& e, long long begin, long long end) {
    constexpr int n = kType == EE_FLOAT32 ? 4 : 8;
    double s[2] = {0.0, 0.0};
    long long from = begin;
    if ((reinterpret_cast<uintptr_t>(e.data) & 15) == 0) {
        const uint4* src = reinterpret_cast<const uint4*>(e.data) + begin / n;
        const int whole = (int)((end - begin) / n);
        if (whole == kThreads * kVecs) {
            uint4 v[kVecs];
#pragma unroll
            for (int k = 0; k < kVecs; ++k) v[k] = ld_stream(src + k * kThreads + threadIdx.x);
#pragma unroll
            for (int k = 0; k < kVecs; ++k) s[k & 1] += squares<kType>(v[k]);
        } else {
            for (int i = threadIdx.x; i < whole; i += kThreads) s[0] += squares<kType>(ld_stream(src + i));
        }
        from += (long long)whole * n;
    }
    for (long long i = from + threadIdx.x; i < end; i += kThreads) {
        const double x = (double)load_one(e.data, i, kType);
        s[1] = fma(x, x, s[1]);
    }
    return s[0] + s[1];
}

__device__ __forceinline__ int elements_of_piece(int type) { return kPieceBytes / (type == EE_FLOAT32 ? 4 : 2); }

// Sum over the CTA, in thread 0.
__device__ __forceinline__ double cta_total(double v) {
    __shared__ double of_warp[kThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) of_warp[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kThreads / 32; ++w) s += of_warp[w];
    __syncthreads();
    return s;
}

// One launch of a call: its CTAs' sums go to parts[base ..], and the CTA that is the last of all launches' `total` adds them up.
template <int N>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const __grid_constant__ Table<N> t, NormSpace* space, int base, int total, float* norm) {
    __shared__ int last;
    launch_dependents();
    grid_dependency_wait();
    double s = 0.0;
    for (unsigned int piece = blockIdx.x; piece < t.pieces; piece += gridDim.x) {
        const Entry& e = t.e[entry_of(t, piece)];
        const int per = elements_of_piece(e.type);
        const long long begin = (long long)(piece - e.first) * per, end = begin + per < e.n ? begin + per : e.n;
        s += e.type == EE_BFLOAT16  ? piece_squares<EE_BFLOAT16>(e, begin, end)
             : e.type == EE_FLOAT32 ? piece_squares<EE_FLOAT32>(e, begin, end)
                                    : piece_squares<EE_FLOAT16>(e, begin, end);
    }
    s = cta_total(s);
    if (threadIdx.x == 0) {
        space->parts[base + blockIdx.x] = s;
        last = ticket_arrive_is_last(&space->ctrl.head_ticket[0], (unsigned)total) ? 1 : 0;
    }
    __syncthreads();
    if (!last) return;
    double all = 0.0;
    for (int b = threadIdx.x; b < total; b += kThreads) all += __ldcg(&space->parts[b]);
    all = cta_total(all);
    if (threadIdx.x == 0) {
        *norm = (float)sqrt(all);
        space->ctrl.head_ticket[0] = 0;                                  // ready for the next call
    }
}

template <int kType>
__device__ __forceinline__ uint4 scaled(uint4 v, float c) {
    constexpr int n = kType == EE_FLOAT32 ? 4 : 8;
    float x[n];
    values<kType>(v, x);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (kType == EE_FLOAT32) w[i] = __float_as_uint(x[i] * c);
        else if constexpr (kType == EE_BFLOAT16) w[i] = pack_bf16(x[2 * i] * c, x[2 * i + 1] * c);
        else {
            const __half2 h = __floats2half2_rn(x[2 * i] * c, x[2 * i + 1] * c);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int kType>
__device__ __forceinline__ void scale_piece(const Entry& e, long long begin, long long end, float c) {
    constexpr int n = kType == EE_FLOAT32 ? 4 : 8;
    long long from = begin;
    if (((reinterpret_cast<uintptr_t>(e.data) | reinterpret_cast<uintptr_t>(e.out)) & 15) == 0) {
        const uint4* src = reinterpret_cast<const uint4*>(e.data) + begin / n;
        uint4* dst = reinterpret_cast<uint4*>(e.out) + begin / n;
        const int whole = (int)((end - begin) / n);
        if (whole == kThreads * kVecs) {
            uint4 v[kVecs];
#pragma unroll
            for (int k = 0; k < kVecs; ++k) v[k] = ld_stream(src + k * kThreads + threadIdx.x);
#pragma unroll
            for (int k = 0; k < kVecs; ++k) __stcs(dst + k * kThreads + threadIdx.x, scaled<kType>(v[k], c));
        } else {
            for (int i = threadIdx.x; i < whole; i += kThreads) dst[i] = scaled<kType>(ld_stream(src + i), c);
        }
        from += (long long)whole * n;
    }
    for (long long i = from + threadIdx.x; i < end; i += kThreads) store_one(e.out, i, kType, load_one(e.data, i, kType) * c);
}

template <int N>
__global__ void __launch_bounds__(kThreads) grad_clip_kernel(const __grid_constant__ Table<N> t, const float* norm, float max_norm) {
    launch_dependents();
    grid_dependency_wait();
    float c = __fdiv_rn(max_norm, ld_dep(norm) + 1e-6f);
    c = c > 1.f ? 1.f : c;                                               // a norm that is not a number scales by what is not one
    for (unsigned int left = t.pieces - blockIdx.x; (int)left > 0; left -= gridDim.x) {
        const unsigned int piece = left - 1;
        const Entry& e = t.e[entry_of(t, piece)];
        if (c == 1.f && e.data == e.out) continue;                       // as they are
        const int per = elements_of_piece(e.type);
        const long long begin = (long long)(piece - e.first) * per, end = begin + per < e.n ? begin + per : e.n;
        if (e.type == EE_BFLOAT16) scale_piece<EE_BFLOAT16>(e, begin, end, c);
        else if (e.type == EE_FLOAT32) scale_piece<EE_FLOAT32>(e, begin, end, c);
        else scale_piece<EE_FLOAT16>(e, begin, end, c);
    }
}

int grid_of(unsigned int pieces, int num_sms) {
    const unsigned int most = (unsigned)(num_sms * 8 < kMaxCtas ? num_sms * 8 : kMaxCtas);
    return (int)(pieces < most ? pieces : most);
}

template <int N>
void fill(Table<N>& t, const ee_tensor* tensors, void* const* out, int count) {
    t.count = 0;
    t.pieces = 0;
    for (int i = 0; i < count; ++i) {
        if (tensors[i].n == 0) continue;
        const int per = kPieceBytes / (tensors[i].type == EE_FLOAT32 ? 4 : 2);
        Entry& e = t.e[t.count++];
        e.data = tensors[i].data;
        e.out = out ? out[i] : tensors[i].data;
        e.n = tensors[i].n;
        e.type = tensors[i].type;
        e.first = t.pieces;
        t.pieces += (unsigned)((e.n + per - 1) / per);
    }
}

unsigned int pieces_of(const ee_tensor* tensors, int count) {
    unsigned int pieces = 0;
    for (int i = 0; i < count; ++i) {
        const int per = kPieceBytes / (tensors[i].type == EE_FLOAT32 ? 4 : 2);
        pieces += (unsigned)((tensors[i].n + per - 1) / per);
    }
    return pieces;
}

template <int N>
cudaError_t launch_norm(const ee_tensor* tensors, int count, NormSpace* space, int base, int total, float* norm, int num_sms, cudaStream_t stream) {
    Table<N> t;
    fill(t, tensors, nullptr, count);
    return launch_pdl(grad_norm_kernel<N>, dim3(grid_of(t.pieces, num_sms)), kThreads, 0, stream, t, space, base, total, norm);
}
template <int N>
cudaError_t launch_clip(const ee_tensor* tensors, void* const* out, int count, float max_norm, const float* norm, int num_sms, cudaStream_t stream) {
    Table<N> t;
    fill(t, tensors, out, count);
    return launch_pdl(grad_clip_kernel<N>, dim3(grid_of(t.pieces, num_sms)), kThreads, 0, stream, t, norm, max_norm);
}

}  // namespace

size_t grad_norm_workspace_bytes(int n_tensors) {
    const int launches = n_tensors > 0 ? (n_tensors + kMany - 1) / kMany : 1;
    return sizeof(Control) + (size_t)launches * kMaxCtas * sizeof(double);
}

ee_status grad_norm_launch(const ee_tensor* tensors, int n_tensors, float* norm, void* workspace, int num_sms, cudaStream_t stream) {
    NormSpace* space = static_cast<NormSpace*>(workspace);
    int total = 0;
    for (int at = 0; at < n_tensors; at += kMany) total += grid_of(pieces_of(tensors + at, n_tensors - at < kMany ? n_tensors - at : kMany), num_sms);
    if (total == 0) return cudaMemsetAsync(norm, 0, sizeof(float), stream) == cudaSuccess ? EE_OK : EE_ERR_CUDA;
    int base = 0;
    for (int at = 0; at < n_tensors; at += kMany) {
        const int count = n_tensors - at < kMany ? n_tensors - at : kMany;
        const int grid = grid_of(pieces_of(tensors + at, count), num_sms);
        if (grid == 0) continue;
        const cudaError_t e = count <= kFew ? launch_norm<kFew>(tensors + at, count, space, base, total, norm, num_sms, stream)
                                            : launch_norm<kMany>(tensors + at, count, space, base, total, norm, num_sms, stream);
        if (e != cudaSuccess) return EE_ERR_CUDA;
        base += grid;
    }
    return EE_OK;
}

ee_status grad_clip_launch(const ee_tensor* tensors, void* const* out, int n_tensors, float max_norm, const float* norm, int num_sms,
                           cudaStream_t stream) {
    for (int end = n_tensors; end > 0; end -= kMany) {                   // backwards here as well
        const int count = end < kMany ? end : kMany, at = end - count;
        if (pieces_of(tensors + at, count) == 0) continue;
        const cudaError_t e = count <= kFew ? launch_clip<kFew>(tensors + at, out ? out + at : nullptr, count, max_norm, norm, num_sms, stream)
                                            : launch_clip<kMany>(tensors + at, out ? out + at : nullptr, count, max_norm, norm, num_sms, stream);
        if (e != cudaSuccess) return EE_ERR_CUDA;
    }
    return EE_OK;
}

}  // namespace ee
