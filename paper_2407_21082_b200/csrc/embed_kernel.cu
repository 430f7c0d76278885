// The embedding that shares its table with a head: out[i] = bf16(scale * table[token_i]), and its gradient
//   dtable[v] = scale * sum over i with token_i = v of dout[i]
// by sorted tokens, in fp32 and in a fixed order (no floating-point atomics: the same bits from run to run).
//
// For up to 512 tokens every position looks for its token in the list (embed_short_kernel).  For longer lists the gradient is
// three steps.  (1) The tokens are sorted, stably, by one cluster of CTAs in its shared memory when they fit
// (n <= 16384 and V < 2^18: 18 bits of token and 14 of position in one word), while the rest of the device clears the table, which
// takes longer (V d bytes against n words); longer lists go through the library's radix sort.  (2) The sorted list is cut into
// chunks of equal length, one CTA (per 128 vectors of the width) each: it adds up the rows of every token in it.  A token
// that lies inside the chunk is finished there; a run that crosses a chunk's border, as frequent tokens' do, leaves
// fp32 partial sums (one for the run that comes in, one for the run that goes out).  (3) A run's partial sums are
// joined in order by the chunk it starts in.  So a token that fills the whole batch costs no more than any other batch.
// Tokens outside [0, V) take no part: they sort behind all others and are skipped.
//
// 16384 tokens, d = 1024, V = 50304, bf16: 37 to 40 us (floor 21: 34 MB of rows, 103 MB of table), of which 16 clear the table (6.4 TB/s)
// beside the sort's 13, 12 add up and 9 join; 16385 tokens through the radix sort 56 to 59 us (words, then three launches per eight bits of
// token, all behind the clearing); 600 tokens x 64 14 us, and 34 where V >= 2^18 does not fit the word; 257 tokens x 520 into 32003 rows of
// fp32 11.5 us.  The lookup of 32 tokens takes 1.5 us on the device.
#include "common.cuh"
#include "kernels.h"
#include "sm100_ptx.cuh"

namespace ee {

namespace {

typedef unsigned long long u64;

__device__ __forceinline__ void unpack8f(uint4 o, float (&x)[8]) {
    x[0] = bf16_lo(o.x); x[1] = bf16_hi(o.x); x[2] = bf16_lo(o.y); x[3] = bf16_hi(o.y);
    x[4] = bf16_lo(o.z); x[5] = bf16_hi(o.z); x[6] = bf16_lo(o.w); x[7] = bf16_hi(o.w);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// One 16-byte vector per thread and turn.
__global__ void __launch_bounds__(256) embed_kernel(const __nv_bfloat16* table, int V, int nvec, const int* tokens, int n, float scale,
                                                    __nv_bfloat16* out, long long ld_out) {
    launch_dependents();
    const long long total = (long long)n * nvec, step = (long long)gridDim.x * 256;
    grid_dependency_wait();
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
        const int row = (int)(i / nvec), c = (int)(i - (long long)row * nvec);
        const int token = ld_dep(tokens + row);
        float x[8] = {};
        if ((unsigned)token < (unsigned)V) {
            unpack8f(ld_dep(reinterpret_cast<const uint4*>(table) + (size_t)token * nvec + c), x);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] *= scale;
        }
        *(reinterpret_cast<uint4*>(out + (size_t)row * ld_out) + c) = pack8(x);
    }
}

// ---------------------------------------------------------------------------------------------------- sorting

constexpr int kSortCtas = 8;                             // one cluster
constexpr int kSortThreads = 1024;
constexpr int kSortItems = 2;                            // per thread
constexpr int kSortCtaItems = kSortThreads * kSortItems;
constexpr int kSortMax = kSortCtas * kSortCtaItems;      // 16384 tokens one cluster sorts
constexpr int kSortIndexBits = 14;
constexpr int kSortMaxV = (1 << (32 - kSortIndexBits)) - 1;
constexpr int kSortWarps = kSortThreads / 32;

__device__ __forceinline__ unsigned int ld_cluster(uint32_t addr) {
    unsigned int v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, unsigned int v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// Clears `vecs` vectors: bulk copies out of zeros in shared memory, all of a CTA's issued by one thread.  The kernel that sorts the
// tokens lets this one start after its own wait for the stream's earlier work, so that clearing (V d bytes) runs beside sorting
// (n words) and needs no wait before it writes; it waits before it ends, so that its own end means that of both.  For short lists it
// comes first itself, as an ordinary launch, and lets what adds up the rows start beside it.  (Its CTAs have to find the SMs evenly
// free: started early, among the CTAs of a kernel that is still there, they crowd on some of them, and clearing 208 MB took 92 us
// instead of 35.)
constexpr unsigned int kClearBytes = 16384;
__global__ void __launch_bounds__(128) embed_clear_kernel(uint4* clear, long long vecs) {
    __shared__ __align__(128) uint4 zeros[kClearBytes / 16];
    launch_dependents();
    for (int i = threadIdx.x; i < (int)(kClearBytes / 16); i += 128) zeros[i] = make_uint4(0, 0, 0, 0);
    ptx::fence_proxy_async();
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t src = ptx::smem_addr(zeros);
        const long long total = vecs * 16;
        unsigned char* out = reinterpret_cast<unsigned char*>(clear);
        for (long long at = (long long)blockIdx.x * kClearBytes; at < total; at += (long long)gridDim.x * kClearBytes) {
            const uint32_t size = (uint32_t)(total - at < kClearBytes ? total - at : kClearBytes);
            asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(out + at), "r"(src), "r"(size) : "memory");
        }
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");       // written, and the zeros are read
    }
    grid_dependency_wait();
}

// One cluster: stable radix sort of (token, position), eight bits a pass, items in registers and the sorted list spread over the
// CTAs' shared memory.  A CTA owns 2048 consecutive items, a warp 64 of them in two rounds, so that (CTA, warp, round, lane) is
// the order in the list; the CTAs exchange their digit counts and scatter into one another's memory.  (One CTA alone took
// 35 us for 16384 tokens, twice the clearing of the table beside it.)
__global__ void __launch_bounds__(kSortThreads, 1) embed_sort_kernel(const int* tokens, int n, int V, int passes, int2* sorted) {
    __shared__ unsigned int list[kSortCtaItems];
    __shared__ unsigned int cnt[kSortWarps][256];
    __shared__ unsigned int total[256];                   // this CTA's items of each digit, read by the others
    __shared__ unsigned int start[256];                   // where this CTA's run of a digit begins
    __shared__ unsigned int warp_part[8];
    grid_dependency_wait();
    launch_dependents();                                  // after the wait: see embed_clear_kernel
    const int rank = (int)ptx::cluster_cta_rank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int local0 = warp * 64 + lane, base = rank * kSortCtaItems;
    unsigned int item[kSortItems];
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) {
        const int i = base + local0 + r * 32;
        item[r] = 0;
        if (i < n) {
            const int t = ld_dep(tokens + i);
            item[r] = ((unsigned int)((unsigned)t < (unsigned)V ? t : V) << kSortIndexBits) | (unsigned int)i;
        }
    }
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = kSortIndexBits + 8 * pass;
        for (int i = threadIdx.x; i < kSortWarps * 256; i += kSortThreads) (&cnt[0][0])[i] = 0;
        __syncthreads();
        unsigned int place[kSortItems];
#pragma unroll
        for (int r = 0; r < kSortItems; ++r) {
            const bool valid = base + local0 + r * 32 < n;
            const unsigned int digit = valid ? (item[r] >> shift) & 255u : 0xffffffffu;
            const unsigned int peers = __match_any_sync(0xffffffffu, digit);
            const int leader = __ffs(peers) - 1;
            unsigned int before = 0;
            if (valid && lane == leader) before = atomicAdd(&cnt[warp][digit], (unsigned int)__popc(peers));
            before = __shfl_sync(0xffffffffu, before, leader);
            place[r] = before + __popc(peers & ((1u << lane) - 1u));
        }
        __syncthreads();
        if (threadIdx.x < 256) {                          // thread = digit: the warps' starts inside the CTA's run
            unsigned int run = 0;
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) {
                const unsigned int k = cnt[w][threadIdx.x];
                cnt[w][threadIdx.x] = run;
                run += k;
            }
            total[threadIdx.x] = run;
        }
        ptx::cluster_sync_all();
        unsigned int all = 0, before = 0, incl = 0;
        if (threadIdx.x < 256) {
            const uint32_t mine = ptx::smem_addr(&total[threadIdx.x]);
            unsigned int k[kSortCtas];
#pragma unroll
            for (int c = 0; c < kSortCtas; ++c) k[c] = ld_cluster(ptx::map_to_cta(mine, c));
#pragma unroll
            for (int c = 0; c < kSortCtas; ++c) {
                all += k[c];
                before += c < rank ? k[c] : 0u;
            }
            incl = all;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned int x = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += x;
            }
            if (lane == 31) warp_part[warp] = incl;
        }
        __syncthreads();
        if (threadIdx.x < 256) {
            unsigned int digits_before = 0;
            for (int w = 0; w < warp; ++w) digits_before += warp_part[w];
            start[threadIdx.x] = digits_before + incl - all + before;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kSortItems; ++r)
            if (base + local0 + r * 32 < n) {
                const unsigned int digit = (item[r] >> shift) & 255u;
                const unsigned int to = start[digit] + cnt[warp][digit] + place[r];
                st_cluster(ptx::map_to_cta(ptx::smem_addr(&list[to % kSortCtaItems]), to / kSortCtaItems), item[r]);
            }
        ptx::cluster_sync_all();                          // the list is whole; and nobody scatters again before everyone has read it,
#pragma unroll                                            // the next pass's first meeting being in between
        for (int r = 0; r < kSortItems; ++r)
            if (base + local0 + r * 32 < n) item[r] = list[local0 + r * 32];
    }
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) {
        const int i = base + local0 + r * 32;
        if (i < n) sorted[i] = make_int2((int)(item[r] & ((1u << kSortIndexBits) - 1u)), (int)(item[r] >> kSortIndexBits));
    }
}

// (position, token) words for the radix sort over memory.
__global__ void __launch_bounds__(256) embed_words_kernel(const int* tokens, int n, int V, u64* words) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int t = ld_dep(tokens + i);
    words[i] = ((u64)(unsigned int)((unsigned)t < (unsigned)V ? t : V) << 32) | (unsigned int)i;
}

// ---------------------------------------------------------------------------------------------------- adding up

struct EmbedGrad {
    const __nv_bfloat16* dout;
    long long ld_dout;
    const int2* sorted;            // (position, token) in order of token, then position
    int n, V, nvec, chunk, n_chunks;
    float scale;
    void* dtable;
    int wide, add;                 // fp32 table; add to what it holds
    float* parts;                  // [n_chunks][2][8 * nvec]: the run that comes in, the run that goes out
};

__device__ __forceinline__ void store_row(const EmbedGrad& a, int token, int c, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= a.scale;
    const size_t at = (size_t)token * a.nvec + c;
    if (a.wide) {
        float4* out = reinterpret_cast<float4*>(a.dtable) + 2 * at;
        if (a.add) {
            const float4 o0 = ld_dep(out), o1 = ld_dep(out + 1);
            x[0] += o0.x; x[1] += o0.y; x[2] += o0.z; x[3] += o0.w;
            x[4] += o1.x; x[5] += o1.y; x[6] += o1.z; x[7] += o1.w;
        }
        out[0] = make_float4(x[0], x[1], x[2], x[3]);
        out[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        uint4* out = reinterpret_cast<uint4*>(a.dtable) + at;
        if (a.add) {
            float o[8];
            unpack8f(ld_dep(out), o);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] += o[j];
        }
        *out = pack8(x);
    }
}
__device__ __forceinline__ void store_part(const EmbedGrad& a, int chunk, int which, int c, const float (&x)[8]) {
    float4* out = reinterpret_cast<float4*>(a.parts + ((size_t)chunk * 2 + which) * a.nvec * 8) + 2 * c;
    out[0] = make_float4(x[0], x[1], x[2], x[3]);
    out[1] = make_float4(x[4], x[5], x[6], x[7]);
}

constexpr int kSumThreads = 128;
constexpr int kSumAhead = 8;                              // rows in flight per thread (16: 96 registers, 12 -> 15.6 us at n = 16384)

__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(const __grid_constant__ EmbedGrad a) {
    __shared__ int2 entry[kSumThreads];
    launch_dependents();
    grid_dependency_wait();
    const int p0 = blockIdx.x * a.chunk, p1 = min(a.n, p0 + a.chunk);
    const int c = blockIdx.y * kSumThreads + threadIdx.x;
    const bool live = c < a.nvec;
    const int token_before = p0 > 0 ? ld_dep(a.sorted + p0 - 1).y : -1;
    const int token_after = p1 < a.n ? ld_dep(a.sorted + p1).y : -1;
    float acc[8] = {};
    int token = token_before;                             // token of the run being added up
    bool comes_in = true;                                 // it started before the chunk
    bool empty = true;
    for (int q0 = p0; q0 < p1; q0 += kSumThreads) {
        __syncthreads();
        if (q0 + (int)threadIdx.x < p1) entry[threadIdx.x] = ld_dep(a.sorted + q0 + threadIdx.x);
        __syncthreads();
        const int count = min(kSumThreads, p1 - q0);
        for (int k0 = 0; k0 < count; k0 += kSumAhead) {
            uint4 v[kSumAhead];
#pragma unroll
            for (int k = 0; k < kSumAhead; ++k)
                if (live && k0 + k < count && entry[k0 + k].y < a.V)
                    v[k] = ld_dep(reinterpret_cast<const uint4*>(a.dout + (size_t)entry[k0 + k].x * a.ld_dout) + c);
#pragma unroll
            for (int k = 0; k < kSumAhead; ++k) {
                if (k0 + k >= count) break;
                const int t = entry[k0 + k].y;
                if (t >= a.V) break;                      // from here on only tokens that take no part
                if (t != token) {                         // the run before this token ends here
                    if (!empty && live) {
                        if (comes_in) store_part(a, blockIdx.x, 0, c, acc);
                        else store_row(a, token, c, acc);
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
                    token = t;
                    comes_in = false;
                }
                empty = false;
                float x[8];
                if (live) {
                    unpack8f(v[k], x);
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[j] += x[j];
                }
            }
        }
    }
    if (empty || !live) return;
    if (comes_in) store_part(a, blockIdx.x, 0, c, acc);
    else if (token_after == token) store_part(a, blockIdx.x, 1, c, acc);
    else store_row(a, token, c, acc);
}

// Joins the partial sums of the run that goes out of chunk blockIdx.x, if one starts there: 128 vectors of the width by four
// groups of the chunks it goes through, whose number the CTA counts first, so that the loads do not wait for one another.
constexpr int kJoinThreads = 512;
constexpr int kJoinGroups = kJoinThreads / 128;
__global__ void __launch_bounds__(kJoinThreads) embed_join_kernel(const __grid_constant__ EmbedGrad a) {
    __shared__ float red[kJoinGroups - 1][8][128];
    launch_dependents();
    grid_dependency_wait();
    const int first = blockIdx.x, p0 = first * a.chunk, p1 = p0 + a.chunk;
    if (p1 >= a.n) return;                                               // nothing goes out of the last chunk
    const int token = ld_dep(a.sorted + p1 - 1).y, next = ld_dep(a.sorted + p1).y;
    const int here = ld_dep(a.sorted + p0).y, before = p0 > 0 ? ld_dep(a.sorted + p0 - 1).y : -1;
    if (token != next || token >= a.V || (here == token && before == token)) return;       // no run crosses the border, or it started earlier
    int through = 0;                                                     // chunks after this one that begin with the token
    for (;;) {
        const int k = first + 1 + through + (int)threadIdx.x;
        const int more = __syncthreads_count(k < a.n_chunks && ld_dep(a.sorted + (size_t)(k < a.n_chunks ? k : first) * a.chunk).y == token);
        through += more;
        if (more < kJoinThreads) break;
    }
    const int v = threadIdx.x & 127, group = threadIdx.x >> 7;
    const int c = blockIdx.y * 128 + v;
    float acc[8] = {};
    if (c < a.nvec) {
        auto add = [&](int chunk, int which) {
            const float4* in = reinterpret_cast<const float4*>(a.parts + ((size_t)chunk * 2 + which) * a.nvec * 8) + 2 * c;
            const float4 x = ld_dep(in), y = ld_dep(in + 1);
            acc[0] += x.x; acc[1] += x.y; acc[2] += x.z; acc[3] += x.w;
            acc[4] += y.x; acc[5] += y.y; acc[6] += y.z; acc[7] += y.w;
        };
        if (group == 0) add(first, 1);
#pragma unroll 8
        for (int k = 1 + group; k <= through; k += kJoinGroups) add(first + k, 0);
    }
    if (group > 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) red[group - 1][j][v] = acc[j];
    }
    __syncthreads();
    if (group == 0 && c < a.nvec) {
#pragma unroll
        for (int k = 0; k < kJoinGroups - 1; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += red[k][j][v];
        store_row(a, token, c, acc);
    }
}

// Lists of up to kShortMax tokens are not sorted: the CTA of position i (per 128 vectors of the width) finds out whether its token came
// earlier in the list, and if not adds up the rows of all positions that have it, four groups of threads taking every fourth of
// them and joining in order.  Two launches instead of four; where the table is cleared, all but the last stores run beside that.
// 257 tokens x 520 into 32003 rows of fp32: 11.5 us instead of 18 (floor 10.3), added to what is there 3.3; 512 tokens x 1024 4.9 us and
// 14.5 if they are all the same one, where sorting takes 13.4 and 14.4 for 513.  It lets nothing start early, for the clearing's sake.
constexpr int kShortMax = 512;
constexpr int kShortThreads = 512, kShortGroups = kShortThreads / 128;
__global__ void __launch_bounds__(kShortThreads) embed_short_kernel(const __grid_constant__ EmbedGrad a, const int* tokens, int beside_clear) {
    __shared__ float red[kShortGroups - 1][8][128];
    __shared__ int list[kShortMax];
    __shared__ int counts[kShortThreads / 32];
    if (!beside_clear) grid_dependency_wait();                           // beside it: the clearing kernel has waited
    const int i = threadIdx.x, lane = i & 31, warp = i >> 5;
    const int token = ld_dep(tokens + blockIdx.x);
    const bool same = i < a.n && ld_dep(tokens + i) == token;
    const unsigned ballot = __ballot_sync(0xffffffffu, same);
    if (lane == 0) counts[warp] = __popc(ballot);
    if (__syncthreads_or((same && i < (int)blockIdx.x) || (unsigned)token >= (unsigned)a.V)) {
        if (beside_clear) grid_dependency_wait();                        // the kernel's end is that of the clearing too
        return;
    }
    int at = __popc(ballot & ((1u << lane) - 1u)), count = 0;
    for (int w = 0; w < kShortThreads / 32; ++w) {
        at += w < warp ? counts[w] : 0;
        count += counts[w];
    }
    if (same) list[at] = i;
    __syncthreads();
    const int v = i & 127, group = i >> 7, c = blockIdx.y * 128 + v;
    const bool live = c < a.nvec;
    float acc[8] = {};
    if (live) {
#pragma unroll 1
        for (int k0 = group; k0 < count; k0 += kShortGroups * kSumAhead) {
            uint4 x[kSumAhead];
#pragma unroll
            for (int k = 0; k < kSumAhead; ++k)
                if (k0 + k * kShortGroups < count)
                    x[k] = ld_dep(reinterpret_cast<const uint4*>(a.dout + (size_t)list[k0 + k * kShortGroups] * a.ld_dout) + c);
#pragma unroll
            for (int k = 0; k < kSumAhead; ++k) {
                if (k0 + k * kShortGroups >= count) break;
                float f[8];
                unpack8f(x[k], f);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += f[j];
            }
        }
    }
    if (count > 1) {                                                     // the same for the whole CTA
        if (group > 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) red[group - 1][j][v] = acc[j];
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int k = 0; k < kShortGroups - 1; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += red[k][j][v];
        }
    }
    if (beside_clear) grid_dependency_wait();                            // the table is clear
    if (group == 0 && live) store_row(a, token, c, acc);
}

// Sorted positions per chunk: at most 1024 chunks (a run over all of them is joined by four groups of 256), at least eight
// positions (a thread's loads in flight).
int chunk_of(int n) { const int c = (n + 1023) / 1024; return c < 8 ? 8 : c; }

bool sorts_in_one_cluster(int n, int V) { return n <= kSortMax && V <= kSortMaxV; }

struct EmbedSpace {
    size_t a, b, scratch, parts, total;
};
EmbedSpace embed_space(int n, int d, int V) {
    EmbedSpace s;
    size_t at = 0;
    auto take = [&](size_t k) { const size_t o = at; at = align_up(at + k, 256); return o; };
    const bool one = sorts_in_one_cluster(n, V);
    const int chunk = chunk_of(n), n_chunks = (n + chunk - 1) / chunk;
    s.a = take((size_t)n * 8);
    s.b = take(one ? 0 : (size_t)n * 8);
    s.scratch = take(one ? 0 : sort_words_scratch_bytes(n));
    s.parts = take((size_t)n_chunks * 2 * d * 4);
    s.total = at > 256 ? at : 256;
    return s;
}

}  // namespace

ee_status embed_launch(const void* table, int V, int d, const int* tokens, int n, float scale, void* out, long long ld_out, int num_sms,
                       cudaStream_t stream) {
    const long long total = (long long)n * (d / 8);
    const long long want = (total + 255) / 256, most = (long long)num_sms * 8;
    return launch_pdl(embed_kernel, dim3((unsigned)(want < most ? want : most)), 256, 0, stream, static_cast<const __nv_bfloat16*>(table), V, d / 8,
                      tokens, n, scale, static_cast<__nv_bfloat16*>(out), ld_out) == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

size_t embed_grad_workspace_bytes(int n, int d, int V) { return embed_space(n, d, V).total; }

ee_status embed_grad_launch(const void* dout, long long ld_dout, const int* tokens, int n, int V, int d, float scale, void* dtable, int wide,
                            int accumulate, void* workspace, int num_sms, cudaStream_t stream) {
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    const EmbedSpace s = embed_space(n, d, V);
    const long long clear_vecs = accumulate ? 0 : (long long)V * d * (wide ? 4 : 2) / 16;
    int bits = 1;                                                        // tokens 0 .. V (V: takes no part)
    while (bits < 31 && (V >> bits) != 0) ++bits;
    const int passes = (bits + 7) / 8;
    EmbedGrad g;
    g.dout = static_cast<const __nv_bfloat16*>(dout); g.ld_dout = ld_dout;
    g.n = n; g.V = V; g.nvec = d / 8;
    g.chunk = chunk_of(n); g.n_chunks = (n + g.chunk - 1) / g.chunk;
    g.scale = scale; g.dtable = dtable; g.wide = wide; g.add = accumulate;
    g.parts = reinterpret_cast<float*>(ws + s.parts);
    g.sorted = nullptr;
    const long long copies = (clear_vecs * 16 + kClearBytes - 1) / kClearBytes, most = 4LL * num_sms;
    const dim3 clear_ctas((unsigned)(copies < most ? copies : most));
    if (n <= kShortMax) {
        if (clear_vecs) {
            embed_clear_kernel<<<clear_ctas, 128, 0, stream>>>(static_cast<uint4*>(dtable), clear_vecs);
            if (cudaGetLastError() != cudaSuccess) return EE_ERR_CUDA;
        }
        return launch_pdl(embed_short_kernel, dim3(n, (g.nvec + 127) / 128), kShortThreads, 0, stream, g, tokens, clear_vecs ? 1 : 0) == cudaSuccess
                   ? EE_OK : EE_ERR_CUDA;
    }
    if (sorts_in_one_cluster(n, V)) {
        int2* sorted = reinterpret_cast<int2*>(ws + s.a);
        cudaLaunchConfig_t cfg;
        cudaLaunchAttribute attr[2];
        pair_launch_config(cfg, attr, dim3(kSortCtas), kSortThreads, 0, stream);
        attr[1].val.clusterDim.x = kSortCtas;
        if (cudaLaunchKernelEx(&cfg, embed_sort_kernel, tokens, n, V, passes, sorted) != cudaSuccess) return EE_ERR_CUDA;
        if (clear_vecs && launch_pdl(embed_clear_kernel, clear_ctas, 128, 0, stream, static_cast<uint4*>(dtable), clear_vecs) != cudaSuccess) return EE_ERR_CUDA;
        g.sorted = sorted;
    } else {
        u64 *a = reinterpret_cast<u64*>(ws + s.a), *b = reinterpret_cast<u64*>(ws + s.b);
        if (clear_vecs && cudaMemsetAsync(dtable, 0, (size_t)clear_vecs * 16, stream) != cudaSuccess) return EE_ERR_CUDA;
        embed_words_kernel<<<(n + 255) / 256, 256, 0, stream>>>(tokens, n, V, a);
        if (cudaGetLastError() != cudaSuccess) return EE_ERR_CUDA;
        const u64* sorted = nullptr;
        const ee_status st = sort_words_launch(a, b, n, 32, passes, ws + s.scratch, &sorted, stream);
        if (st != EE_OK) return st;
        g.sorted = reinterpret_cast<const int2*>(sorted);
    }
    const int nvec = d / 8;
    if (launch_pdl(embed_sum_kernel, dim3(g.n_chunks, (nvec + kSumThreads - 1) / kSumThreads), kSumThreads, 0, stream, g) != cudaSuccess ||
        launch_pdl(embed_join_kernel, dim3(g.n_chunks, (nvec + 127) / 128), kJoinThreads, 0, stream, g) != cudaSuccess)
        return EE_ERR_CUDA;
    return EE_OK;
}

}  // namespace ee
