// Losses over the tokens of sequences, between ee_head_ce, which gives every token's cross-entropy ce = -ln p, and ee_head_ce_grad, which
// takes every token's weight: the clipped policy loss with a penalty for leaving a reference, and the loss of preferred and rejected
// sequences.  Each call is one launch that writes the weights and the means.
//
// The work is light -- 12 to 24 bytes and some twenty operations per token -- so that what counts is the shape: a mean over each
// sequence's own tokens, or a sequence's sum, is needed before any of its weights.  A unit (a sequence, a pair of sequences, or, where
// all tokens count alike, a stretch of tokens) is therefore walked twice, the second time out of L1 or L2, by a warp where units are
// short, by a CTA where they are long, and by a cluster of eight or sixteen CTAs, which exchange their sums through distributed shared memory,
// where they are long and few.
//
// What decides or cancels is done in fp64, which costs little here: the difference of two cross-entropies before the comparison with the
// clip's border, and all sums, in a fixed order (a unit's by its threads, the units' by CTA, the CTAs' by the one that finishes last).
// Powers and what is made of them are fp32: the ratio, the divergence and its slope to some 2^-21 of themselves (infinite where the power leaves fp32, from
// an argument of 88.7 on), a pair's slope to 2^-22 of the larger of its two parts, which cancel where the margin is ln((1 - smoothing) / smoothing).
//
// Device times in a graph: policy loss of 512 tokens 3.1 us, of 65537 in 200 sequences 7.6; preference loss of 4001 tokens
// in 8 pairs 5.3, of 300000 in 3 pairs 15 (1024 threads per CTA: 16; eight instead of sixteen CTAs: 17.5; loops that test for their end between two loads:
// 19).  All of it is latency: reading and writing takes 0.8 us of the last one at the copy rate, the rest are start, two walks of some ten tokens
// a thread on 48 SMs, the exchange within the cluster and the last sums.
#include <cooperative_groups.h>

#include "common.cuh"
#include "kernels.h"

namespace ee {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256, kClusterThreads = 512, kMaxWarps = kClusterThreads / 32;
constexpr int kClusterCtas = 8, kWideClusterCtas = 16;
constexpr int kMaxCtas = 2048;
constexpr int kBatch = 8, kHalfBatch = 4;        // tokens whose loads a thread issues at once: a loop that tests for its end in between waits for each
constexpr int kSums = 4;

enum Span { kWarpSpan, kCtaSpan, kClusterSpan };         // what walks a unit
// Tokens of a unit above which a warp leaves it to its CTA, which takes 2 us for each.  Policy loss of 600 sequences of random lengths around 256, us: borders of
// 256, 512, 1024, 2048 19, 18, 18, 22, of 2400 around 512 29, 29, 31, 33; preference loss of 600 pairs around 512 23, 24, 17, 13, of 4800 around 1024 52, 47, 38, 33.
constexpr int kPolicyHandOver = 512, kPreferenceHandOver = 2048;

struct LossSpace {
    Control ctrl;
    double parts[kMaxCtas][kSums];
};

struct Term {
    float policy, kl, grad;
    bool cut;
};

// expm1(g) - g without the cancellation of small g: the series of g^2 (1/2 + g/6 + ...), whose next term is below 2^-26 of it.
__device__ __forceinline__ float expm1_minus(float g, float expm1_g) {
    if (fabsf(g) < 0.25f) {
        float s = 1.f / 40320.f;
        s = fmaf(s, g, 1.f / 5040.f);
        s = fmaf(s, g, 1.f / 720.f);
        s = fmaf(s, g, 1.f / 120.f);
        s = fmaf(s, g, 1.f / 24.f);
        s = fmaf(s, g, 1.f / 6.f);
        s = fmaf(s, g, 0.5f);
        return g * g * s;
    }
    return expm1_g - g;
}

__device__ __forceinline__ Term policy_term(const PolicyArgs& p, float ce, float old_ce, float ref_ce, float adv) {
    Term t;
    const double x = (double)old_ce - (double)ce;                        // ln of the ratio of the new to the old probability
    t.cut = adv > 0.f ? x > p.log_high : adv < 0.f && x < p.log_low;
    float ln_ratio = (float)x;
    if (adv == 0.f && ln_ratio > 0.f) ln_ratio = 0.f;                    // 0 times infinity: a token that asks for nothing, however far it has come
    const float ratio = expf(ln_ratio);
    t.policy = -adv * (t.cut ? (adv > 0.f ? p.high : p.low) : ratio);
    t.grad = t.cut ? 0.f : adv * ratio;
    t.kl = 0.f;
    if (p.ref_ce) {
        float g = (float)((double)ce - (double)ref_ce);
        g = g > 1e30f ? 1e30f : g;                                       // infinity less infinity: its divergence is infinite
        const float e = expm1f(g);
        t.kl = expm1_minus(g, e);
        if (p.kl_weight != 0.f) t.grad = fmaf(p.kl_weight, e, t.grad);   // 0 only watches the divergence, which may be infinite
    }
    return t;
}

__device__ __forceinline__ double total_loss(const PolicyArgs& p, double policy, double kl) {
    return p.kl_weight != 0.f ? fma((double)p.kl_weight, kl, policy) : policy;
}

__device__ __forceinline__ double warp_total(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The sums of v and w over the threads that walk a unit, the same in each of them.  Two arrays of shared memory take turns, so that one barrier
// (or two of the cluster) is enough.  Of a cluster each warp reads all CTAs' sums at once, one to a lane.
struct Slots {
    double2 of_warp[kMaxWarps], of_cta;
};
template <int kSpan>
__device__ __forceinline__ double2 span_totals(double v, double w, Slots (&slots)[2], int& turn) {
    constexpr int kWarps = (kSpan == kClusterSpan ? kClusterThreads : kThreads) / 32;
    const int lane = threadIdx.x & 31;
    double2 sum = make_double2(warp_total(v), warp_total(w));
    if (kSpan == kWarpSpan) return sum;
    Slots& slot = slots[turn];
    turn ^= 1;
    if (lane == 0) slot.of_warp[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = lane < kWarps ? slot.of_warp[lane] : make_double2(0.0, 0.0);
    sum = make_double2(warp_total(sum.x), warp_total(sum.y));
    if (kSpan == kCtaSpan) return sum;
    if (threadIdx.x == 0) slot.of_cta = sum;
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    sum = lane < (int)cluster.num_blocks() ? *cluster.map_shared_rank(&slot.of_cta, lane) : make_double2(0.0, 0.0);
    return make_double2(warp_total(sum.x), warp_total(sum.y));
}

// Four sums over the CTA's units, to the means: the CTA that finishes last adds up the CTAs'.
template <int kWarps>
__device__ __forceinline__ void finish(double (&sums)[kSums], LossSpace* space, float* loss) {
    __shared__ double warp_sums[kWarps][kSums];
    __shared__ int last;
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        const double v = warp_total(sums[k]);
        if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5][k] = v;
    }
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;          // warp k adds up sum k
    if (warp < kSums) {
        const double v = warp_total(lane < kWarps ? warp_sums[lane][warp] : 0.0);
        if (lane == 0 && gridDim.x == 1) loss[warp] = (float)v;
        if (lane == 0 && gridDim.x > 1) space->parts[blockIdx.x][warp] = v;
    }
    if (gridDim.x == 1) return;
    __syncthreads();
    if (threadIdx.x == 0) last = ticket_arrive_is_last(&space->ctrl.head_ticket[0], gridDim.x) ? 1 : 0;
    __syncthreads();
    if (!last) return;
    double total[kSums] = {};
    for (int b = threadIdx.x; b < (int)gridDim.x; b += 32 * kWarps) {
        const double2* part = reinterpret_cast<const double2*>(space->parts[b]);
        const double2 lo = __ldcg(part), hi = __ldcg(part + 1);
        total[0] += lo.x; total[1] += lo.y; total[2] += hi.x; total[3] += hi.y;
    }
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        const double v = warp_total(total[k]);
        if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5][k] = v;
    }
    __syncthreads();
    if (warp < kSums) {
        const double v = warp_total(lane < kWarps ? warp_sums[lane][warp] : 0.0);
        if (lane == 0) loss[warp] = (float)v;
    }
    if (threadIdx.x == 0) space->ctrl.head_ticket[0] = 0;                // ready for the next launch
}

// Boundaries of sequences are data: brought into the range of the rows, whatever they say.
__device__ __forceinline__ int boundary(const int* seq_start, int i, int M) { return min(max(ld_dep(seq_start + i), 0), M); }

// Rows before the first sequence and behind the last belong to none: their weight is zero.
__device__ __forceinline__ void clear_outside(const int* seq_start, int n, int M, float* dce) {
    const int first = boundary(seq_start, 0, M), end = max(boundary(seq_start, n, M), first);
    const long long stride = (long long)gridDim.x * blockDim.x, at = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    for (long long i = at; i < first; i += stride) dce[i] = 0.f;
    for (long long i = end + at; i < M; i += stride) dce[i] = 0.f;
}

__device__ __forceinline__ bool is_counted(const int* labels, long long i, int V) { return (unsigned)ld_dep(labels + i) < (unsigned)V; }

// All tokens count alike.
__global__ void __launch_bounds__(kThreads) policy_tokens_kernel(const PolicyArgs p) {
    launch_dependents();
    grid_dependency_wait();
    const float n = ld_dep(p.counted + 1);
    const double w = n > 0.f ? 1.0 / (double)n : 0.0;
    const float wf = (float)w;
    double sums[kSums] = {};
    const long long stride = (long long)gridDim.x * kThreads;
    for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < p.M; i += stride) {
        float d = 0.f;
        const float ce = ld_dep(p.ce + i), old_ce = ld_dep(p.old_ce + i), adv = ld_dep(p.adv + i), ref = p.ref_ce ? ld_dep(p.ref_ce + i) : 0.f;
        if (is_counted(p.labels, i, p.V)) {
            const Term t = policy_term(p, ce, old_ce, ref, adv);
            d = wf * t.grad;
            sums[1] += (double)t.policy;
            sums[2] += (double)t.kl;
            sums[3] += t.cut ? 1.0 : 0.0;
        }
        p.dce[i] = d;
    }
#pragma unroll
    for (int k = 1; k < kSums; ++k) sums[k] *= w;
    sums[0] = total_loss(p, sums[1], sums[2]);
    finish<kThreads / 32>(sums, reinterpret_cast<LossSpace*>(p.workspace), p.loss);
}

template <int kValue>
struct IntConstant {
    static constexpr int value = kValue;
};

// Which units a thread has part in, and where in them it begins and how far it steps.
template <int kSpan>
constexpr int threads_of = kSpan == kClusterSpan ? kClusterThreads : kThreads;
template <int kSpan>
struct Walk {
    static constexpr int kThreads = threads_of<kSpan>, kWarps = kThreads / 32;
    int unit, units_step, from, step;
    __device__ __forceinline__ Walk() {
        if (kSpan == kWarpSpan) {
            unit = blockIdx.x * kWarps + (threadIdx.x >> 5);
            units_step = gridDim.x * kWarps;
            from = threadIdx.x & 31;
            step = 32;
        } else if (kSpan == kCtaSpan) {
            unit = blockIdx.x;
            units_step = gridDim.x;
            from = threadIdx.x;
            step = kThreads;
        } else {
            const int ctas = (int)cg::this_cluster().num_blocks();
            unit = blockIdx.x / ctas;
            units_step = gridDim.x / ctas;
            from = (blockIdx.x % ctas) * kThreads + threadIdx.x;
            step = ctas * kThreads;
        }
    }
};

// Calls walk_unit(IntConstant<span>, unit, its rows (begin and end), from, step) for every unit that the thread has part in.  Among units that warps walk
// one of more than `hand_over` rows is left to the whole CTA, after the warps' own.
template <int kSpan, class Bounds, class WalkUnit>
__device__ __forceinline__ void for_units(int units, int hand_over, const Bounds& bounds, const WalkUnit& walk_unit) {
    const Walk<kSpan> walk;
    if constexpr (kSpan == kWarpSpan) {
        constexpr int kWarps = Walk<kSpan>::kWarps;
        __shared__ int2 spans[kWarps];                                   // read once: what threads decide to walk together they decide alike
        const int warp = threadIdx.x >> 5;
        for (int first = blockIdx.x * kWarps; first < units; first += walk.units_step) {
            const int unit = first + warp;
            int2 b = unit < units ? bounds(unit) : make_int2(0, 0);
            b.x = __shfl_sync(0xffffffffu, b.x, 0);
            b.y = __shfl_sync(0xffffffffu, b.y, 0);
            if (walk.from == 0) spans[warp] = b;
            const bool is_long = b.y - b.x > hand_over;
            if (unit < units && !is_long) walk_unit(IntConstant<kWarpSpan>{}, unit, b, walk.from, walk.step);
            if (!__syncthreads_or(is_long ? 1 : 0)) continue;
            for (int w = 0; w < kWarps; ++w) {
                const int2 whole = spans[w];
                if (whole.y - whole.x > hand_over) walk_unit(IntConstant<kCtaSpan>{}, first + w, whole, (int)threadIdx.x, kThreads);
            }
            __syncthreads();
        }
    } else {
        for (int unit = walk.unit; unit < units; unit += walk.units_step) walk_unit(IntConstant<kSpan>{}, unit, bounds(unit), walk.from, walk.step);
    }
}

// Every sequence counts alike, and within a sequence every token.  (Rows are at most 2^30, so that 32 bits hold every index here and below.)
template <int kSpan>
__device__ __forceinline__ void policy_unit(const PolicyArgs& p, int unit, int begin, int end, int from, int step, Slots (&slots)[2], int& turn,
                                            double (&sums)[kSums]) {
    const float adv = ld_dep(p.adv + unit);
    int have = 0;
    for (int i0 = begin + from; i0 < end; i0 += kBatch * step) {
        bool in[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) in[u] = i0 + u * step < end && is_counted(p.labels, i0 + u * step, p.V);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) have += in[u] ? 1 : 0;
    }
    const double n = span_totals<kSpan>((double)have, 0.0, slots, turn).x;
    const double w = n > 0.0 ? 1.0 / (n * (double)p.S) : 0.0;
    const float wf = (float)w;
    double policy = 0.0, kl = 0.0, cut = 0.0;
    for (int i0 = begin + from; i0 < end; i0 += kHalfBatch * step) {
        float ce[kHalfBatch], old_ce[kHalfBatch], ref[kHalfBatch];
        bool in[kHalfBatch];
#pragma unroll
        for (int u = 0; u < kHalfBatch; ++u) {
            const int i = i0 + u * step;
            ce[u] = i < end ? ld_dep(p.ce + i) : 0.f;
            old_ce[u] = i < end ? ld_dep(p.old_ce + i) : 0.f;
            ref[u] = i < end && p.ref_ce ? ld_dep(p.ref_ce + i) : 0.f;
            in[u] = i < end && is_counted(p.labels, i, p.V);
        }
#pragma unroll
        for (int u = 0; u < kHalfBatch; ++u) {
            float d = 0.f;
            if (in[u]) {
                const Term t = policy_term(p, ce[u], old_ce[u], ref[u], adv);
                d = wf * t.grad;
                policy += (double)t.policy;
                kl += (double)t.kl;
                cut += t.cut ? 1.0 : 0.0;
            }
            if (i0 + u * step < end) p.dce[i0 + u * step] = d;
        }
    }
    if (n > 0.0) {
        sums[1] = fma(w, policy, sums[1]);
        sums[2] = fma(w, kl, sums[2]);
        sums[3] = fma(w, cut, sums[3]);
    }
}

template <int kSpan>
__global__ void __launch_bounds__(threads_of<kSpan>) policy_sequences_kernel(const PolicyArgs p) {
    __shared__ Slots slots[2];
    launch_dependents();
    grid_dependency_wait();
    clear_outside(p.seq_start, p.S, p.M, p.dce);
    double sums[kSums] = {};
    int turn = 0;
    for_units<kSpan>(
        p.S, kPolicyHandOver, [&](int unit) { return make_int2(boundary(p.seq_start, unit, p.M), boundary(p.seq_start, unit + 1, p.M)); },
        [&](auto span, int unit, int2 b, int from, int step) { policy_unit<decltype(span)::value>(p, unit, b.x, b.y, from, step, slots, turn, sums); });
    sums[0] = total_loss(p, sums[1], sums[2]);
    if (kSpan == kClusterSpan) cg::this_cluster().sync();                // nobody leaves while its sums may still be read
    finish<threads_of<kSpan> / 32>(sums, reinterpret_cast<LossSpace*>(p.workspace), p.loss);
}

// A thread's part of the sum of a sequence's gains, rows first, first + step, .. below end, and which of its first 64 tokens are counted, so that
// their labels are read once.
__device__ __forceinline__ double gains(const PreferenceArgs& p, int first, int end, int step, unsigned long long& counted) {
    double sum = 0.0;
    int k = 0;
    counted = 0;
    for (int i0 = first; i0 < end; i0 += kBatch * step, k += kBatch) {
        float ce[kBatch], ref[kBatch];
        bool in[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {                               // the loads of a batch at once
            const int i = i0 + u * step;
            ce[u] = i < end ? ld_dep(p.ce + i) : 0.f;
            ref[u] = i < end && p.ref_ce ? ld_dep(p.ref_ce + i) : 0.f;
            in[u] = i < end && is_counted(p.labels, i, p.V);
        }
        unsigned bits = 0;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            bits |= in[u] ? 1u << u : 0u;
            sum += in[u] ? (double)ref[u] - (double)ce[u] : 0.0;
        }
        if (k < 64) counted |= (unsigned long long)bits << k;
    }
    return sum;
}
__device__ __forceinline__ void put_weights(const PreferenceArgs& p, int first, int end, int step, unsigned long long counted, float d) {
    int k = 0;
    for (int i0 = first; i0 < end; i0 += kBatch * step, k += kBatch) {
        const unsigned bits = (unsigned)(counted >> (k & 63));
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int i = i0 + u * step;
            if (i < end) p.dce[i] = (k < 64 ? (bits >> u & 1u) != 0 : is_counted(p.labels, i, p.V)) ? d : 0.f;
        }
    }
}

// Pairs of sequences 2u (preferred) and 2u + 1 (rejected).
template <int kSpan>
__device__ __forceinline__ void preference_unit(const PreferenceArgs& p, int unit, int begin, int end, int from, int step, Slots (&slots)[2], int& turn,
                                                double (&sums)[kSums]) {
    const int middle = max(boundary(p.seq_start, 2 * unit + 1, p.M), begin);
    unsigned long long counted[2];                                       // of the thread's first 64 tokens of each sequence
    const double first = gains(p, begin + from, middle, step, counted[0]), second = gains(p, middle + from, end, step, counted[1]);
    const double2 sum = span_totals<kSpan>(first, second, slots, turn);
    const double good = (double)p.beta * sum.x, bad = (double)p.beta * sum.y;
    // with t = e^-|m|: -ln sigma(m) = ln(1 + t) + max(-m, 0), and sigma(m) is 1 / (1 + t) or t / (1 + t)
    const double margin = good - bad;
    const float m = (float)margin, t = expf(-fabsf(m)), near = 1.f / (1.f + t), far = t * near;
    const float up = log1pf(t) + fmaxf(-m, 0.f), down = log1pf(t) + fmaxf(m, 0.f);
    const float slope = p.smoothing * (m >= 0.f ? near : far) - (1.f - p.smoothing) * (m >= 0.f ? far : near);
    const float d = (float)((double)p.beta * (double)slope * p.share);
    if (from == 0) {
        p.margin[unit] = m;
        sums[0] += (double)((1.f - p.smoothing) * up + (p.smoothing > 0.f ? p.smoothing * down : 0.f));
        sums[1] += m > 0.f ? 1.0 : 0.0;
        sums[2] += good;
        sums[3] += bad;
    }
    put_weights(p, begin + from, middle, step, counted[0], -d);
    put_weights(p, middle + from, end, step, counted[1], d);
}

template <int kSpan>
__global__ void __launch_bounds__(threads_of<kSpan>) preference_kernel(const PreferenceArgs p) {
    __shared__ Slots slots[2];
    launch_dependents();
    grid_dependency_wait();
    clear_outside(p.seq_start, 2 * p.P, p.M, p.dce);
    double sums[kSums] = {};
    int turn = 0;
    for_units<kSpan>(
        p.P, kPreferenceHandOver,
        [&](int unit) {
            const int begin = boundary(p.seq_start, 2 * unit, p.M), middle = max(boundary(p.seq_start, 2 * unit + 1, p.M), begin);
            return make_int2(begin, max(boundary(p.seq_start, 2 * unit + 2, p.M), middle));
        },
        [&](auto span, int unit, int2 b, int from, int step) { preference_unit<decltype(span)::value>(p, unit, b.x, b.y, from, step, slots, turn, sums); });
#pragma unroll
    for (int k = 0; k < kSums; ++k) sums[k] *= p.share;
    if (kSpan == kClusterSpan) cg::this_cluster().sync();
    finish<threads_of<kSpan> / 32>(sums, reinterpret_cast<LossSpace*>(p.workspace), p.loss);
}

// What walks a unit, by the units' average length and their number.  A warp needs no exchange and starts soonest, but takes 10.7 ns for a token of
// the policy loss and 4.1 of the preference loss, whose two sequences overlap; a CTA takes 1.2 and 0.8, and as more of them queue than SMs, it pays
// the later the more units there are; a cluster of eight costs 3 us to start and 0.2 us more for every unit.  How far the longest is from the average
// is on the device and decides as much: the borders are between those of equal units and of units cut at random places (the longest six times the average).
// Device times, us, equal / random; policy loss:
//   units of      8: 64 a warp 3.3 / 4.6, a CTA 4.3 / 4.5;  256 5.0 / 10.7, 4.5 / 4.7;   1024 a CTA 5.0 / 7.2, a cluster 7.4 / 7.2;  2048 6.1 / 10.2, 7.3 / 7.5
//                36: 32 4.6 / 5.8, 4.5 / 4.8;  64 4.8 / 7.3, 4.7 / 4.9;                   2048 6.7 / 15.3, 15.2 / 14.8;  4096 8.8 / 26.7, 15.3 / 15.2
//               148: 64 5.1 / 6.3, 5.0 / 5.2;  128 5.5 / 9.1, 5.1 / 5.3;                  8192 14 / 42, 40 / 40;  16384 24 / 79, 44 / 46
//               600: 128 5.7 / 11.9, 8.5 / 9.3;  256 6.8 / 18.3, 9.0 / 10.3      2400: 256 10.6 / 20.1, 17.0 / 18.0;  512 15.8 / 27.8, 18.7 / 22.6
// preference loss:
//                 8: 128 4.1 / 4.3, 5.1 / 5.1;  256 4.3 / 5.5, 5.1 / 5.3;                 2048 5.8 / 7.0, 8.6 / 8.6;  4096 6.6 / 9.2, 8.8 / 8.8
//                36: 128 5.6 / 6.4, 5.5 / 5.5;  256 5.8 / 7.6, 5.5 / 5.7;                 4096 6.8 / 12.9, 16.0 / 15.2;  8192 9.6 / 21.2, 16.1 / 15.6
//               148: 256 6.2 / 8.2, 5.8 / 6.0;  512 6.4 / 11.0, 5.9 / 6.2;                16384 15 / 55, 41 / 42;  32768 41 / 131, 47 / 53
//               600: 512 6.4 / 12.7, 10.8 / 10.9;  1024 8.8 / 24.6, 11.3 / 11.7  2400: 1024 12.3 / 26.1, 23.5 / 24.6;  2048 21.8 / 46.1, 27.9 / 33.4
// A long unit among many short ones goes from its warp to its CTA (kPolicyHandOver, kPreferenceHandOver): 600 sequences of random lengths around 256 take
// 18 us instead of 22, 600 pairs around 1024 25 instead of 34, 2000 sequences of 32 tokens with one of 100000 135 instead of 1040 (without it 6).  From a CTA
// nothing is handed on: 90 sequences of 300 and one of 300000 take 350 us.
struct Borders {                                 // average lengths from which a CTA or a cluster walks a unit: so many, and so many more for 16 units
    int cta, cta_more, cluster, cluster_more;
};
constexpr Borders kPolicyBorders{48, 3, 1024, 1024}, kPreferenceBorders{160, 12, 3072, 1536};

int span_of(int M, int units, int num_sms, const Borders& b) {
    const long long each = M / units, n = units;
    if (units <= num_sms && each >= b.cluster + b.cluster_more * n / 16) return kClusterSpan;
    return each >= b.cta + b.cta_more * n / 16 ? kCtaSpan : kWarpSpan;
}

// Clusters of sixteen CTAs instead of eight where units are long and few.  Eight and sixteen, equal / random, policy loss: 1 unit of 16384 7.2, 7.4, of
// 131072 18.6, 12.9; 4 of 32768 9.4 / 15.4, 9.2 / 12.3, of 131072 19 / 43, 14 / 26; 8 of 32768 9.6 / 15.0, 12.7 / 13.6, of 131072 19 / 39, 21 / 25; 12 of 131072
// 27 / 61, 21 / 37.  Preference loss: 1 of 16384 8.0, 8.6; 4 of 65536 11.7 / 14.4, 10.7 / 12.2; 8 of 32768 10.2 / 12.0, 14.5 / 14.5, of 131072 17 / 26, 17 / 20.
bool is_wide(int M, int units) { return M / units >= 8192ll * (units + 2); }

// How many clusters of sixteen CTAs of this kernel (`kind`: which of the two it is) the device runs at once; 0 if it cannot.
int wide_clusters(const void* kernel, int kind, int device) {
    static int clusters[2][kMaxDevices];
    static bool asked[2][kMaxDevices] = {};
    if (!asked[kind][device]) {
        int n = 0;
        cudaLaunchConfig_t cfg;
        cudaLaunchAttribute attr[2];
        pair_launch_config(cfg, attr, dim3(kWideClusterCtas), kClusterThreads, 0, nullptr);
        attr[1].val.clusterDim.x = kWideClusterCtas;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
            n = 0;
            (void)cudaGetLastError();
        }
        clusters[kind][device] = n;
        asked[kind][device] = true;
    }
    return clusters[kind][device];
}

template <class Args>
cudaError_t launch_spans(int kind, void (*warp)(Args), void (*cta)(Args), void (*cluster)(Args), const Args& p, const Borders& borders, int M, int units,
                         int num_sms, int device, cudaStream_t stream) {
    const int most = kMaxCtas < 8 * num_sms ? kMaxCtas : 8 * num_sms;
    switch (span_of(M, units, num_sms, borders)) {
        case kWarpSpan: {
            const int grid = (units + kThreads / 32 - 1) / (kThreads / 32);
            return launch_pdl(warp, dim3(grid < most ? grid : most), kThreads, 0, stream, p);
        }
        case kCtaSpan: return launch_pdl(cta, dim3(units < most ? units : most), kThreads, 0, stream, p);
        default: {
            const bool wide = is_wide(M, units) && units <= wide_clusters(reinterpret_cast<const void*>(cluster), kind, device);
            const int ctas = wide ? kWideClusterCtas : kClusterCtas;
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute attr[2];
            pair_launch_config(cfg, attr, dim3(units * ctas), kClusterThreads, 0, stream);
            attr[1].val.clusterDim.x = ctas;
            return cudaLaunchKernelEx(&cfg, cluster, p);
        }
    }
}

}  // namespace

size_t token_loss_workspace_bytes() { return sizeof(LossSpace); }

ee_status policy_loss_launch(const PolicyArgs& p, int num_sms, int device, cudaStream_t stream) {
    cudaError_t e;
    if (p.seq_start) {
        e = launch_spans<PolicyArgs>(0, policy_sequences_kernel<kWarpSpan>, policy_sequences_kernel<kCtaSpan>, policy_sequences_kernel<kClusterSpan>, p,
                                     kPolicyBorders, p.M, p.S, num_sms, device, stream);
    } else {
        const long long need = ((long long)p.M + kThreads - 1) / kThreads;
        const int most = kMaxCtas < 8 * num_sms ? kMaxCtas : 8 * num_sms;
        e = launch_pdl(policy_tokens_kernel, dim3(need < most ? (int)need : most), kThreads, 0, stream, p);
    }
    return e == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

ee_status preference_loss_launch(const PreferenceArgs& p, int num_sms, int device, cudaStream_t stream) {
    return launch_spans<PreferenceArgs>(1, preference_kernel<kWarpSpan>, preference_kernel<kCtaSpan>, preference_kernel<kClusterSpan>, p, kPreferenceBorders,
                                        p.M, p.P, num_sms, device, stream) == cudaSuccess ? EE_OK : EE_ERR_CUDA;
}

}  // namespace ee
