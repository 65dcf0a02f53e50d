// Tokens from logits and given random numbers, and the branch of a drafted tree that agrees with given answers.
//
// A row's tokens stand in order: largest logit first, the lowest index first among equals.  With top the largest logit,
//   w_i = 2^44 exp((x_i - top) / temperature), rounded to a whole number,
// and a token is drawn with a probability that is proportional to w among the tokens that are kept, which are the first ones of the order: no more
// than top_k; the fewest that have top_p of the weight of those; those with w >= min_p 2^44; the first one always.
// Drawn is the first token at which the sum of the weights in that order exceeds u times the kept ones' sum.
//
// Weights are whole numbers so that their sums do not depend on the order in which they are formed: any division of the work, and
// atomics in LDS too, give the same tokens.  2^-44 is far below what a random number of 24 bits can tell apart; 2^19 tokens'
// sums fit 64 bits.
//
// Every question (the k-th token, the token at a given weight) is one about places in the order, answered from a histogram with counts and
// weights; then from one over the keys of the bin where the answer lies, until that is one key.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svdp_device.h"
#include "svdp_order.h"

namespace svdp {

constexpr int SAMPLE_THREADS = 1024, SAMPLE_WAVES = SAMPLE_THREADS / 64;
constexpr int SAMPLE_BINS = SAMPLE_THREADS;
constexpr double SAMPLE_UNIT = 17592186044416.0;            // 2^44
constexpr int SAMPLE_MAX_V = 1 << 19;

struct SampleArgs {
    const void *logits;
    int64_t stride;
    const float *u, *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p;
    int32_t *answers;
    float *logp;
    int V;
};

__device__ __forceinline__ float of_order(uint32_t o)
{
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

// f(value, index) for the elements of a row that a thread has; vectors of 16 bytes but at the row's ends.
template <typename W, typename F>
__device__ __forceinline__ void each_logit(const W *row, int V, int tid, int threads, F &&f)
{
    constexpr int VEC = Elem<W>::VEC, AHEAD = 4;
    const int skew = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / Elem<W>::BYTES);
    const int head = min(skew > 0 ? VEC - skew : 0, V), vectors = (V - head) / VEC, tail = head + vectors * VEC;
    for (int i0 = tid; i0 < vectors; i0 += AHEAD * threads) {
        uint4 in[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) in[a] = load_raw(row + head + (int64_t)min(i0 + a * threads, vectors - 1) * VEC);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int i = i0 + a * threads;
            if (i >= vectors) break;
            float v[VEC];
            widen(in[a], v, row);
#pragma unroll
            for (int j = 0; j < VEC; ++j) f(v[j], head + i * VEC + j);
        }
    }
    if (tid < head) f(to_f32(row[tid]), tid);
    if (tail + tid < V) f(to_f32(row[tail + tid]), tail + tid);
}

// Counts and weights of bins; after sums() those of a bin and all before it.
struct SampleBins {
    uint64_t weight[SAMPLE_BINS];
    uint32_t count[SAMPLE_BINS];
};
struct SampleShared {
    SampleBins first, fine;
    uint64_t wave_weight[SAMPLE_WAVES];
    uint64_t wave_key[SAMPLE_WAVES];
    uint32_t wave_count[SAMPLE_WAVES], wave_low[SAMPLE_WAVES];
    uint64_t before_weight, bin_weight;
    uint32_t before_count, bin_count;
    int bin;
    int index;
};

__device__ __forceinline__ uint64_t wave_sums_u64(uint64_t v, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t o = __shfl_up((unsigned long long)v, d);
        v += lane >= d ? o : 0;
    }
    return v;
}
__device__ __forceinline__ void sample_clear(SampleBins &b, int tid)
{
    b.weight[tid] = 0;
    b.count[tid] = 0;
}
// Inclusive sums over the bins.
__device__ __forceinline__ void sample_sums(SampleShared &s, SampleBins &b, int tid)
{
    const int lane = tid & 63, wave = tid >> 6;
    __syncthreads();
    const uint64_t w = wave_sums_u64(b.weight[tid], lane);
    const uint32_t c = (uint32_t)wave_inclusive_scan((int)b.count[tid]);
    if (lane == 63) {
        s.wave_weight[wave] = w;
        s.wave_count[wave] = c;
    }
    __syncthreads();
    uint64_t w0 = 0;
    uint32_t c0 = 0;
    for (int i = 0; i < wave; ++i) {
        w0 += s.wave_weight[i];
        c0 += s.wave_count[i];
    }
    b.weight[tid] = w0 + w;
    b.count[tid] = c0 + c;
    __syncthreads();
}
// A place in the order: the bin, or in the end the key, at which count (or weight) reaches `need`, with what is before it and in it.
struct SamplePlace {
    uint32_t key, before_count, count;
    uint64_t before_weight, weight;
};
__device__ __forceinline__ int sample_find(SampleShared &s, const SampleBins &b, bool by_count, uint64_t need, int tid, SamplePlace &p)
{
    const uint64_t w0 = tid > 0 ? b.weight[tid - 1] : 0, w1 = b.weight[tid];
    const uint32_t c0 = tid > 0 ? b.count[tid - 1] : 0, c1 = b.count[tid];
    if (by_count ? (c0 < need && need <= c1) : (w0 < need && need <= w1)) {
        s.bin = tid;
        s.before_weight = w0;
        s.before_count = c0;
        s.bin_weight = w1 - w0;
        s.bin_count = c1 - c0;
    }
    __syncthreads();
    const int bin = s.bin;
    p.before_weight += s.before_weight;
    p.before_count += s.before_count;
    p.weight = s.bin_weight;
    p.count = s.bin_count;
    __syncthreads();
    return bin;
}

// One block a row.
template <typename W>
__global__ __launch_bounds__(SAMPLE_THREADS) void k_sample(SampleArgs A)
{
    __shared__ SampleShared s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, t = blockIdx.x;
    const W *row = static_cast<const W *>(A.logits) + (int64_t)t * A.stride;
    const float temperature = A.temperature != nullptr ? A.temperature[t] : 1.f, top_p = A.top_p != nullptr ? A.top_p[t] : 1.f;
    const float min_p = A.min_p != nullptr ? A.min_p[t] : 0.f;
    const int top_k = A.top_k != nullptr ? A.top_k[t] : 0;

    // the first token of the order, and the smallest finite logit
    uint64_t best = 0;
    uint32_t low = 0xffffffffu;
    each_logit(row, A.V, tid, SAMPLE_THREADS, [&](float x, int i) {
        const uint64_t key = best_key(x, i);
        best = key > best ? key : best;
        const uint32_t o = (uint32_t)(key >> 32);
        low = o > best_order(-INFINITY) && o < low ? o : low;
    });
    best = wave_max_u64(best);
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) low = min(low, (uint32_t)__shfl_xor((int)low, m));
    if (lane == 0) {
        s.wave_key[wave] = best;
        s.wave_low[wave] = low;
    }
    sample_clear(s.first, tid);
    __syncthreads();
    for (int w = 0; w < SAMPLE_WAVES; ++w) {
        best = s.wave_key[w] > best ? s.wave_key[w] : best;
        low = min(low, s.wave_low[w]);
    }
    const uint32_t top_order = (uint32_t)(best >> 32);
    const bool none = top_order == best_order(-INFINITY);
    if (none || top_order >= best_order(INFINITY) || !(temperature > 0.f)) {
        if (tid == 0) {
            A.answers[t] = none ? -1 : best_index(best);
            if (A.logp != nullptr) A.logp[t] = none ? -INFINITY : 0.f;
        }
        return;
    }
    const float top = of_order(top_order);
    const double inverse = 1.0 / (double)temperature;
    const auto weight_of = [&](float x) -> uint64_t {
        return x == -INFINITY ? 0 : (uint64_t)rint(exp(((double)x - (double)top) * inverse) * SAMPLE_UNIT);
    };
    // Bins over the values that have a weight, or over all if these lie closer.
    const float range = fminf(32.f * temperature, top - of_order(low)), per = range > 0.f ? fminf(SAMPLE_BINS / range, 3e38f) : 0.f;
    const auto bin_of = [&](float x) { return (int)fminf((top - x) * per, SAMPLE_BINS - 1.f); };
    each_logit(row, A.V, tid, SAMPLE_THREADS, [&](float x, int) {
        const int b = bin_of(x);
        const uint64_t w = weight_of(x);
        atomicAdd(&s.first.count[b], 1u);
        if (w > 0) atomicAdd(reinterpret_cast<unsigned long long *>(&s.first.weight[b]), (unsigned long long)w);
    });
    sample_sums(s, s.first, tid);

    const auto locate = [&](bool by_count, uint64_t need) {
        SamplePlace p{};
        const int bin = sample_find(s, s.first, by_count, need, tid, p);
        // the keys in it
        uint32_t lo = 0xffffffffu, hi = 0;
        each_logit(row, A.V, tid, SAMPLE_THREADS, [&](float x, int) {
            if (bin_of(x) != bin) return;
            lo = min(lo, best_order(x));
            hi = max(hi, best_order(x));
        });
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) {
            lo = min(lo, (uint32_t)__shfl_xor((int)lo, m));
            hi = max(hi, (uint32_t)__shfl_xor((int)hi, m));
        }
        if (lane == 0) {
            s.wave_low[wave] = lo;
            s.wave_count[wave] = hi;
        }
        __syncthreads();
        for (int w = 0; w < SAMPLE_WAVES; ++w) {
            lo = min(lo, s.wave_low[w]);
            hi = max(hi, s.wave_count[w]);
        }
        __syncthreads();
        while (lo < hi) {
            const int shift = max(0, 32 - __clz(hi - lo) - 10);
            sample_clear(s.fine, tid);
            __syncthreads();
            each_logit(row, A.V, tid, SAMPLE_THREADS, [&](float x, int) {
                const uint32_t o = best_order(x);
                if (o < lo || o > hi || bin_of(x) != bin) return;
                const uint64_t w = weight_of(x);
                atomicAdd(&s.fine.count[(hi - o) >> shift], 1u);
                if (w > 0) atomicAdd(reinterpret_cast<unsigned long long *>(&s.fine.weight[(hi - o) >> shift]), (unsigned long long)w);
            });
            sample_sums(s, s.fine, tid);
            const uint32_t b = (uint32_t)sample_find(s, s.fine, by_count, by_count ? need - p.before_count : need - p.before_weight, tid, p);
            hi -= b << shift;
            lo = max(lo, hi - min(hi, (1u << shift) - 1));
        }
        p.key = hi;
        return p;
    };

    uint64_t kept = s.first.weight[SAMPLE_BINS - 1];
    if (top_k > 0 && top_k < A.V) {
        const SamplePlace p = locate(true, (uint64_t)top_k);
        kept = p.before_weight + (uint64_t)(top_k - (int)p.before_count) * weight_of(of_order(p.key));
    }
    const uint64_t one = (uint64_t)SAMPLE_UNIT;
    if (top_p < 1.f) {
        const double share = ceil((double)fmaxf(top_p, 0.f) * (double)kept);
        const uint64_t need = min((uint64_t)share, kept);
        if (need <= one) {
            kept = one;
        } else {
            const SamplePlace p = locate(false, need);
            const uint64_t each = weight_of(of_order(p.key));
            kept = p.before_weight + (need - p.before_weight + each - 1) / each * each;
        }
    }
    if (min_p > 0.f) {
        const uint64_t least = (uint64_t)ceil((double)fminf(min_p, 1.f) * SAMPLE_UNIT);
        uint64_t sum = 0;
        each_logit(row, A.V, tid, SAMPLE_THREADS, [&](float x, int) {
            const uint64_t w = weight_of(x);
            sum += w >= least ? w : 0;
        });
        sum = wave_sums_u64(sum, lane);
        if (lane == 63) s.wave_weight[wave] = sum;
        __syncthreads();
        sum = 0;
        for (int w = 0; w < SAMPLE_WAVES; ++w) sum += s.wave_weight[w];
        kept = min(kept, sum);
        __syncthreads();
    }
    // the token at u times the weight that is kept
    const double u = A.u[t], at = u > 0.0 ? floor(fmin(u, 1.0) * (double)kept) : 0.0;
    const uint64_t goal = min((uint64_t)at, kept - 1);
    const SamplePlace p = locate(false, goal + 1);
    const uint32_t which = (uint32_t)((goal - p.before_weight) / weight_of(of_order(p.key)));
    // the token of that key, by index: waves take pieces of the row one after the other
    const int piece = (A.V + SAMPLE_WAVES - 1) / SAMPLE_WAVES, begin = min(wave * piece, A.V), end = min(begin + piece, A.V);
    int mine = 0;
    for (int i = begin; i < end; i += 64) mine += __popcll(__ballot(i + lane < end && best_order(to_f32(row[min(i + lane, end - 1)])) == p.key));
    if (lane == 0) s.wave_count[wave] = mine;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += s.wave_count[w];
    if ((int)which >= before && (int)which < before + mine) {
        int left = (int)which - before;
        for (int i = begin; i < end; i += 64) {
            uint64_t same = __ballot(i + lane < end && best_order(to_f32(row[min(i + lane, end - 1)])) == p.key);
            const int n = __popcll(same);
            if (left < n) {
                for (; left > 0; --left) same &= same - 1;
                if (lane == 0) {
                    A.answers[t] = i + __ffsll((unsigned long long)same) - 1;
                    if (A.logp != nullptr) A.logp[t] = (float)(((double)of_order(p.key) - (double)top) * inverse - log((double)kept / SAMPLE_UNIT));
                }
                break;
            }
            left -= n;
        }
    }
}

}  // namespace svdp
