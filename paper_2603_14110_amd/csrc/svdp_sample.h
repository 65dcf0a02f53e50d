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
// Every question (the k-th token, the token at a given weight) is one about a place in the order, which a histogram over the values answers
// up to a bin, by sums over its bins.
//  bf16: a bin is one value (2^-30 <= |x| < 2^8, and zero): a bin's weight is its count times one exponential, and a pass over the row
//    is one atomic addition an element, with no maximum and no exponential.  Rows with values between or above these go the other way.
//  else: SAMPLE_BINS bins between the largest logit and where weights end, with an exponential in 64 bits for each element.  The elements
//    of the one bin that a question leads to are listed and ordered; if they are too many, the bin is divided by their keys' bits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svdp_device.h"
#include "svdp_order.h"

namespace svdp {

constexpr int SAMPLE_THREADS = 1024, SAMPLE_WAVES = SAMPLE_THREADS / 64;
constexpr int SAMPLE_EACH = 4, SAMPLE_BINS = SAMPLE_THREADS * SAMPLE_EACH;
constexpr int SAMPLE_LIST = 768;                            // elements of a bin that are ordered by comparing all with all
constexpr double SAMPLE_UNIT = 17592186044416.0;            // 2^44
constexpr float SAMPLE_ZERO = 31.5f;                        // (top - x) / temperature from which weights are 0: 45 ln 2 = 31.19
constexpr int SAMPLE_MAX_V = 1 << 19;

// Bins of bf16 values, the largest first: magnitudes (bits without sign) from VALUE_LOW on, VALUE_SPAN of them; zero; then negative ones.
constexpr int VALUE_LOW = (127 - 30) << 7, VALUE_HIGH = (127 + 8) << 7, VALUE_SPAN = VALUE_HIGH - VALUE_LOW;
constexpr int VALUE_BINS = 2 * VALUE_SPAN + 1, VALUE_EACH = (VALUE_BINS + SAMPLE_THREADS - 1) / SAMPLE_THREADS;
constexpr float VALUE_FAR = -256.f;                         // what lies at or below it has no bin

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

// 2^44 exp(z), rounded to a whole number, z = at / ln 2 <= 0 in 64 bits: 2^at by its Taylor series to the eleventh power around the nearest
// whole number, within 2^-47 of its value.  at > -46.
__device__ __forceinline__ uint64_t sample_weight(double at)
{
    constexpr double L = 0.693147180559945309417232;
    constexpr double c[12] = {1.0, L, L * L / 2, L * L * L / 6, L * L * L * L / 24, L * L * L * L * L / 120, L * L * L * L * L * L / 720,
                              L * L * L * L * L * L * L / 5040, L * L * L * L * L * L * L * L / 40320, L * L * L * L * L * L * L * L * L / 362880,
                              L * L * L * L * L * L * L * L * L * L / 3628800, L * L * L * L * L * L * L * L * L * L * L / 39916800};
    const double whole = rint(at), r = at - whole;
    double p = c[11];
#pragma unroll
    for (int k = 10; k >= 0; --k) p = fma(p, r, c[k]);
    // the sum with 2^52 rounds to whole numbers, which are its lower bits
    const double v = ldexp(p, (int)whole + 44) + 4503599627370496.0;
    return (uint64_t)__double_as_longlong(v) & (((uint64_t)1 << 52) - 1);
}

// The weight of a logit relative to the largest one.
struct SampleScale {
    double top, per;                        // per: 1 / (temperature ln 2)
    float zero;                             // distance from the top at which weights are 0
    __device__ __forceinline__ SampleScale(float top_, float temperature) : top(top_), per(1.4426950408889634074 / (double)temperature), zero(SAMPLE_ZERO * temperature) {}
    __device__ __forceinline__ bool live(float x) const { return (float)top - x < zero; }
    __device__ __forceinline__ uint64_t of(float x) const { return live(x) ? sample_weight(((double)x - top) * per) : 0; }
};

struct SampleShared {
    union {
        uint32_t values[SAMPLE_THREADS * VALUE_EACH];
        struct {
            uint64_t bin_weight[SAMPLE_BINS];
            uint32_t bin_count[SAMPLE_BINS];
            uint64_t list[SAMPLE_LIST], list_weight[SAMPLE_LIST];
        };
    };
    uint64_t wave_weight[SAMPLE_WAVES], wave_key[SAMPLE_WAVES];
    uint32_t wave_count[SAMPLE_WAVES], wave_low[SAMPLE_WAVES];
    // what the thread that a question leads to answers
    uint64_t before_weight, weight, key;
    uint32_t before_count, count, listed;
    int bin, odd;
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
// Sums over the threads before this one, and all of them.
struct SampleSums {
    uint64_t before_weight, weight;
    uint32_t before_count, count;
};
__device__ __forceinline__ SampleSums sample_sums(SampleShared &s, uint64_t weight, uint32_t count, int tid)
{
    const int lane = tid & 63, wave = tid >> 6;
    const uint64_t w = wave_sums_u64(weight, lane);
    const uint32_t c = (uint32_t)wave_inclusive_scan((int)count);
    if (lane == 63) {
        s.wave_weight[wave] = w;
        s.wave_count[wave] = c;
    }
    __syncthreads();
    SampleSums r{w - weight, 0, c - count, 0};
    for (int i = 0; i < SAMPLE_WAVES; ++i) {
        r.before_weight += i < wave ? s.wave_weight[i] : 0;
        r.before_count += i < wave ? s.wave_count[i] : 0;
        r.weight += s.wave_weight[i];
        r.count += s.wave_count[i];
    }
    __syncthreads();
    return r;
}
__device__ __forceinline__ uint64_t sample_sum(SampleShared &s, uint64_t v, int tid)
{
    return sample_sums(s, v, 0, tid).weight;
}

// How a row's token is drawn.
struct SampleHow {
    float temperature, top_p, min_p, u;
    int top_k;
    // weight that top_p asks for, of `kept`; at least one token's
    __device__ __forceinline__ uint64_t share(uint64_t kept) const
    {
        return min((uint64_t)ceil((double)fmaxf(top_p, 0.f) * (double)kept), kept);
    }
    __device__ __forceinline__ uint64_t least() const { return (uint64_t)ceil((double)fminf(min_p, 1.f) * SAMPLE_UNIT); }
    // the drawn token is the first one with more than this up to it
    __device__ __forceinline__ uint64_t goal(uint64_t kept) const
    {
        const double at = u > 0.f ? floor(fmin((double)u, 1.0) * (double)kept) : 0.0;
        return min((uint64_t)at, kept - 1);
    }
};
constexpr uint64_t SAMPLE_ONE = (uint64_t)1 << 44;

// The index of the which-th element of a row (from 0) that is(value): waves take pieces of the row one after the other.
template <typename W, typename F>
__device__ __forceinline__ void sample_index(SampleShared &s, const W *row, int V, uint32_t which, int tid, F &&is, int32_t *answer)
{
    constexpr int VEC = Elem<W>::VEC, AHEAD = 4;
    const int lane = tid & 63, wave = tid >> 6, skew = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / Elem<W>::BYTES);
    const int head = min(skew > 0 ? VEC - skew : 0, V), vectors = (V - head) / VEC, tail = head + vectors * VEC;
    const int piece = (vectors + SAMPLE_WAVES - 1) / SAMPLE_WAVES, begin = min(wave * piece, vectors), end = min(begin + piece, vectors);
    const bool first = wave == 0, last = wave == SAMPLE_WAVES - 1;
    const auto is_head = [&] { return first && lane < head && is(to_f32(row[lane])); };
    const auto is_tail = [&] { return last && tail + lane < V && is(to_f32(row[tail + lane])); };
    const auto bits_of = [&](const uint4 &in) {
        float v[VEC];
        widen(in, v, row);
        uint32_t bits = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) bits |= is(v[j]) ? 1u << j : 0u;
        return bits;
    };
    int mine = 0;
    for (int i0 = begin + lane; i0 < end; i0 += AHEAD * 64) {
        uint4 in[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) in[a] = load_raw(row + head + (int64_t)min(i0 + a * 64, end - 1) * VEC);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) mine += i0 + a * 64 < end ? __popc(bits_of(in[a])) : 0;
    }
    mine += (is_head() ? 1 : 0) + (is_tail() ? 1 : 0);
    const int all = wave_inclusive_scan(mine);
    if (lane == 63) s.wave_count[wave] = (uint32_t)all;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave; ++w) before += s.wave_count[w];
    if (which < before || which >= before + s.wave_count[wave]) return;
    uint32_t left = which - before;
    const uint64_t heads = __ballot(is_head());
    const auto nth = [](uint64_t set, uint32_t n) {
        for (; n > 0; --n) set &= set - 1;
        return __ffsll((unsigned long long)set) - 1;
    };
    if (left < (uint32_t)__popcll(heads)) {
        if (lane == 0) *answer = nth(heads, left);
        return;
    }
    left -= (uint32_t)__popcll(heads);
    for (int i0 = begin; i0 < end; i0 += 64) {
        const uint32_t bits = i0 + lane < end ? bits_of(load_raw(row + head + (int64_t)(i0 + lane) * VEC)) : 0;
        if (__ballot(bits != 0) == 0) continue;
        const int n = __popc(bits), upto = wave_inclusive_scan(n), sum = __builtin_amdgcn_readlane(upto, 63);
        if (left < (uint32_t)sum) {
            if ((int)left >= upto - n && (int)left < upto) *answer = head + (i0 + lane) * VEC + nth(bits, left - (uint32_t)(upto - n));
            return;
        }
        left -= (uint32_t)sum;
    }
    const uint64_t tails = __ballot(is_tail());
    if (lane == 0) *answer = tail + nth(tails, left);
}

// ---- bf16: one bin a value --------------------------------------------------------------------------------------------------

__device__ __forceinline__ float value_of_bin(int b)
{
    const uint32_t bits = b < VALUE_SPAN ? VALUE_HIGH - 1 - b : b == VALUE_SPAN ? 0u : 0x8000u | (VALUE_LOW + b - VALUE_SPAN - 1);
    return __uint_as_float(bits << 16);
}
// False: the row has to go the other way.
__device__ __forceinline__ bool sample_by_value(SampleShared &s, const bf16 *row, int V, const SampleHow &how, int tid, int32_t *answer, float *logp)
{
#pragma unroll
    for (int j = 0; j < VALUE_EACH; ++j) s.values[j * SAMPLE_THREADS + tid] = 0;
    if (tid == 0) {
        s.odd = 0;
        s.bin = VALUE_BINS;
    }
    __syncthreads();
    bool odd = false;
    each_logit(row, V, tid, SAMPLE_THREADS, [&](float x, int) {
        const uint32_t u = __float_as_uint(x), m = (u >> 16) & 0x7fffu;
        const bool negative = u >> 31, binned = m - VALUE_LOW < (uint32_t)VALUE_SPAN;
        const uint32_t b = negative ? m + (VALUE_SPAN + 1 - VALUE_LOW) : VALUE_HIGH - 1 - m;
        if (binned || m == 0) atomicAdd(&s.values[m == 0 ? VALUE_SPAN : b], 1u);
        else odd = odd || !negative || m < VALUE_LOW || m > 0x7f80u;            // else far below, or -inf
    });
    if (odd) s.odd = 1;
    __syncthreads();
    if (s.odd) return false;
    uint32_t c[VALUE_EACH], count = 0;
    int first = VALUE_BINS;
#pragma unroll
    for (int j = VALUE_EACH - 1; j >= 0; --j) {
        c[j] = s.values[tid * VALUE_EACH + j];
        count += c[j];
        first = c[j] > 0 ? tid * VALUE_EACH + j : first;
    }
    if (__any(count > 0)) {
        const int lowest = __builtin_amdgcn_readlane(first, __ffsll((unsigned long long)__ballot(count > 0)) - 1);
        if ((tid & 63) == 0) atomicMin(&s.bin, lowest);
    }
    __syncthreads();
    first = s.bin;
    if (first == VALUE_BINS) return false;
    const SampleScale scale(value_of_bin(first), how.temperature);
    uint64_t w[VALUE_EACH], weight = 0;
#pragma unroll
    for (int j = 0; j < VALUE_EACH; ++j) {
        w[j] = c[j] > 0 ? scale.of(value_of_bin(tid * VALUE_EACH + j)) : 0;
        weight += w[j] * c[j];
    }
    const SampleSums sums = sample_sums(s, weight, count, tid);
    if (sums.count < (uint32_t)V && scale.live(VALUE_FAR)) return false;
    // the bin that a question leads to: what is before it, and in it
    const auto locate = [&](bool by_count, uint64_t need) {
        const uint64_t lo = by_count ? sums.before_count : sums.before_weight, hi = lo + (by_count ? count : weight);
        if (lo < need && need <= hi) {
            uint64_t bw = sums.before_weight;
            uint32_t bc = sums.before_count;
            bool found = false;
#pragma unroll
            for (int j = 0; j < VALUE_EACH; ++j) {
                if (!found && need <= (by_count ? bc + c[j] : bw + w[j] * c[j])) {
                    found = true;
                    s.bin = tid * VALUE_EACH + j;
                    s.before_weight = bw;
                    s.before_count = bc;
                    s.weight = w[j];
                }
                bw += w[j] * c[j];
                bc += c[j];
            }
        }
        __syncthreads();
    };
    uint64_t kept = sums.weight;
    if (how.top_k > 0 && (uint32_t)how.top_k < sums.count) {
        locate(true, (uint64_t)how.top_k);
        kept = s.before_weight + (uint64_t)((uint32_t)how.top_k - s.before_count) * s.weight;
        __syncthreads();
    }
    if (how.top_p < 1.f) {
        const uint64_t need = how.share(kept);
        if (need <= SAMPLE_ONE) {
            kept = SAMPLE_ONE;
        } else {
            locate(false, need);
            kept = s.before_weight + (need - s.before_weight + s.weight - 1) / s.weight * s.weight;
            __syncthreads();
        }
    }
    if (how.min_p > 0.f) {
        const uint64_t least = how.least();
        uint64_t sum = 0;
#pragma unroll
        for (int j = 0; j < VALUE_EACH; ++j) sum += w[j] >= least ? w[j] * c[j] : 0;
        kept = min(kept, sample_sum(s, sum, tid));
    }
    const uint64_t goal = how.goal(kept);
    locate(false, goal + 1);
    const float x = value_of_bin(s.bin);
    const uint32_t which = (uint32_t)((goal - s.before_weight) / s.weight);
    if (tid == 0 && logp != nullptr) *logp = (float)(((double)x - scale.top) / (double)how.temperature - log((double)kept / SAMPLE_UNIT));
    sample_index(s, row, V, which, tid, [&](float v) { return v == x; }, answer);
    return true;
}

// ---- any values -------------------------------------------------------------------------------------------------------------

template <typename W>
__device__ __forceinline__ void sample_by_range(SampleShared &s, const W *row, int V, const SampleHow &how, int tid, int32_t *answer, float *logp)
{
    const int lane = tid & 63, wave = tid >> 6;
    // the first token of the order, and the smallest finite logit
    uint64_t best = 0;
    uint32_t low = 0xffffffffu;
    __syncthreads();
    each_logit(row, V, tid, SAMPLE_THREADS, [&](float x, int i) {
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
    const auto clear = [&] {
#pragma unroll
        for (int j = 0; j < SAMPLE_EACH; ++j) {
            s.bin_weight[j * SAMPLE_THREADS + tid] = 0;
            s.bin_count[j * SAMPLE_THREADS + tid] = 0;
        }
        __syncthreads();
    };
    clear();
    for (int w = 0; w < SAMPLE_WAVES; ++w) {
        best = s.wave_key[w] > best ? s.wave_key[w] : best;
        low = min(low, s.wave_low[w]);
    }
    const uint32_t top_order = (uint32_t)(best >> 32);
    const bool none = top_order == best_order(-INFINITY);
    if (none || top_order >= best_order(INFINITY) || !(how.temperature > 0.f)) {
        if (tid == 0) {
            *answer = none ? -1 : best_index(best);
            if (logp != nullptr) *logp = none ? -INFINITY : 0.f;
        }
        return;
    }
    const float top = of_order(top_order);
    const SampleScale scale(top, how.temperature);
    // Bins over the values that have a weight, or over all if these lie closer.
    const float range = fminf(scale.zero, top - of_order(low)), per = range > 0.f ? fminf(SAMPLE_BINS / range, 3e38f) : 0.f;
    const auto bin_of = [&](float x) { return (int)fminf((top - x) * per, SAMPLE_BINS - 1.f); };
    const bool counted = how.top_k > 0 && how.top_k < V;
    each_logit(row, V, tid, SAMPLE_THREADS, [&](float x, int) {
        if (counted) atomicAdd(&s.bin_count[bin_of(x)], 1u);
        if (scale.live(x)) atomicAdd(reinterpret_cast<unsigned long long *>(&s.bin_weight[bin_of(x)]), (unsigned long long)scale.of(x));
    });
    __syncthreads();

    // The thread and bin that a question leads to: s.bin, and what is before it.
    const auto find = [&](const SampleSums &sums, const uint64_t (&w)[SAMPLE_EACH], const uint32_t (&c)[SAMPLE_EACH], uint64_t weight, uint32_t count,
                          bool by_count, uint64_t need) {
        const uint64_t lo = by_count ? sums.before_count : sums.before_weight, hi = lo + (by_count ? count : weight);
        if (lo < need && need <= hi) {
            uint64_t bw = sums.before_weight;
            uint32_t bc = sums.before_count;
            bool found = false;
#pragma unroll
            for (int j = 0; j < SAMPLE_EACH; ++j) {
                if (!found && need <= (by_count ? bc + c[j] : bw + w[j])) {
                    found = true;
                    s.bin = tid * SAMPLE_EACH + j;
                    s.before_weight = bw;
                    s.before_count = bc;
                }
                bw += w[j];
                bc += c[j];
            }
        }
        __syncthreads();
    };
    uint64_t w[SAMPLE_EACH], weight = 0;
    uint32_t c[SAMPLE_EACH], count = 0;
    const auto read = [&](uint64_t (&w)[SAMPLE_EACH], uint32_t (&c)[SAMPLE_EACH], uint64_t &weight, uint32_t &count) {
        weight = 0;
        count = 0;
#pragma unroll
        for (int j = 0; j < SAMPLE_EACH; ++j) {
            w[j] = s.bin_weight[tid * SAMPLE_EACH + j];
            c[j] = s.bin_count[tid * SAMPLE_EACH + j];
            weight += w[j];
            count += c[j];
        }
    };
    read(w, c, weight, count);
    const SampleSums sums = sample_sums(s, weight, count, tid);

    // The token that a question leads to: weight up to it and with it, and its key (order, and index in reverse); by_index: the index is needed.
    struct Place {
        uint64_t upto;
        uint32_t order;
        int index;                          // -1: it is the which-th of its value
        uint32_t which;
    };
    const auto locate = [&](bool by_count, uint64_t need) {
        if (tid == 0) s.listed = 0;
        find(sums, w, c, weight, count, by_count, need);
        const int bin = s.bin;
        uint64_t before_weight = s.before_weight;
        uint32_t before_count = s.before_count;
        uint32_t lo = 0xffffffffu, hi = 0;
        each_logit(row, V, tid, SAMPLE_THREADS, [&](float x, int i) {
            if (bin_of(x) != bin) return;
            const uint64_t key = best_key(x, i);
            lo = min(lo, (uint32_t)(key >> 32));
            hi = max(hi, (uint32_t)(key >> 32));
            const uint32_t at = atomicAdd(&s.listed, 1u);
            if (at < SAMPLE_LIST) {
                s.list[at] = key;
                s.list_weight[at] = scale.of(x);
            }
        });
        __syncthreads();
        const int n = (int)s.listed;
        if (n <= SAMPLE_LIST) {
            for (int i = tid; i < n; i += SAMPLE_THREADS) {
                const uint64_t mine = s.list[i], own = s.list_weight[i];
                uint64_t bw = before_weight;
                uint32_t bc = before_count;
                for (int j = 0; j < n; ++j) {
                    const bool ahead = s.list[j] > mine;
                    bw += ahead ? s.list_weight[j] : 0;
                    bc += ahead ? 1 : 0;
                }
                if (by_count ? need == bc + 1u : bw < need && need <= bw + own) {
                    s.key = mine;
                    s.before_weight = bw + own;
                }
            }
            __syncthreads();
            const Place p{s.before_weight, (uint32_t)(s.key >> 32), best_index(s.key), 0};
            __syncthreads();
            return p;
        }
        // too many: by the bits of their order, from the top
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
        for (int i = 0; i < SAMPLE_WAVES; ++i) {
            lo = min(lo, s.wave_low[i]);
            hi = max(hi, s.wave_count[i]);
        }
        __syncthreads();
        while (lo < hi) {
            const int shift = max(0, 32 - __clz(hi - lo) - 12);
            clear();
            each_logit(row, V, tid, SAMPLE_THREADS, [&](float x, int) {
                const uint32_t o = best_order(x);
                if (o < lo || o > hi || bin_of(x) != bin) return;
                atomicAdd(&s.bin_count[(hi - o) >> shift], 1u);
                if (scale.live(x)) atomicAdd(reinterpret_cast<unsigned long long *>(&s.bin_weight[(hi - o) >> shift]), (unsigned long long)scale.of(x));
            });
            __syncthreads();
            uint64_t w[SAMPLE_EACH], weight;
            uint32_t c[SAMPLE_EACH], count;
            read(w, c, weight, count);
            SampleSums inner = sample_sums(s, weight, count, tid);
            inner.before_weight += before_weight;
            inner.before_count += before_count;
            find(inner, w, c, weight, count, by_count, need);
            before_weight = s.before_weight;
            before_count = s.before_count;
            hi -= (uint32_t)s.bin << shift;
            lo = max(lo, hi - min(hi, (1u << shift) - 1));
            __syncthreads();
        }
        const uint64_t each = scale.of(of_order(hi));
        const uint64_t tokens = by_count ? need - before_count : (need - before_weight + each - 1) / each;
        return Place{before_weight + tokens * each, hi, -1, (uint32_t)(tokens - 1)};
    };

    uint64_t kept = sums.weight;
    if (counted) kept = locate(true, (uint64_t)how.top_k).upto;
    if (how.top_p < 1.f) {
        const uint64_t need = how.share(kept);
        kept = need <= SAMPLE_ONE ? SAMPLE_ONE : locate(false, need).upto;
    }
    if (how.min_p > 0.f) {
        const uint64_t least = how.least();
        uint64_t sum = 0;
        each_logit(row, V, tid, SAMPLE_THREADS, [&](float x, int) {
            const uint64_t w = scale.of(x);
            sum += w >= least ? w : 0;
        });
        kept = min(kept, sample_sum(s, sum, tid));
    }
    const Place p = locate(false, how.goal(kept) + 1);
    if (tid == 0) {
        if (logp != nullptr) *logp = (float)(((double)of_order(p.order) - (double)top) / (double)how.temperature - log((double)kept / SAMPLE_UNIT));
        if (p.index >= 0) *answer = p.index;
    }
    if (p.index < 0) sample_index(s, row, V, p.which, tid, [&](float v) { return best_order(v) == p.order; }, answer);
}

// One block a row.
template <typename W>
__global__ __launch_bounds__(SAMPLE_THREADS) void k_sample(SampleArgs A)
{
    __shared__ SampleShared s;
    const int tid = threadIdx.x, t = blockIdx.x;
    const W *row = static_cast<const W *>(A.logits) + (int64_t)t * A.stride;
    const SampleHow how{A.temperature != nullptr ? A.temperature[t] : 1.f, A.top_p != nullptr ? A.top_p[t] : 1.f, A.min_p != nullptr ? A.min_p[t] : 0.f, A.u[t],
                        A.top_k != nullptr ? A.top_k[t] : 0};
    float *logp = A.logp != nullptr ? A.logp + t : nullptr;
    if constexpr (sizeof(W) == 2)
        if (how.temperature > 0.f && sample_by_value(s, row, A.V, how, tid, A.answers + t, logp)) return;
    sample_by_range(s, row, A.V, how, tid, A.answers + t, logp);
}

}  // namespace svdp
