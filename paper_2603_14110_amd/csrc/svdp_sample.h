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
//  else: SAMPLE_BINS bins between the largest logit and where weights end, each element's weight being that of a place in a table times
//    a series of five terms, in 64 bits.  The elements of the one bin that a question leads to are listed and ordered; if they are too many,
//    the bin is divided by their keys' bits.
//
// What bounds it.  bf16, 769 rows of 152 064, 234 MB: 72 us (and 4.6 for the launch that looks after left rows), where reading takes 46: vector
// units 59 % of the time (10 instructions for two elements, and half of all for the bins' weights and the questions), LDS 42 %, of which two
// thirds are bank conflicts of the counters (10.5 of 15.0 million cycles); a row whose token's value is not the only one of its kind is read
// once more, and so is one with zeros or masked logits (-inf, or the type's lowest value), whose others are looked at: 769 rows of 152 064
// 70 -> 97 us, one of them 18.9 -> 26.5, 8 rows of 32 000 16.6 -> 18.6.  8 rows of 32 000: 13 us, by the latency of one block's passes.
// fp32: weights and additions of 64 bits in LDS.  One row of 32 000, by one compute unit: 19 us (with a series of 11 terms and no table 21.7,
// of which the weights' pass took 9.5, each question 3, the maximum 3); 256 rows of 152 064: 111 us, where reading takes 30.  Tried and
// dropped: bins over the front of the values only, all others just summed up (more registers than there are: 31 us for one row of 32 000);
// for bf16 the row in registers, 20 vectors a thread (spills: 177 us).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "svdp_device.h"
#include "svdp_order.h"

namespace svdp {

constexpr int SAMPLE_MAX_V = 1 << 19;
constexpr int SAMPLE_THREADS = 1024, SAMPLE_WAVES = SAMPLE_THREADS / 64;
constexpr int SAMPLE_EACH = 4, SAMPLE_BINS = SAMPLE_THREADS * SAMPLE_EACH;
constexpr int SAMPLE_TABLE = SAMPLE_BINS / 2;
constexpr int SAMPLE_LIST = 768;                            // elements of a bin that are ordered by comparing all with all
constexpr double SAMPLE_UNIT = 17592186044416.0;            // 2^44
constexpr float SAMPLE_ZERO = 31.5f;                        // (top - x) / temperature from which weights are 0: 45 ln 2 = 31.19

// Bins of bf16 values, the largest first: magnitudes (bits without sign) from VALUE_LOW on, VALUE_SPAN of them; zero; then negative ones.
constexpr int VALUE_LOW = (127 - 30) << 7, VALUE_HIGH = (127 + 8) << 7, VALUE_SPAN = VALUE_HIGH - VALUE_LOW;
constexpr float VALUE_FAR = -256.f;                         // what lies at or below it has no bin
// In LDS: counters of positive magnitudes, then of negative ones, each followed by one a lane for all that has no bin: lanes do
// not meet there, whatever a row is filled up with.
// A counter's lower bits are the count; the upper ones are the sum of the places of what was counted, in pieces of the row: where the
// count is one, the piece that has the element.
constexpr int VALUE_OTHER = 64, VALUE_SIDE = VALUE_SPAN + VALUE_OTHER;
constexpr int VALUE_COUNT = 20, VALUE_PIECE = 16;           // bits of the count; 16-byte vectors of a piece
static_assert(SAMPLE_MAX_V < 1 << VALUE_COUNT && SAMPLE_MAX_V / 8 / VALUE_PIECE <= 1 << (32 - VALUE_COUNT));
static_assert(4 * 2 * VALUE_SIDE < 65536, "addresses of counters are halves of a word");

typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
typedef int16_t i16x2_t __attribute__((ext_vector_type(2)));

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

// v(16 bytes, index of their first element) for a thread's share of a row, and f(value, index) for the elements at the row's ends that are
// no whole vector.
template <int AHEAD, typename W, typename Fv, typename F>
__device__ __forceinline__ void each_vector(const W *row, int V, int tid, int threads, Fv &&v, F &&f)
{
    constexpr int VEC = Elem<W>::VEC;
    const int skew = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / Elem<W>::BYTES);
    const int head = min(skew > 0 ? VEC - skew : 0, V), vectors = (V - head) / VEC, tail = head + vectors * VEC;
    // the next vectors are requested before these are looked at
    uint4 in[AHEAD], next[AHEAD];
    const auto request = [&](int i0, uint4 (&to)[AHEAD]) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) to[a] = load_raw(row + head + (int64_t)min(i0 + a * threads, vectors - 1) * VEC);
    };
    if (tid < vectors) request(tid, in);
    for (int i0 = tid; i0 < vectors; i0 += AHEAD * threads) {
        request(i0 + AHEAD * threads, next);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int i = i0 + a * threads;
            if (i < vectors) v(in[a], head + i * VEC);
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) in[a] = next[a];
    }
    if (tid < head) f(to_f32(row[tid]), tid);
    if (tail + tid < V) f(to_f32(row[tail + tid]), tail + tid);
}
// f(value, index) for a thread's share.
template <int AHEAD, typename W, typename F>
__device__ __forceinline__ void each_logit(const W *row, int V, int tid, int threads, F &&f)
{
    constexpr int VEC = Elem<W>::VEC;
    each_vector<AHEAD>(row, V, tid, threads, [&](const uint4 &in, int i) {
        float v[VEC];
        widen(in, v, row);
#pragma unroll
        for (int j = 0; j < VEC; ++j) f(v[j], i + j);
    }, f);
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

// What the threads of a row share.
template <int THREADS>
struct SampleWaveSums {
    static constexpr int WAVES = THREADS / 64;
    uint64_t weight[WAVES];
    uint32_t count[WAVES], low[WAVES];
};
template <int THREADS>
struct SampleValues {
    uint32_t values[2 * VALUE_SIDE];
    SampleWaveSums<THREADS> waves;
    uint32_t zeros, others, odd;
    // where a question leads to, of three a row: the thread, and what is before its bins
    struct {
        uint64_t before_weight;
        uint32_t before_count;
        int thread;
    } asked[3];
};
struct SampleBins {
    double table[SAMPLE_TABLE];             // weights, not rounded, in the middle of every two bins
    uint64_t weight[SAMPLE_BINS];
    uint32_t count[SAMPLE_BINS];
    uint64_t list[SAMPLE_LIST], list_weight[SAMPLE_LIST];
    SampleWaveSums<SAMPLE_THREADS> waves;
    // what the thread that a question leads to answers
    uint64_t before_weight, key;
    uint32_t before_count, listed;
    int bin;
};
static_assert(2 * sizeof(SampleBins) <= LDS_MAX && 4 * sizeof(SampleValues<512>) <= LDS_MAX);

// Inclusive sums over a wave, as wave_inclusive_scan.
template <int CTRL, int ROW_MASK, int BANK_MASK>
__device__ __forceinline__ uint64_t dpp_take_u64(uint64_t v)
{
    return (uint32_t)dpp_take<CTRL, ROW_MASK, BANK_MASK>((int)(uint32_t)v) | (uint64_t)(uint32_t)dpp_take<CTRL, ROW_MASK, BANK_MASK>((int)(v >> 32)) << 32;
}
__device__ __forceinline__ uint64_t wave_sums_u64(uint64_t v)
{
    uint64_t s = v + dpp_take_u64<0x111, 0xf, 0xf>(v);
    s += dpp_take_u64<0x112, 0xf, 0xf>(v);
    s += dpp_take_u64<0x113, 0xf, 0xf>(v);
    s += dpp_take_u64<0x114, 0xf, 0xe>(s);
    s += dpp_take_u64<0x118, 0xf, 0xc>(s);
    s += dpp_take_u64<0x142, 0xa, 0xf>(s);
    s += dpp_take_u64<0x143, 0xc, 0xf>(s);
    return s;
}
__device__ __forceinline__ uint64_t lane_of_u64(uint64_t v, int lane)
{
    return (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32;
}
// a / b, of less than 2^31: the quotient in fp64 is at most one off, and put right.
__device__ __forceinline__ uint32_t sample_quotient(uint64_t a, uint64_t b)
{
    uint32_t q = (uint32_t)((double)a / (double)b);
    if ((uint64_t)q * b > a) --q;
    if ((uint64_t)(q + 1) * b <= a) ++q;
    return q;
}
// Sums over the threads before this one, and all of them.
struct SampleSums {
    uint64_t before_weight, weight;
    uint32_t before_count, count;
};
template <int THREADS>
__device__ __forceinline__ SampleSums sample_sums(SampleWaveSums<THREADS> &s, uint64_t weight, uint32_t count, int tid)
{
    constexpr int WAVES = THREADS / 64;
    const int lane = tid & 63, wave = tid >> 6;
    const uint64_t w = wave_sums_u64(weight);
    const uint32_t c = (uint32_t)wave_inclusive_scan((int)count);
    if (lane == 63) {
        s.weight[wave] = w;
        s.count[wave] = c;
    }
    __syncthreads();
    // the waves' sums, a lane each
    const uint64_t each_weight = lane < WAVES ? s.weight[lane] : 0, upto_weight = wave_sums_u64(each_weight);
    const uint32_t each_count = lane < WAVES ? s.count[lane] : 0, upto_count = (uint32_t)wave_inclusive_scan((int)each_count);
    const int at = __builtin_amdgcn_readfirstlane(wave);
    const SampleSums r{w - weight + lane_of_u64(upto_weight - each_weight, at), lane_of_u64(upto_weight, 63),
                       c - count + (uint32_t)__builtin_amdgcn_readlane((int)(upto_count - each_count), at), (uint32_t)__builtin_amdgcn_readlane((int)upto_count, 63)};
    __syncthreads();
    return r;
}
template <int THREADS>
__device__ __forceinline__ uint64_t sample_sum(SampleWaveSums<THREADS> &s, uint64_t v, int tid)
{
    return sample_sums(s, v, 0, tid).weight;
}

// How a row's token is drawn.
struct SampleHow {
    float temperature, top_p, min_p, u;
    int top_k;
    bool first;                             // the first token of the order: nothing is drawn
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

// Which elements of a vector have the value x (zero: of either sign; NaN: any NaN), as bits.
template <typename W>
__device__ __forceinline__ bool same_value(float v, float x)
{
    return v == x || (v != v && x != x);
}
__device__ __forceinline__ bool has_value(const uint4 &in, float x, const float *)
{
    const float4 v = as_float4(in);
    return same_value<float>(v.x, x) || same_value<float>(v.y, x) || same_value<float>(v.z, x) || same_value<float>(v.w, x);
}
// The smallest of all halves' differences from x in bits: a half of zero is x.  NaN is compared one by one, the other sign of zero too.
__device__ __forceinline__ bool has_value(const uint4 &in, float x, const bf16 *)
{
    if (!(x < 0.f || x > 0.f)) return true;
    const uint32_t h = __float_as_uint(x) >> 16, both = h | h << 16;
    const auto far = [&](uint32_t w) { return __builtin_bit_cast(u16x2_t, w ^ both); };
    const u16x2_t a = __builtin_elementwise_min(far(in.x), far(in.y)), b = __builtin_elementwise_min(far(in.z), far(in.w));
    const u16x2_t m = __builtin_elementwise_min(a, b);
    return min(m[0], m[1]) == 0;
}
// The index of the which-th element (from 0) of value x: waves take pieces of the row one after the other.
template <int THREADS, typename W>
__device__ __forceinline__ void sample_index(SampleWaveSums<THREADS> &s, const W *row, int V, uint32_t which, int tid, float x, int32_t *answer)
{
    constexpr int VEC = Elem<W>::VEC, AHEAD = 8, WAVES = THREADS / 64;
    const int lane = tid & 63, wave = tid >> 6, skew = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / Elem<W>::BYTES);
    const int head = min(skew > 0 ? VEC - skew : 0, V), vectors = (V - head) / VEC, tail = head + vectors * VEC;
    const int piece = (vectors + WAVES - 1) / WAVES, begin = min(wave * piece, vectors), end = min(begin + piece, vectors);
    const bool first = wave == 0, last = wave == WAVES - 1;
    const auto is_head = [&] { return first && lane < head && same_value<W>(to_f32(row[lane]), x); };
    const auto is_tail = [&] { return last && tail + lane < V && same_value<W>(to_f32(row[tail + lane]), x); };
    const auto bits_of = [&](const uint4 &in) {
        float v[VEC];
        widen(in, v, row);
        uint32_t bits = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) bits |= same_value<W>(v[j], x) ? 1u << j : 0u;
        return bits;
    };
    int mine = 0, at = 0;                   // what a lane has, and the last place of them
    for (int i0 = begin; i0 < end; i0 += AHEAD * 64) {
        uint4 in[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) in[a] = load_raw(row + head + (int64_t)min(i0 + lane + a * 64, end - 1) * VEC);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
            if (__any(has_value(in[a], x, row))) {
                const int i = i0 + lane + a * 64;
                const uint32_t bits = i < end ? bits_of(in[a]) : 0;
                mine += __popc(bits);
                at = bits != 0 ? head + i * VEC + __ffs((int)bits) - 1 : at;
            }
    }
    if (is_head()) {
        ++mine;
        at = lane;
    }
    if (is_tail()) {
        ++mine;
        at = tail + lane;
    }
    const int all = wave_inclusive_scan(mine);
    if (lane == 63) s.count[wave] = (uint32_t)all;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave; ++w) before += s.count[w];
    if (which < before || which >= before + s.count[wave]) return;
    if (s.count[wave] == 1) {
        if (mine > 0) *answer = at;
        return;
    }
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
    for (int i0 = begin; i0 < end; i0 += AHEAD * 64) {
        uint4 in[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) in[a] = load_raw(row + head + (int64_t)min(i0 + lane + a * 64, end - 1) * VEC);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (!__any(has_value(in[a], x, row))) continue;
            const int i = i0 + lane + a * 64;
            const uint32_t bits = i < end ? bits_of(in[a]) : 0;
            const int n = __popc(bits), upto = wave_inclusive_scan(n), sum = __builtin_amdgcn_readlane(upto, 63);
            if (left < (uint32_t)sum) {
                if ((int)left >= upto - n && (int)left < upto) *answer = head + i * VEC + nth(bits, left - (uint32_t)(upto - n));
                return;
            }
            left -= (uint32_t)sum;
        }
    }
    const uint64_t tails = __ballot(is_tail());
    if (lane == 0) *answer = tail + nth(tails, left);
}

// The index of the only element of value x, which lies in a piece of VALUE_PIECE vectors or at the end of the row beside it: by one wave.
__device__ __forceinline__ void sample_index_in(const bf16 *row, int V, int piece, int lane, float x, int32_t *answer)
{
    const int skew = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / 2), head = min(skew > 0 ? 8 - skew : 0, V), vectors = (V - head) / 8, tail = head + vectors * 8;
    const int i = piece * VALUE_PIECE + lane;
    if (lane < VALUE_PIECE && i < vectors) {
        float v[8];
        widen(load_raw(row + head + (int64_t)i * 8), v, row);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (v[j] == x) *answer = head + i * 8 + j;
    }
    if (lane < head && to_f32(row[lane]) == x) *answer = lane;
    if (tail + lane < V && to_f32(row[tail + lane]) == x) *answer = tail + lane;
}

// ---- bf16: one bin a value --------------------------------------------------------------------------------------------------

// A thread's bins, the largest value first: the first half of the threads has the positive ones and, in its last thread, zero.
template <int THREADS>
struct ValueBins {
    static constexpr int HALF = THREADS / 2, EACH = (VALUE_SPAN + HALF - 2) / (HALF - 1);     // threads of a sign; bins of a thread, below 64
    static_assert(EACH * (HALF - 1) >= VALUE_SPAN && EACH < 64, "the last thread of the positive ones has zero");
    int bits, step, at, n;                  // of the first bin's value, from one to the next; its counter
    bool zero;
    __device__ __forceinline__ ValueBins(int tid)
    {
        const bool positive = tid < HALF;
        const int first = (positive ? tid : tid - HALF) * EACH;
        step = positive ? -1 : 1;
        zero = tid == HALF - 1;
        n = zero ? 1 : min(max(VALUE_SPAN - first, 0), EACH);
        bits = zero ? 0 : positive ? VALUE_HIGH - 1 - first : 0x8000 + VALUE_LOW + first;
        at = positive ? VALUE_SPAN - 1 - first : VALUE_SIDE + first;
    }
    __device__ __forceinline__ float value(int j) const { return __uint_as_float((uint32_t)(bits + j * step) << 16); }
    __device__ __forceinline__ uint32_t count(const SampleValues<THREADS> &s, int j, uint32_t zeros) const
    {
        return j >= n ? 0u : zero ? zeros : s.values[at + j * step] & ((1u << VALUE_COUNT) - 1);
    }
    // the piece of an element that is the only one of its value; -1: not known
    __device__ __forceinline__ int piece(const SampleValues<THREADS> &s, int j) const
    {
        const uint32_t c = zero ? 0u : s.values[at + j * step];
        return (c & ((1u << VALUE_COUNT) - 1)) == 1 ? (int)(c >> VALUE_COUNT) : -1;
    }
};
// False: the row has to go the other way.
template <int THREADS>
__device__ __forceinline__ bool sample_by_value(SampleValues<THREADS> &s, const bf16 *row, int V, const SampleHow &how, int tid, int32_t *answer, float *logp)
{
    using Bins = ValueBins<THREADS>;
    constexpr int EACH = Bins::EACH;
    for (int i = tid; i < 2 * VALUE_SIDE; i += THREADS) s.values[i] = 0;
    if (tid == 0) s.zeros = s.others = s.odd = 0;
    __syncthreads();
    // Two elements at a time, as halves of a word, in two bytes a bin until the last step: magnitude from VALUE_LOW on (below it: a large
    // number; doubled, an element has lost its sign), up to the lane's own counter for others, plus one side for a sign.
    const uint16_t other = (uint16_t)(2 * (VALUE_SPAN + (tid & (VALUE_OTHER - 1))));
    // Factors that the compiler does not know stay factors: a product and a sum in one instruction.
    u16x2_t two = {2, 2}, side = {2 * VALUE_SIDE, 2 * VALUE_SIDE};
    asm("" : "+v"(two), "+v"(side));
    const auto pair = [&](uint32_t w, uint32_t one) {
        const u16x2_t x = __builtin_bit_cast(u16x2_t, w);
        const u16x2_t m = __builtin_elementwise_min(x * two - (uint16_t)(2 * VALUE_LOW), u16x2_t{other, other});
        const uint32_t at = __builtin_bit_cast(uint32_t, (x >> 15) * side + m) << 1;
        char *counters = reinterpret_cast<char *>(s.values);
        atomicAdd(reinterpret_cast<uint32_t *>(counters + (at & 0xffffu)), one);
        return reinterpret_cast<uint32_t *>(counters + (at >> 16));
    };
    each_vector<4>(row, V, tid, THREADS, [&](const uint4 &in, int i) {
        // i begins at the row's head, less than a vector: that leaves the quotient by vectors alone
        const uint32_t one = 1u + ((uint32_t)(i / 8 / VALUE_PIECE) << VALUE_COUNT);
        atomicAdd(pair(in.x, one), one);
        atomicAdd(pair(in.y, one), one);
        atomicAdd(pair(in.z, one), one);
        atomicAdd(pair(in.w, one), one);
    }, [&](float x, int) { pair(__float_as_uint(x) >> 16, 1u); });
    __syncthreads();
    // Others: zeros are counted, values far below (-inf among them) have no weight; with any else (small: smaller than VALUE_LOW, but not zero;
    // large or NaN) the row goes the other way.
    if (tid < VALUE_OTHER && (s.values[VALUE_SPAN + tid] | s.values[VALUE_SIDE + VALUE_SPAN + tid]) != 0) s.others = 1;
    __syncthreads();
    uint32_t zeros = 0;
    if (s.others != 0) {
        u16x2_t small = {0xffff, 0xffff}, negative = {0, 0}, nonzero = {0, 0};
        i16x2_t large = {0, 0};
        uint32_t elements = 0;
        const auto look = [&](uint32_t w) {
            const u16x2_t x = __builtin_bit_cast(u16x2_t, w), m = x & (uint16_t)0x7fff;
            small = __builtin_elementwise_min(small, m - (uint16_t)1);
            nonzero += __builtin_elementwise_min(m, u16x2_t{1, 1});
            large = __builtin_elementwise_max(large, __builtin_bit_cast(i16x2_t, x));
            negative = __builtin_elementwise_max(negative, x);
        };
        each_vector<4>(row, V, tid, THREADS, [&](const uint4 &in, int) {
            look(in.x);
            look(in.y);
            look(in.z);
            look(in.w);
            elements += 8;
        }, [&](float x, int) {
            look(__float_as_uint(x) >> 16);
            ++elements;                                      // and a half that is zero
        });
        const bool odd = min(small[0], small[1]) < VALUE_LOW - 1 || max(large[0], large[1]) >= VALUE_HIGH || max(negative[0], negative[1]) > 0xff80u;
        zeros = (uint32_t)wave_inclusive_scan((int)(elements - nonzero[0] - nonzero[1]));
        if ((tid & 63) == 63 && zeros > 0) atomicAdd(&s.zeros, zeros);
        if (odd) s.odd = 1;
        __syncthreads();
        if (s.odd != 0) return false;
        zeros = s.zeros;
    }
    // the thread's bins: the largest value that there is, then the weights
    const Bins bins(tid);
    uint32_t count = 0;
    int first = THREADS * EACH;
#pragma unroll
    for (int j = EACH - 1; j >= 0; --j) {
        const uint32_t c = bins.count(s, j, zeros);
        count += c;
        first = c > 0 ? tid * EACH + j : first;
    }
    const uint64_t some = __ballot(count > 0);
    const int lowest = __builtin_amdgcn_readlane(first, some != 0 ? __ffsll((unsigned long long)some) - 1 : 0);       // by all lanes
    if ((tid & 63) == 0) s.waves.low[tid >> 6] = (uint32_t)lowest;
    __syncthreads();
    first = (tid & 63) < THREADS / 64 ? (int)s.waves.low[tid & 63] : THREADS * EACH;
    const uint64_t where = __ballot(first < THREADS * EACH);           // waves' bins are in order
    if (where == 0) return false;
    first = __builtin_amdgcn_readlane(first, __ffsll((unsigned long long)where) - 1);
    const Bins top_bins(first / EACH);
    const float top = top_bins.value(first % EACH);
    const auto answer_with = [&](float x, uint32_t which, int piece) {
        if (piece < 0) sample_index(s.waves, row, V, which, tid, x, answer);
        else if (tid < 64) sample_index_in(row, V, piece, tid, x, answer);
    };
    if (how.first) {
        if (tid == 0 && logp != nullptr) *logp = 0.f;
        answer_with(top, 0, __builtin_amdgcn_readfirstlane(top_bins.piece(s, first % EACH)));
        return true;
    }
    const SampleScale scale(top, how.temperature);
    uint64_t weight = 0;
    if (some != 0) {
#pragma unroll 1
        for (int j = 0; j < EACH; ++j) {
            const uint32_t c = bins.count(s, j, zeros);
            if (c > 0) weight += scale.of(bins.value(j)) * c;
        }
    }
    const SampleSums sums = sample_sums(s.waves, weight, count, tid);
    if (sums.count < (uint32_t)V && scale.live(VALUE_FAR)) return false;
    // The bin that a question leads to: one thread has it among its own, and every wave looks for it there, a lane a bin.
    struct Place {
        float value;
        uint64_t before_weight, weight;
        uint32_t before_count;
        int piece;
    };
    const auto locate = [&](int question, bool by_count, uint64_t need) {
        const uint64_t lo = by_count ? sums.before_count : sums.before_weight, hi = lo + (by_count ? count : weight);
        if (lo < need && need <= hi) {
            s.asked[question].thread = tid;
            s.asked[question].before_weight = sums.before_weight;
            s.asked[question].before_count = sums.before_count;
        }
        __syncthreads();
        const int lane = tid & 63;
        const Bins its(__builtin_amdgcn_readfirstlane(s.asked[question].thread));
        const float x = its.value(lane);
        const uint32_t c = its.count(s, lane, zeros);
        const uint64_t w = c > 0 ? scale.of(x) : 0;
        const uint64_t upto_weight = s.asked[question].before_weight + wave_sums_u64(w * c);
        const uint32_t upto_count = s.asked[question].before_count + (uint32_t)wave_inclusive_scan((int)c);
        const int found = __ffsll((unsigned long long)__ballot(need <= (by_count ? upto_count : upto_weight))) - 1;
        return Place{__uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), found)), lane_of_u64(upto_weight - w * c, found), lane_of_u64(w, found),
                     (uint32_t)__builtin_amdgcn_readlane((int)(upto_count - c), found), __builtin_amdgcn_readfirstlane(its.piece(s, found))};
    };
    uint64_t kept = sums.weight;
    if (how.top_k > 0 && (uint32_t)how.top_k < sums.count) {
        const Place p = locate(0, true, (uint64_t)how.top_k);
        kept = p.before_weight + (uint64_t)((uint32_t)how.top_k - p.before_count) * p.weight;
    }
    if (how.top_p < 1.f) {
        const uint64_t need = how.share(kept);
        if (need <= SAMPLE_ONE) {
            kept = SAMPLE_ONE;
        } else {
            const Place p = locate(1, false, need);
            kept = p.before_weight + (uint64_t)(sample_quotient(need - p.before_weight - 1, p.weight) + 1) * p.weight;
        }
    }
    if (how.min_p > 0.f) {
        const uint64_t least = how.least();
        uint64_t sum = 0;
#pragma unroll 1
        for (int j = 0; j < EACH; ++j) {
            const uint32_t c = bins.count(s, j, zeros);
            const uint64_t w = c > 0 ? scale.of(bins.value(j)) : 0;
            sum += w >= least ? w * c : 0;
        }
        kept = min(kept, sample_sum(s.waves, sum, tid));
    }
    const uint64_t goal = how.goal(kept);
    const Place p = locate(2, false, goal + 1);
    const float x = p.value;
    const uint32_t which = sample_quotient(goal - p.before_weight, p.weight);
    if (tid == 0 && logp != nullptr) *logp = (float)(((double)x - scale.top) / (double)how.temperature - log((double)kept / SAMPLE_UNIT));
    answer_with(x, which, p.piece);
    return true;
}

// ---- any values -------------------------------------------------------------------------------------------------------------

template <typename W>
__device__ __forceinline__ void sample_by_range(SampleBins &s, const W *row, int V, const SampleHow &how, int tid, int32_t *answer, float *logp)
{
    const int lane = tid & 63, wave = tid >> 6;
    __syncthreads();
    float top = -INFINITY, low = INFINITY;
    bool nan = false;
    each_logit<4>(row, V, tid, SAMPLE_THREADS, [&](float x, int) {
        top = fmaxf(top, x);
        low = fminf(low, x);
        nan = nan || x != x;
    });
    top = group_max<6>(top);
    low = -group_max<6>(-low);
    if (lane == 0) {
        s.waves.low[wave] = __float_as_uint(low);
        s.waves.count[wave] = __float_as_uint(top);
    }
    const auto clear = [&] {
#pragma unroll
        for (int j = 0; j < SAMPLE_EACH; ++j) {
            s.weight[j * SAMPLE_THREADS + tid] = 0;
            s.count[j * SAMPLE_THREADS + tid] = 0;
        }
        __syncthreads();
    };
    clear();
    for (int w = 0; w < SAMPLE_WAVES; ++w) {
        top = fmaxf(top, __uint_as_float(s.waves.count[w]));
        low = fminf(low, __uint_as_float(s.waves.low[w]));
    }
    nan = __syncthreads_or(nan);
    const bool none = !nan && top == -INFINITY;
    if (nan || none || top == INFINITY || how.first) {
        if (tid == 0 && logp != nullptr) *logp = none ? -INFINITY : 0.f;
        if (none && tid == 0) *answer = -1;
        if (!none) sample_index(s.waves, row, V, 0, tid, nan ? NAN : top, answer);
        return;
    }
    // Bins over the values that have a weight, or over all if these lie closer; every two of them have an entry of the table, from which a
    // weight is no further away than z = 0.0077: 2^44 exp(z) by five more terms of the series, within 2^-50 of its value.  All in 64 bits;
    // an infinite temperature has one bin.
    const bool flat = how.temperature == INFINITY;
    const double zero = (double)SAMPLE_ZERO * (double)how.temperature, range = flat ? 0.0 : fmin(zero, ((double)top - (double)low) * (1.0 + 0x1p-20));
    const double per = range > 0.0 ? SAMPLE_TABLE / range : 0.0, step = flat ? 0.0 : range / SAMPLE_TABLE / (double)how.temperature;
    for (int i = tid; i < SAMPLE_TABLE; i += SAMPLE_THREADS) s.table[i] = SAMPLE_UNIT * exp(-(i + 0.5) * step);
    const double c1 = -step, c2 = step * step / 2, c3 = c2 * c1 / 3, c4 = c3 * c1 / 4, c5 = c4 * c1 / 5;
    struct Spot {
        int bin;
        uint64_t weight;
    };
    const auto spot_of = [&](float x) {
        const double away = (double)top - (double)x, y = away * per;
        if (!(away < zero)) return Spot{SAMPLE_BINS - 1, 0};
        const int i = min((int)y, SAMPLE_TABLE - 1);
        const double d = __builtin_amdgcn_fract(y) - 0.5;
        const double p = fma(fma(fma(fma(fma(c5, d, c4), d, c3), d, c2), d, c1), d, 1.0);
        // the sum with 2^52 rounds to whole numbers, which are its lower bits
        const uint64_t bits = (uint64_t)__double_as_longlong(fma(s.table[i], p, 4503599627370496.0));
        return Spot{2 * i + (d >= 0.0 ? 1 : 0), bits & (((uint64_t)1 << 52) - 1)};
    };
    const auto bin_of = [&](float x) {
        const double away = (double)top - (double)x;
        return away < zero ? min((int)(away * (2 * per)), SAMPLE_BINS - 1) : SAMPLE_BINS - 1;
    };
    const auto weight_of = [&](float x) { return spot_of(x).weight; };
    __syncthreads();
    const bool counted = how.top_k > 0 && how.top_k < V;
    each_logit<4>(row, V, tid, SAMPLE_THREADS, [&](float x, int) {
        const Spot p = spot_of(x);
        if (counted) atomicAdd(&s.count[p.bin], 1u);
        if (p.weight > 0) atomicAdd(reinterpret_cast<unsigned long long *>(&s.weight[p.bin]), (unsigned long long)p.weight);
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
            w[j] = s.weight[tid * SAMPLE_EACH + j];
            c[j] = s.count[tid * SAMPLE_EACH + j];
            weight += w[j];
            count += c[j];
        }
    };
    read(w, c, weight, count);
    const SampleSums sums = sample_sums(s.waves, weight, count, tid);

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
        // in fp32, and with more than its error on both sides, what lies in the bin: all others are not looked at in 64 bits
        const float slack = 1e-6f * (fabsf(top) + (float)range);
        const double wide = 0.5 / per;
        const bool bounded = per > 0.0 && slack < 1e30f;
        const float from = bounded && bin < SAMPLE_BINS - 1 ? (float)((double)top - (bin + 1) * wide) - slack : -INFINITY;
        const float to = bounded ? (float)((double)top - bin * wide) + slack : INFINITY;
        uint32_t lo = 0xffffffffu, hi = 0;
        each_logit<4>(row, V, tid, SAMPLE_THREADS, [&](float x, int i) {
            if (x < from || x > to || bin_of(x) != bin) return;
            const uint64_t key = best_key(x, i);
            lo = min(lo, (uint32_t)(key >> 32));
            hi = max(hi, (uint32_t)(key >> 32));
            const uint32_t at = atomicAdd(&s.listed, 1u);
            if (at < SAMPLE_LIST) {
                s.list[at] = key;
                s.list_weight[at] = weight_of(x);
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
            s.waves.low[wave] = lo;
            s.waves.count[wave] = hi;
        }
        __syncthreads();
        for (int i = 0; i < SAMPLE_WAVES; ++i) {
            lo = min(lo, s.waves.low[i]);
            hi = max(hi, s.waves.count[i]);
        }
        __syncthreads();
        while (lo < hi) {
            const int shift = max(0, 32 - __clz(hi - lo) - 12);
            clear();
            each_logit<4>(row, V, tid, SAMPLE_THREADS, [&](float x, int) {
                const uint32_t o = best_order(x);
                if (o < lo || o > hi || bin_of(x) != bin) return;
                atomicAdd(&s.count[(hi - o) >> shift], 1u);
                const uint64_t w = weight_of(x);
                if (w > 0) atomicAdd(reinterpret_cast<unsigned long long *>(&s.weight[(hi - o) >> shift]), (unsigned long long)w);
            });
            __syncthreads();
            uint64_t w[SAMPLE_EACH], weight;
            uint32_t c[SAMPLE_EACH], count;
            read(w, c, weight, count);
            SampleSums inner = sample_sums(s.waves, weight, count, tid);
            inner.before_weight += before_weight;
            inner.before_count += before_count;
            find(inner, w, c, weight, count, by_count, need);
            before_weight = s.before_weight;
            before_count = s.before_count;
            hi -= (uint32_t)s.bin << shift;
            lo = max(lo, hi - min(hi, (1u << shift) - 1));
            __syncthreads();
        }
        const uint64_t each = weight_of(of_order(hi));
        const uint64_t tokens = by_count ? need - before_count : sample_quotient(need - before_weight - 1, each) + 1;
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
        // no weight behind that is so large: ln(2^44 / (least - 1/2)) and some more
        const float reach = (31.3f - logf((float)least)) * 1.001f * how.temperature;
        uint64_t sum = 0;
        each_logit<4>(row, V, tid, SAMPLE_THREADS, [&](float x, int) {
            if (top - x > reach) return;
            const uint64_t w = weight_of(x);
            sum += w >= least ? w : 0;
        });
        kept = min(kept, sample_sum(s.waves, sum, tid));
    }
    const Place p = locate(false, how.goal(kept) + 1);
    if (tid == 0) {
        if (logp != nullptr) *logp = (float)(((double)of_order(p.order) - (double)top) / (double)how.temperature - log((double)kept / SAMPLE_UNIT));
        if (p.index >= 0) *answer = p.index;
    }
    if (p.index < 0) sample_index(s.waves, row, V, p.which, tid, of_order(p.order), answer);
}

// One block a row.  WAYS: by value, and by range where that does not do (one launch); by value only, and SAMPLE_LATER for such a row;
// by range only, the rows that were left.
constexpr int SAMPLE_LATER = -2;
enum class SampleWays { ALL, VALUE, LEFT };
constexpr int VALUE_THREADS = 512;
template <typename W, SampleWays WAYS>
constexpr int sample_threads() { return WAYS == SampleWays::VALUE ? VALUE_THREADS : SAMPLE_THREADS; }
template <typename W, SampleWays WAYS>
constexpr size_t sample_lds()
{
    constexpr size_t values = sizeof(W) == 2 && WAYS != SampleWays::LEFT ? sizeof(SampleValues<sample_threads<W, WAYS>()>) : 0;
    return WAYS != SampleWays::VALUE && sizeof(SampleBins) > values ? sizeof(SampleBins) : values;
}
template <typename W, SampleWays WAYS>
__global__ __launch_bounds__((sample_threads<W, WAYS>()), WAYS == SampleWays::VALUE ? 8 : 4) void k_sample(SampleArgs A)
{
    constexpr int THREADS = sample_threads<W, WAYS>();
    constexpr bool BY_VALUE = sizeof(W) == 2 && WAYS != SampleWays::LEFT, BY_RANGE = WAYS != SampleWays::VALUE;
    extern __shared__ __align__(16) char sample_smem[];
    auto &values = *reinterpret_cast<SampleValues<BY_VALUE ? THREADS : 64> *>(sample_smem);
    auto &bins = *reinterpret_cast<SampleBins *>(sample_smem);
    const int tid = threadIdx.x, t = blockIdx.x;
    if (WAYS == SampleWays::LEFT && A.answers[t] != SAMPLE_LATER) return;
    const W *row = static_cast<const W *>(A.logits) + (int64_t)t * A.stride;
    const float temperature = A.temperature != nullptr ? A.temperature[t] : 1.f;
    const SampleHow how{temperature, A.top_p != nullptr ? A.top_p[t] : 1.f, A.min_p != nullptr ? A.min_p[t] : 0.f, A.u[t], A.top_k != nullptr ? A.top_k[t] : 0,
                        !(temperature > 0.f)};
    float *logp = A.logp != nullptr ? A.logp + t : nullptr;
    if constexpr (BY_VALUE && BY_RANGE) {
        if (sample_by_value<THREADS>(values, row, A.V, how, tid, A.answers + t, logp)) return;
        __syncthreads();                    // the bins lie where other waves may still read why the row goes this way
        sample_by_range(bins, row, A.V, how, tid, A.answers + t, logp);
    } else if constexpr (BY_VALUE) {
        if (!sample_by_value<THREADS>(values, row, A.V, how, tid, A.answers + t, logp) && tid == 0) A.answers[t] = SAMPLE_LATER;
    } else {
        sample_by_range(bins, row, A.V, how, tid, A.answers + t, logp);
    }
}

}  // namespace svdp
