// Attention of drafted tokens over paged K and V and over their own tree:
//   out[t][h] = sum_j softmax_j(scale q[t][h] . k_j) v_j
// over the cached tokens of t's request and the nodes of its tree that t sees.
//
// Rows and tiles.  The query heads that share a head of K and V, times the nodes of a request, are the rows of one matrix
// product: K and V are read once for all of them.  A wave takes tiles of 32 tokens and 16 NT rows, on the matrix cores:
//   S^T = K Q^T     A operand: tokens x channels, B operand: channels x rows; a lane ends up with 8 scores of ONE row
//   O^T += V^T P^T  A operand: channels x tokens, B operand: tokens x rows
// The tokens that a lane's K rows stand for are chosen so that the 8 weights which a lane then holds are the 8 tokens
// that the second product's B operand wants in that lane: the weights never leave their registers.  V is kept with e tokens of a channel
// side by side, so its operand is a 16-byte load as well: neither K nor V passes through LDS, and a tile of each is one contiguous
// piece of memory (8 KB for bf16 and 128 channels).
//
// Division of the work.  A unit is four tiles (one a wave).  All units of all requests, heads and row tiles stand in a
// row, and each block takes an equal piece of it, whatever the requests' lengths are (they are known on the device only).  What a block
// has of a (request, head, row tile) goes to the output where it is the whole of it, and otherwise, as a sum with its maximum, to
// the workspace, where k_tree_join puts the parts together.
//
// What bounds it: reading K and V.  24 requests of 3000 tokens, one row a head, bf16, 128 channels: 1180 MB in 199 us, 5.9 TB/s;
// a ragged batch of 592 MB in 106 us; 32 rows over 30 000 tokens, 123 MB, in 26.0 us, of which some 5 go by before and behind the
// reading.  One row over 780 tokens, 12.8 MB, takes 7.6 us, the latency of five loads after each other (lengths, page, K and V, parts).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "svdp_device.h"

namespace svdp {

constexpr int TA_WAVES = 4, TA_THREADS = 64 * TA_WAVES;
constexpr int TA_TILE = 32;                      // tokens of a tile; divides every page
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

typedef __bf16 ta_bf16x8 __attribute__((ext_vector_type(8)));
typedef float ta_f32x8 __attribute__((ext_vector_type(8)));

// What the division of the work and the join need, in front: 16 words, which a wave finds in its registers when it starts.
struct TreeJoinArgs {
    const int32_t *lens, *starts;
    void *out;
    float *lse;
    float *parts;                       // [2 << Cut::BITS] parts of tree_part_floats(part_rows, dim)
    int room, heads, group, R, T;       // room: tokens that a request's row of the table can have
    uint16_t max_nodes;
    uint16_t part_rows;                 // rows of a part: no more than a request has, nor a block; 0: nothing is cut
};
static_assert(sizeof(TreeJoinArgs) == 64, "as many as are loaded ahead");
struct TreeAttnArgs : TreeJoinArgs {
    const void *K, *V;                  // of the layer
    const uint8_t *K_scale, *V_scale;   // of a cache in 8 bits
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    const uint64_t *tree;
    const int32_t *table;
    float scale;
    int max_pages, pages, page_bits;
};

// How a kernel cuts the work: ROWS rows a block, units of TILES tiles, 1 << BITS blocks; the tree's own tiles follow the cached
// ones, or begin a unit of their own.
template <int ROWS_, int TILES, int BITS_, bool APART>
struct TreeCut {
    static constexpr int ROWS = ROWS_, UNIT = TILES, BITS = BITS_;
    static __device__ __forceinline__ int steps(int tiles, int n)
    {
        const int more = (n + TA_TILE - 1) / TA_TILE;
        return APART ? (tiles + TILES - 1) / TILES + (more + TILES - 1) / TILES : (tiles + more + TILES - 1) / TILES;
    }
};

typedef const __attribute__((address_space(4))) int32_t *table_t;            // read through the scalar cache

// One request's share: rows, tiles, and units: as many as its steps for each head and row tile, or one where nothing is cut.
struct TreeSpan {
    int len, start, n, tiles, steps, cuts, row_tiles, units;
};
template <typename Cut>
__device__ __forceinline__ TreeSpan tree_span(const TreeJoinArgs &A, int len, int start, int n)
{
    constexpr int ROWS = Cut::ROWS;
    TreeSpan s{len, start, n};
    s.tiles = (s.len + TA_TILE - 1) / TA_TILE;
    s.steps = Cut::steps(s.tiles, s.n);
    s.cuts = A.part_rows == 0 ? min(s.steps, 1) : s.steps;
    s.row_tiles = (s.n * A.group + ROWS - 1) / ROWS;
    s.units = s.row_tiles * s.cuts * A.heads;
    return s;
}
// 64 requests, a lane each: what there is of them, their units and the inclusive sums of these.  They are read once, all
// together; a request's share is then read out of its lane.
template <typename Cut>
struct TreeChunk {
    int first, len, start, n, units, upto;
    __device__ __forceinline__ void load(const TreeJoinArgs &A, int lane, int at)
    {
        const int r = at + lane, i = min(r, A.R - 1);
        const int raw_len = A.lens[i], raw_start = A.starts[i], raw_end = A.starts[i + 1];
        first = at;
        len = min(max(raw_len, 0), A.room);
        start = min(max(raw_start, 0), A.T);
        n = r < A.R ? min(min(max(raw_end - start, 0), (int)A.max_nodes), A.T - start) : 0;
        units = tree_span<Cut>(A, len, start, n).units;              // none without rows
        upto = wave_inclusive_scan(units);
    }
    __device__ __forceinline__ int all() const { return __builtin_amdgcn_readlane(upto, 63); }
    __device__ __forceinline__ int before(int l) const { return __builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(units, l); }
    __device__ __forceinline__ TreeSpan span(const TreeJoinArgs &A, int l) const
    {
        return tree_span<Cut>(A, __builtin_amdgcn_readlane(len, l), __builtin_amdgcn_readlane(start, l), __builtin_amdgcn_readlane(n, l));
    }
};

// The same value, of which the compiler knows nothing: what is computed from it stays where it is written.  Without it, what the
// rare parts of a loop need per lane is kept in registers that the products' operands could be read ahead into.
__device__ __forceinline__ int here(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

__device__ __forceinline__ int lane_of_first(uint64_t ballot) { return __ffsll((unsigned long long)ballot) - 1; }

// Units of all requests; the first 64 of them stay in the chunk.
template <typename Cut>
__device__ __forceinline__ int tree_units(const TreeJoinArgs &A, int lane, TreeChunk<Cut> &chunk)
{
    chunk.load(A, lane, 0);
    int all = chunk.all();
    for (int c = 64; c < A.R; c += 64) {
        TreeChunk<Cut> other;
        other.load(A, lane, c);
        all += other.all();
    }
    return all;
}

// The unit where block b begins: an equal share for each, or one unit each for the first blocks.  No block in between has none.
template <typename Cut>
__device__ __forceinline__ int tree_begin(int b, int units)
{
    return units >> Cut::BITS == 0 ? min(b, units) : (int)(((int64_t)b * units) >> Cut::BITS);
}
// The block that has unit u: the first one whose successor begins behind u.  A quotient in fp32 is at most one off (its relative
// error is some 2^-22, of 512 at the most), and put right; a 64-bit division would take as long as a load.
template <typename Cut>
__device__ __forceinline__ int tree_block_of(int u, int units)
{
    if (units >> Cut::BITS == 0) return u;
    int b = min((int)((float)u * (float)(1 << Cut::BITS) * __builtin_amdgcn_rcpf((float)units)), (1 << Cut::BITS) - 1);
    if (tree_begin<Cut>(b, units) > u) --b;
    if (tree_begin<Cut>(b + 1, units) <= u) ++b;
    return b;
}

// The request that unit u belongs to, as the lane that has it in the chunk, and how far into it that is.
template <typename Cut>
__device__ __forceinline__ int tree_request(const TreeJoinArgs &A, int u, int lane, TreeChunk<Cut> &chunk, int *rem)
{
    for (int base = 0;; base += chunk.all(), chunk.load(A, lane, chunk.first + 64)) {
        const uint64_t behind = __ballot(base + chunk.upto > u);
        if (behind != 0) {
            const int l = lane_of_first(behind);
            *rem = u - base - chunk.before(l);
            return l;
        }
    }
}

// Floats of a part: its rows' sums and behind them their maxima and denominators, up to whole 16 bytes, which it is written and read in.
__host__ __device__ constexpr size_t tree_part_floats(int rows, int dim) { return ((size_t)rows * (dim + 2) + 3) & ~(size_t)3; }
static_assert(tree_part_floats(1, 128) == 132 && tree_part_floats(7, 64) == 464 && tree_part_floats(256, 128) == 256 * 130);
// A part's address: block b has two.
__device__ __forceinline__ float *tree_part(const TreeJoinArgs &A, int b, int which, int dim)
{
    return A.parts + (size_t)(2 * b + which) * tree_part_floats(A.part_rows, dim);
}

// ---- operands, by storage type --------------------------------------------------------------------------------------------
// Lane = 16 g + m.  KEY(t, m): the token of a tile whose K row m of the t-th product comes from; the result's rows 4 g + i lie
// in lane group g, so that this lane group ends up with the tokens KEY(t, 4 g + i), which are those it has of V below.
template <typename W, int DIM>
struct TreeTile;

template <int DIM>
struct TreeTile<bf16, DIM> {
    using Row = bf16;
    static constexpr bool CODED = false;
    static constexpr uint32_t SIGNS = 0x80008000u;
    static constexpr int E = 8, KC = DIM / 32, VT = 1;
    static __device__ __forceinline__ int channel(int c, int g) { return (4 * c + g) * E; }      // first of E, of Q and K, in product c
    static __device__ __forceinline__ int v_channel(int dt, int m) { return 16 * dt + m; }       // of V, in product dt
    static __device__ __forceinline__ int key(int t, int m) { return (m >> 2) * 8 + (m & 3) + 4 * t; }
    static __device__ __forceinline__ int pack(int, int g) { return g; }          // of 8 tokens
    static __device__ __forceinline__ f32x4_t score(const uint4 &k, const uint4 &q, f32x4_t s)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(ta_bf16x8, k), __builtin_bit_cast(ta_bf16x8, q), s, 0, 0, 0);
    }
    // The weights of a lane's 8 tokens as two terms, hi + lo, each for its own product with V: within 2^-15 of the fp32 weight (one
    // term: 2^-8, as much as the output's own rounding).  hi lies below the weight by half of its last place at the least, so that neither
    // term of a weight is zero or negative: an infinity in V stays one.
    struct Weights {
        uint4 hi, lo;
    };
    static __device__ __forceinline__ Weights pack_weights(const float (&p)[8])
    {
        uint32_t hi[4];
        ta_f32x8 rest;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t a = __builtin_elementwise_sub_sat(__float_as_uint(p[2 * i]), 0x8000u);
            const uint32_t b = __builtin_elementwise_sub_sat(__float_as_uint(p[2 * i + 1]), 0x8000u);
            hi[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);            // the upper halves of a and b
            rest[2 * i] = p[2 * i] - __uint_as_float(a & 0xffff0000u);     // exact
            rest[2 * i + 1] = p[2 * i + 1] - __uint_as_float(b & 0xffff0000u);
        }
        return {make_uint4(hi[0], hi[1], hi[2], hi[3]), __builtin_bit_cast(uint4, __builtin_convertvector(rest, ta_bf16x8))};
    }
    static __device__ __forceinline__ f32x4_t sum(const uint4 (&v)[1], const Weights &p, f32x4_t o)
    {
        return score(v[0], p.lo, score(v[0], p.hi, o));
    }
    // each element: f(its bits in front of 16 zeros) as a new element
    template <typename F>
    static __device__ __forceinline__ uint4 each(const uint4 &v, F &&f)
    {
        const auto two = [&](uint32_t w) { return (f(w << 16) >> 16) | (f(w & 0xffff0000u) & 0xffff0000u); };
        return make_uint4(two(v.x), two(v.y), two(v.z), two(v.w));
    }
    static __device__ __forceinline__ bool finite(const uint4 &v)
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        bool ok = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) ok = ok && (w[i] & 0x7f80u) != 0x7f80u && (w[i] & 0x7f800000u) != 0x7f800000u;
        return ok;
    }
    // the first n of 8 tokens, zeros behind them
    static __device__ __forceinline__ uint4 first(const uint4 &v, int n)
    {
        const auto keep = [&](uint32_t w, int at) { return n >= at + 2 ? w : n == at + 1 ? w & 0xffffu : 0u; };
        return make_uint4(keep(v.x, 0), keep(v.y, 2), keep(v.z, 4), keep(v.w, 6));
    }
};

template <int DIM>
struct TreeTile<float, DIM> {
    using Row = float;
    static constexpr bool CODED = false;
    static constexpr uint32_t SIGNS = 0x80000000u;
    static constexpr int E = 4, KC = DIM / 16, VT = 2;
    static __device__ __forceinline__ int channel(int c, int g) { return (4 * c + g) * E; }
    static __device__ __forceinline__ int v_channel(int dt, int m) { return 16 * dt + m; }
    static __device__ __forceinline__ int key(int t, int m) { return 16 * t + m; }
    static __device__ __forceinline__ int pack(int t, int g) { return 4 * t + g; } // of 4 tokens
    static __device__ __forceinline__ f32x4_t score(const uint4 &k, const uint4 &q, f32x4_t s)
    {
        const float4 a = as_float4(k), b = as_float4(q);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x, b.x, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(a.y, b.y, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(a.z, b.z, s, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x4f32(a.w, b.w, s, 0, 0, 0);
    }
    struct Weights {
        float p[8];
    };
    static __device__ __forceinline__ Weights pack_weights(const float (&p)[8])
    {
        Weights w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.p[i] = p[i];
        return w;
    }
    template <typename F>
    static __device__ __forceinline__ uint4 each(const uint4 &v, F &&f)
    {
        return make_uint4(f(v.x), f(v.y), f(v.z), f(v.w));
    }
    static __device__ __forceinline__ f32x4_t sum(const uint4 (&v)[2], const Weights &w, f32x4_t o)
    {
        const float (&p)[8] = w.p;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float4 a = as_float4(v[t]);
            o = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x, p[4 * t], o, 0, 0, 0);
            o = __builtin_amdgcn_mfma_f32_16x16x4f32(a.y, p[4 * t + 1], o, 0, 0, 0);
            o = __builtin_amdgcn_mfma_f32_16x16x4f32(a.z, p[4 * t + 2], o, 0, 0, 0);
            o = __builtin_amdgcn_mfma_f32_16x16x4f32(a.w, p[4 * t + 3], o, 0, 0, 0);
        }
        return o;
    }
    static __device__ __forceinline__ bool finite(const uint4 &v)
    {
        return (v.x & 0x7f800000u) != 0x7f800000u && (v.y & 0x7f800000u) != 0x7f800000u && (v.z & 0x7f800000u) != 0x7f800000u &&
               (v.w & 0x7f800000u) != 0x7f800000u;
    }
    static __device__ __forceinline__ uint4 first(const uint4 &v, int n)
    {
        return make_uint4(n > 0 ? v.x : 0u, n > 1 ? v.y : 0u, n > 2 ? v.z : 0u, n > 3 ? v.w : 0u);
    }
};

// A cache in 8 bits: its elements become bf16 operands in registers, with their tokens' powers of two: K's (one token a lane) in the
// conversion, V's (eight tokens in an operand, one power each) as fp32, which is rounded to bf16, exactly.  Multiplied into the weights
// instead, which are up to 2^SLACK, powers near either end of fp32's range would make them infinite or cost them their second terms.  That was
// no faster either: eight requests of 4096 tokens, 32 rows 27.4 us against 26.5, 64 rows 40.6 against 38.6.
// A lane's 16 bytes are the operands of two products, so that the channels that a product takes are others than in 16 bits.
// 24 requests of 500 to 16 384 tokens, four query heads a head, 210 MB: 42 to 49 us, 4.3 to 5.0 TB/s, of which some 5 us go by before and
// behind the reading; half of what 16 bits take.
template <int DIM>
struct TreeTile<e4m3, DIM> : TreeTile<bf16, DIM> {
    static constexpr bool CODED = true;
    static __device__ __forceinline__ int channel(int c, int g) { return (c >> 1) * 64 + g * 16 + (c & 1) * 8; }
    static __device__ __forceinline__ int v_channel(int dt, int m) { return (dt >> 1) * 32 + 2 * m + (dt & 1); }
    static __device__ __forceinline__ uint4 operand(const uint4 &raw, int half, float by)
    {
        return half == 0 ? widen_e4m3(raw.x, raw.y, by) : widen_e4m3(raw.z, raw.w, by);
    }
    // the first n of eight tokens' powers, 2^0 behind them
    static __device__ __forceinline__ uint64_t first_powers(uint64_t by, int n)
    {
        const uint64_t keep = n >= 8 ? ~0ull : n <= 0 ? 0ull : (1ull << (8 * n)) - 1;
        return (by & keep) | (0x7f7f7f7f7f7f7f7full & ~keep);
    }
    // eight tokens of a channel, each with its own power
    static __device__ __forceinline__ uint4 decoded(uint32_t a, uint32_t b, uint64_t by)
    {
        ta_f32x8 x;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t w = i == 0 ? a : b, s = (uint32_t)(by >> (32 * i));
            const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), high = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
            x[4 * i] = low[0] * power_of(s & 0xffu);
            x[4 * i + 1] = low[1] * power_of((s >> 8) & 0xffu);
            x[4 * i + 2] = high[0] * power_of((s >> 16) & 0xffu);
            x[4 * i + 3] = high[1] * power_of(s >> 24);
        }
        return __builtin_bit_cast(uint4, __builtin_convertvector(x, ta_bf16x8));
    }
    // the first n of 8 tokens of two channels, zeros behind them
    static __device__ __forceinline__ uint4 first_coded(const uint4 &v, int n)
    {
        const uint32_t a = n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1, b = n >= 8 ? ~0u : n <= 4 ? 0u : (1u << (8 * (n - 4))) - 1;
        return make_uint4(v.x & a, v.y & b, v.z & a, v.w & b);
    }
};

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }
// Scores are taken relative to a `shift` that follows their maximum, in base two: it moves only where a score exceeds it by more than
// SLACK (then to the maximum), so that the sums are rarely brought down to a new one.  A weight is then at most 2^SLACK, far from any
// limit of fp32 (and of bf16, which has the same exponents).
constexpr float SLACK = 8.f;
// -inf (nothing but zero weights so far) must not make -inf - -inf
__device__ __forceinline__ float finite_shift(float shift) { return shift == -INFINITY ? 0.f : shift; }

// Infinities and NaN in V where not every row sees every token: a weight of zero would not hide them from a product.  So that is
// taken over the finite elements, and for each of +inf, -inf and NaN it is counted how many of them a row sees.
__device__ __forceinline__ bool is_finite_bits(uint32_t u) { return (u & 0x7f800000u) != 0x7f800000u; }
template <typename X>
__device__ __forceinline__ uint4 only_finite(const uint4 &v)
{
    return X::each(v, [](uint32_t u) { return is_finite_bits(u) ? u : 0u; });
}
__device__ __forceinline__ float value_of_kind(int kind) { return kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN; }
template <typename X>
__device__ __forceinline__ uint4 ones_of_kind(const uint4 &v, int kind)
{
    const uint32_t inf = kind == 0 ? 0x7f800000u : 0xff800000u;
    return X::each(v, [&](uint32_t u) {
        return (kind == 2 ? !is_finite_bits(u) && (u & 0x007fffffu) != 0 : u == inf) ? 0x3f800000u : 0u;
    });
}

// What a wave has of its rows: the sum O^T (channels 16 dt + 4 g + i of row m), the shift, and the lane group's part of the denominator.
template <typename W, int DIM, int NT>
struct TreeWave {
    using X = TreeTile<W, DIM>;
    using Weights = typename X::Weights;
    static constexpr int DT = DIM / 16, VT = X::VT;
    f32x4_t o[DT][NT];
    float shift[NT], total[NT];         // shift: zero for a row that has not seen anything
    float limit[NT];                    // what a relative score has to exceed for the shift to move: -inf for such a row

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            shift[nt] = 0.f;
            limit[nt] = -INFINITY;
            total[nt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt][nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    }
    // the maximum that others compare theirs with: -inf for a row that has not seen anything
    __device__ __forceinline__ float top(int nt) const { return limit[nt] == -INFINITY ? -INFINITY : shift[nt]; }

    // Scores in base two, relative to the shift -> weights.
    template <int N>
    __device__ __forceinline__ void weights(float (&z)[NT][8 * N], Weights (&w)[NT][N])
    {
        float top[NT];
        bool grew = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float t = z[nt][0];
#pragma unroll
            for (int i = 1; i < 8 * N; ++i) t = fmaxf(t, z[nt][i]);
            top[nt] = max_xor32(max_xor16(t));
            grew = grew || top[nt] > limit[nt];
        }
        if (__any(grew)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float to = top[nt] > limit[nt] ? shift[nt] + top[nt] : shift[nt];
                // nothing so far: there is nothing to bring down, and the shift may come down itself
                const float down = to - shift[nt], old = limit[nt] == -INFINITY ? 0.f : exp2_fast(-down);
                shift[nt] = to;
                limit[nt] = top[nt] > limit[nt] ? SLACK : limit[nt];
                total[nt] *= old;
#pragma unroll
                for (int i = 0; i < 8 * N; ++i) z[nt][i] -= down;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt][nt] *= old;
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float e[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = exp2_fast(z[nt][8 * n + i]);
                total[nt] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
                w[nt][n] = X::pack_weights(e);
            }
    }
    // One V operand (16 channels) against the weights of all rows.
    template <int N>
    __device__ __forceinline__ void add(int dt, const uint4 (&v)[VT], const Weights (&w)[NT][N], int n = 0)
    {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[dt][nt] = X::sum(v, w[nt][n], o[dt][nt]);
    }
    // What V's infinities and NaN add (see only_finite).
    __device__ __forceinline__ void add_special(int dt, const uint4 (&v)[VT], const uint32_t (&mask)[NT])
    {
        uint4 part[VT];
#pragma unroll 1
        for (int kind = 0; kind < 3; ++kind) {
#pragma unroll
            for (int t = 0; t < VT; ++t) part[t] = ones_of_kind<X>(v[t], kind);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float seen[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) seen[i] = (mask[nt] >> i) & 1 ? 1.f : 0.f;
                const f32x4_t count = X::sum(part, X::pack_weights(seen), f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int c = 0; c < 4; ++c) o[dt][nt][c] += count[c] > 0.f ? value_of_kind(kind) : 0.f;
            }
        }
    }
};

// Scores stay in units of |scale| > 0, so that the sign goes to Q; for a scale of zero Q is zero, and the unit one.
struct TreeScale {
    float unit;
    uint32_t stays, flip;
    __device__ __forceinline__ TreeScale(float scale, uint32_t signs)
    {
        unit = fabsf(scale) * LOG2E;
        stays = unit == 0.f ? 0u : ~0u;
        unit = unit == 0.f ? 1.f : unit;
        flip = scale < 0.f ? signs : 0u;
    }
    __device__ __forceinline__ uint4 of(const uint4 &q) const
    {
        return make_uint4((q.x & stays) ^ flip, (q.y & stays) ^ flip, (q.z & stays) ^ flip, (q.w & stays) ^ flip);
    }
};

// One block: its piece of the row of units, a segment (what it has of one request, head and row tile) after the other.
// Waves of a SIMD that its registers have room for: the sum, Q, and one tile of K and of V.  (Three where they would fit measured
// the same as two.)
constexpr int ta_waves(int element, int dim, int nt)
{
    return nt * (dim / 4 + dim * element / 16) + 2 * dim * element / 8 <= 200 ? 2 : 1;
}
// One block a compute unit, so that there are few parts to join (32 rows over 30 000 tokens: 25.9 + 4.2 us; with 512 blocks
// 25.9 + 4.8).  Two where the registers have room and the parts are small: their starts and ends overlap (a ragged batch
// of eight requests, 590 MB: 108.5 us; with 256 blocks 112).
template <typename W, int DIM, int NT>
constexpr int ta_waves_of() { return ta_waves(sizeof(typename RowOf<W>::type), DIM, NT); }
template <typename W, int DIM, int NT>
using NarrowCut = TreeCut<16 * NT, TA_WAVES, NT == 1 && ta_waves_of<W, DIM, NT>() == 2 ? 9 : 8, false>;

template <typename W, int DIM, int NT>
__global__ __launch_bounds__(TA_THREADS, (ta_waves_of<W, DIM, NT>())) void k_tree_attn(TreeAttnArgs A)
{
    using X = TreeTile<W, DIM>;
    using Row = typename X::Row;
    using Cut = NarrowCut<W, DIM, NT>;
    constexpr int ROWS = Cut::ROWS, E = X::E, KC = X::KC, VT = X::VT, DT = DIM / 16;
    constexpr int DC = DIM * NT <= 128 ? DIM : 128 / NT;       // channels that the waves' sums meet in LDS by: 32 KB
    __shared__ float s_top[TA_WAVES][ROWS], s_total[TA_WAVES][ROWS];
    __shared__ __align__(16) float s_sum[TA_WAVES][ROWS][DC + 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, m = lane & 15;
    const int heads_q = A.heads * A.group;

    TreeChunk<Cut> chunk;
    const int units = tree_units(A, lane, chunk);
    int u = tree_begin<Cut>(blockIdx.x, units);
    const int u1 = tree_begin<Cut>(blockIdx.x + 1, units);
    if (u >= u1) return;
    int rem, l = tree_request(A, u, lane, chunk, &rem);

    for (bool first = true; u < u1; ++l, rem = 0) {
        if (l == 64) {
            chunk.load(A, lane, chunk.first + 64);
            l = 0;
        }
        const TreeSpan S = chunk.span(A, l);
        if (S.units == 0) continue;
        const int r = chunk.first + l;
        const table_t table = (table_t)(uintptr_t)(A.table + (size_t)r * A.max_pages);
        int task = rem / S.cuts, s0 = rem - task * S.cuts;
        for (; task < A.heads * S.row_tiles && u < u1; ++task, s0 = 0, first = false) {
            const int s1 = A.part_rows == 0 ? S.steps : min(S.steps, s0 + u1 - u);
            const int h = task / S.row_tiles, row0 = (task - h * S.row_tiles) * ROWS, rows = S.n * A.group;
            const bool whole = s0 == 0 && s1 == S.steps;

            // Q of the rows (a row past the last one repeats it: computed and never written)
            uint4 q[KC][NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int row = min(row0 + 16 * nt + m, rows - 1), node = row / A.group, head = h * A.group + row - node * A.group;
                const Row *from = static_cast<const Row *>(A.q) + (S.start + node) * A.q_stride + (int64_t)head * DIM;
#pragma unroll
                for (int c = 0; c < KC; ++c) q[c][nt] = load_raw(from + X::channel(c, g));
            }

            // cached tokens: K of the next tile is requested when this one's has been used, and so is V
            int i = s0 * TA_WAVES + wave, id = -1, id_next = -1;
            const int i_end = min(s1 * TA_WAVES, S.tiles), per_page = A.page_bits - 5;
            const auto page_of = [&](int tile) { return table[min(tile, S.tiles - 1) >> per_page]; };
            const auto real = [&](int id) { return (uint32_t)id < (uint32_t)A.pages; };
            const auto tile_at = [&](int tile, int id) {
                const int64_t page = (int64_t)(real(id) ? id : 0) * A.heads + h;
                return (((page << per_page) + (tile & ((1 << per_page) - 1))) * TA_TILE) * DIM;
            };
            const TreeScale scale(A.scale, X::SIGNS);
            const auto scale_q = [&] {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < KC; ++c) q[c][nt] = scale.of(q[c][nt]);
            };
            TreeWave<W, DIM, NT> mine;
            typename X::Weights p[NT][1];
            mine.clear();
            const auto scores = [&](const uint4 (&k)[2][KC], float (&z)[NT][8]) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int c = 0; c < KC; ++c) s = X::score(k[t][c], q[c][nt], s);
#pragma unroll
                        for (int i = 0; i < 4; ++i) z[nt][4 * t + i] = fmaf(s[i], scale.unit, -mine.shift[nt]);
                    }
            };

            if (i >= i_end) {
                scale_q();
            } else {
                // what a lane holds of a tile: operands, or in 8 bits what they are made of
                constexpr int KR = X::CODED ? KC / 2 : KC, VR = X::CODED ? DT / 2 : DT;
                uint4 k[2][KR], v[VR][VT];
                uint32_t k_by[2];
                uint64_t v_by;
                const auto load_k = [&](int64_t at) {
                    const W *from = static_cast<const W *>(A.K) + at;
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
#pragma unroll
                        for (int c = 0; c < KR; ++c) k[t][c] = load_raw(from + X::key(t, m) * DIM + X::channel(X::CODED ? 2 * c : c, g));
                        if constexpr (X::CODED) k_by[t] = A.K_scale[at / DIM + X::key(t, m)];
                    }
                };
                const auto load_v = [&](int64_t at) {
                    const W *from = static_cast<const W *>(A.V) + at;
#pragma unroll
                    for (int dt = 0; dt < VR; ++dt)
#pragma unroll
                        for (int t = 0; t < VT; ++t) v[dt][t] = load_raw(from + (X::pack(t, g) * DIM + X::v_channel(X::CODED ? 2 * dt : dt, m)) * E);
                    if constexpr (X::CODED) v_by = *reinterpret_cast<const uint64_t *>(A.V_scale + at / DIM + 8 * g);
                };
                id = page_of(i);
                id_next = page_of(i + TA_WAVES);
                load_k(tile_at(i, id));
                load_v(tile_at(i, id));
                scale_q();                                       // only now what waits for Q
                for (; i < i_end; i += TA_WAVES) {
                    const int count = real(id) ? min(S.len - i * TA_TILE, TA_TILE) : 0;
                    id = id_next;
                    id_next = page_of(i + 2 * TA_WAVES);
                    const int64_t at = tile_at(min(i + TA_WAVES, S.tiles - 1), id);
                    float z[NT][8];
                    if constexpr (X::CODED) {
                        uint4 wide[2][KC];
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int c = 0; c < KC; ++c) wide[t][c] = X::operand(k[t][c >> 1], c & 1, power_of(k_by[t]));
                        scores(wide, z);
                    } else {
                        scores(k, z);
                    }
                    if (i + TA_WAVES < i_end) load_k(at);
                    if (count < TA_TILE) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const bool behind = X::key(j >> 2, 4 * g + (j & 3)) >= count;
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
                                if (behind) z[nt][j] = -INFINITY;
                        }
                        if constexpr (X::CODED) v_by = X::first_powers(v_by, count - 8 * g);
#pragma unroll
                        for (int dt = 0; dt < VR; ++dt)
#pragma unroll
                            for (int t = 0; t < VT; ++t) {
                                if constexpr (X::CODED) v[dt][t] = X::first_coded(v[dt][t], count - X::pack(t, g) * E);
                                else v[dt][t] = X::first(v[dt][t], count - X::pack(t, g) * E);
                            }
                    }
                    mine.template weights<1>(z, p);
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        if constexpr (X::CODED) {
                            const uint4 &raw = v[dt >> 1][0], wide[1] = {dt & 1 ? X::decoded(raw.z, raw.w, v_by) : X::decoded(raw.x, raw.y, v_by)};
                            mine.add(dt, wide, p);
                        } else {
                            mine.add(dt, v[dt], p);
                        }
                    }
                    if (i + TA_WAVES < i_end) load_v(at);
                }
            }

            // the tree's own tokens
#pragma unroll 1
            for (; i < min(s1 * TA_WAVES, S.tiles + (S.n + TA_TILE - 1) / TA_TILE); i += TA_WAVES) {
                const int g = here(lane) >> 4, m = here(lane) & 15;
                const int node0 = (i - S.tiles) * TA_TILE;
                const Row *key = static_cast<const Row *>(A.k) + (int64_t)h * DIM, *value = static_cast<const Row *>(A.v) + (int64_t)h * DIM;
                // K, what the rows see, and (where the registers have room) V, all requested before anything is waited for
                constexpr bool EARLY = NT * DIM <= 128 && DIM * (int)sizeof(Row) <= 256;
                uint4 k[2][KC], v[DT][VT];
                uint64_t sees[NT];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const Row *from = key + (S.start + min(node0 + X::key(t, m), S.n - 1)) * A.k_stride;
#pragma unroll
                    for (int c = 0; c < KC; ++c) k[t][c] = load_raw(from + X::channel(c, g));
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int node = min(row0 + 16 * nt + m, rows - 1) / A.group;
                    sees[nt] = A.tree != nullptr ? A.tree[S.start + node] : ~0ull >> (63 - node);
                }
                // these rows of V lie token by token: an operand is put together from its elements
                const auto read_v = [&](int dt, uint4 (&to)[VT]) {
#pragma unroll
                    for (int t = 0; t < VT; ++t) {
                        const int node = node0 + X::pack(t, g) * E;
                        Row in[E];
#pragma unroll
                        for (int j = 0; j < E; ++j) in[j] = value[(S.start + min(node + j, S.n - 1)) * A.v_stride + X::v_channel(dt, m)];
                        __builtin_memcpy(&to[t], in, 16);
                    }
                };
                if constexpr (EARLY) {
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) read_v(dt, v[dt]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                float z[NT][8];
                scores(k, z);
                uint32_t mask[NT];                               // of the lane's 8 tokens
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mask[nt] = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int node = node0 + X::key(j >> 2, 4 * g + (j & 3));
                        if (node < S.n && ((sees[nt] >> node) & 1)) mask[nt] |= 1u << j;
                        else z[nt][j] = -INFINITY;
                    }
                }
                mine.template weights<1>(z, p);
                bool finite = true;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    if constexpr (!EARLY) read_v(dt, v[dt]);
#pragma unroll
                    for (int t = 0; t < VT; ++t) {
                        v[dt][t] = X::first(v[dt][t], S.n - node0 - X::pack(t, g) * E);
                        finite = finite && X::finite(v[dt][t]);
                        v[dt][t] = only_finite<X>(v[dt][t]);
                    }
                    mine.add(dt, v[dt], p);
                }
                if (!__all(finite)) {
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        uint4 all[VT];
                        read_v(dt, all);
#pragma unroll
                        for (int t = 0; t < VT; ++t) all[t] = X::first(all[t], S.n - node0 - X::pack(t, g) * E);
                        mine.add_special(dt, all, mask);
                    }
                }
            }

            // the waves' sums together, DC channels at a time
            const int g = here(lane) >> 4, m = here(lane) & 15;
            __syncthreads();
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float all = add_xor32(add_xor16(mine.total[nt]));
                if (g == 0) {
                    s_top[wave][16 * nt + m] = mine.top(nt);
                    s_total[wave][16 * nt + m] = all;
                }
            }
            __syncthreads();
            const auto top_of = [&](int row) {
                float top = s_top[0][row];
#pragma unroll
                for (int w = 1; w < TA_WAVES; ++w) top = fmaxf(top, s_top[w][row]);
                return top;
            };
            const auto total_of = [&](int row, float shift) {
                float t = 0.f;
#pragma unroll
                for (int w = 0; w < TA_WAVES; ++w) t += s_total[w][row] * exp2_fast(s_top[w][row] - shift);
                return t;
            };
            float mine_by[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mine_by[nt] = exp2_fast(mine.top(nt) - finite_shift(top_of(16 * nt + m)));
            float *part = tree_part(A, blockIdx.x, first ? 0 : 1, DIM);
#pragma unroll
            for (int d0 = 0; d0 < DIM; d0 += DC) {
                if (d0 > 0) __syncthreads();
#pragma unroll
                for (int dt = 0; dt < DC / 16; ++dt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        f32x4_t o = mine.o[d0 / 16 + dt][nt];
                        int at = 16 * dt + 4 * g;
                        if constexpr (X::CODED) {                // two products have every other channel: halves of both
                            const f32x4_t a = mine.o[d0 / 16 + (dt & ~1)][nt], b = mine.o[d0 / 16 + (dt | 1)][nt];
                            o = dt & 1 ? f32x4_t{a[2], b[2], a[3], b[3]} : f32x4_t{a[0], b[0], a[1], b[1]};
                            at = 16 * (dt & ~1) + 8 * g + 4 * (dt & 1);
                        }
                        *reinterpret_cast<float4 *>(&s_sum[wave][16 * nt + m][at]) =
                            make_float4(o[0] * mine_by[nt], o[1] * mine_by[nt], o[2] * mine_by[nt], o[3] * mine_by[nt]);
                    }
                __syncthreads();
                for (int e = tid; e < ROWS * (DC / 4); e += TA_THREADS) {
                    const int row = e / (DC / 4), c = (e - row * (DC / 4)) * 4;
                    if (row0 + row >= rows) continue;
                    float4 a = *reinterpret_cast<const float4 *>(&s_sum[0][row][c]);
#pragma unroll
                    for (int w = 1; w < TA_WAVES; ++w) {
                        const float4 b = *reinterpret_cast<const float4 *>(&s_sum[w][row][c]);
                        a.x += b.x;
                        a.y += b.y;
                        a.z += b.z;
                        a.w += b.w;
                    }
                    if (whole) {
                        const float top = top_of(row), total = total_of(row, finite_shift(top));
                        const float by = total == 0.f ? 0.f : 1.f / total;
                        const int node = (row0 + row) / A.group, head = h * A.group + row0 + row - node * A.group;
                        const int64_t at = (int64_t)(S.start + node) * heads_q + head;
                        Row to[4];
                        from_f32(a.x * by, to);
                        from_f32(a.y * by, to + 1);
                        from_f32(a.z * by, to + 2);
                        from_f32(a.w * by, to + 3);
                        __builtin_memcpy(__builtin_assume_aligned(static_cast<Row *>(A.out) + at * DIM + d0 + c, sizeof(to)), to, sizeof(to));
                        if (d0 + c == 0 && A.lse != nullptr) A.lse[at] = total == 0.f ? -INFINITY : (top + log2f(total)) * LN2;
                    } else {
                        *reinterpret_cast<float4 *>(part + (size_t)row * DIM + d0 + c) = a;
                    }
                }
            }
            if (!whole && tid < min(ROWS, (int)A.part_rows)) {
                const float top = top_of(tid);
                part[(size_t)A.part_rows * DIM + 2 * tid] = top;
                part[(size_t)A.part_rows * DIM + 2 * tid + 1] = total_of(tid, finite_shift(top));
            }
            u += A.part_rows == 0 ? 1 : s1 - s0;
        }
    }
}

// The parts of a row and head, where there are more than one: a wave each (SHARED false), or a block each, whose eight waves take
// parts in turn (few rows with many parts).  Bound by latency, of the lengths and then of the parts, which other XCDs have written:
// 2.8 us at the least; 4.0 us for 256 rows and heads with 32 parts each; 5740 rows and heads of wide blocks, 34 MB, in 8.7 us.
template <bool SHARED>
constexpr int tj_waves() { return SHARED ? 8 : 4; }
template <typename W, int DIM, typename Cut, bool SHARED>
__global__ __launch_bounds__(64 * tj_waves<SHARED>()) void k_tree_join(TreeJoinArgs A)
{
    // a lane has four channels; where that leaves lanes over, groups of them take different parts
    constexpr int WAVES = tj_waves<SHARED>(), ROWS = Cut::ROWS, LANES = DIM / 4, GROUPS = 64 / LANES;
    constexpr int STEP = (SHARED ? WAVES : 1) * GROUPS, AHEAD = GROUPS == 1 ? 8 : 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), heads_q = A.heads * A.group;
    const int item = SHARED ? blockIdx.x : blockIdx.x * WAVES + wave, t = item / heads_q, hq = item - t * heads_q;
    if (t >= A.T) return;
    const int h = hq / A.group;

    TreeChunk<Cut> chunk;
    const int units = tree_units(A, lane, chunk);
    int base = 0;
    uint64_t found;
    while ((found = __ballot(t >= chunk.start && t < chunk.start + chunk.n)) == 0) {
        if (chunk.first + 64 >= A.R) return;                     // a row of no request
        base += chunk.all();
        chunk.load(A, lane, chunk.first + 64);
    }
    const int l = lane_of_first(found);
    const TreeSpan S = chunk.span(A, l);
    base += chunk.before(l);
    const int node = t - S.start;
    const int row = node * A.group + hq - h * A.group, in_part = row % ROWS, u0 = base + (h * S.row_tiles + row / ROWS) * S.steps;
    const int b0 = tree_block_of<Cut>(u0, units), b1 = tree_block_of<Cut>(u0 + S.steps - 1, units);
    if (b0 == b1) return;                                        // one block had the whole and has written it
    // a block's first segment is its part 0: that of b0 is if b0 begins with this task
    const int part0 = tree_begin<Cut>(b0, units) == u0 ? 0 : 1;

    float top = -INFINITY, total = 0.f;
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
    const int c = lane % LANES * 4;
    for (int b = b0 + (SHARED ? wave * GROUPS : 0) + lane / LANES; b <= b1; b += STEP * AHEAD) {
        float2 head[AHEAD];
        f32x4_t in[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int at = min(b + j * STEP, b1);
            const float *part = tree_part(A, at, at == b0 ? part0 : 0, DIM);
            head[j] = *reinterpret_cast<const float2 *>(part + (size_t)A.part_rows * DIM + 2 * in_part);
            in[j] = *reinterpret_cast<const f32x4_t *>(part + (size_t)in_part * DIM + c);
        }
        float next = top;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (b + j * STEP > b1) head[j] = make_float2(-INFINITY, 0.f);
            next = fmaxf(next, head[j].x);
        }
        const float shift = finite_shift(next), old = exp2_fast(top - shift);
        top = next;
        total *= old;
        sum *= old;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (b + j * STEP > b1) break;
            const float by = exp2_fast(head[j].x - shift);
            total += head[j].y * by;
            sum += in[j] * by;
        }
    }
    // the groups together: all lanes of the same channels end up with the same
    if constexpr (GROUPS > 1) {
        float all = top;
#pragma unroll
        for (int m = LANES; m < 64; m *= 2) all = fmaxf(all, __shfl_xor(all, m));
        const float by = exp2_fast(top - finite_shift(all));
        top = all;
        total *= by;
        sum *= by;
#pragma unroll
        for (int m = LANES; m < 64; m *= 2) {
            total += __shfl_xor(total, m);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], m);
        }
    }
    if constexpr (SHARED) {
        __shared__ float s_top[WAVES], s_total[WAVES];
        __shared__ __align__(16) float s_sum[WAVES][DIM];
        if (lane == 0) {
            s_top[wave] = top;
            s_total[wave] = total;
        }
        if (lane < LANES) *reinterpret_cast<f32x4_t *>(&s_sum[wave][c]) = sum;
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, s_top[w]);
        total = 0.f;
        sum = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float by = exp2_fast(s_top[w] - finite_shift(top));
            total += s_total[w] * by;
            sum += *reinterpret_cast<const f32x4_t *>(&s_sum[w][c]) * by;
        }
    }
    if (lane >= LANES) return;
    const int64_t at = (int64_t)t * heads_q + hq;
    const float by = total == 0.f ? 0.f : 1.f / total;
    using Row = typename RowOf<W>::type;
    Row to[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) from_f32(sum[i] * by, to + i);
    __builtin_memcpy(__builtin_assume_aligned(static_cast<Row *>(A.out) + at * DIM + c, sizeof(to)), to, sizeof(to));
    if (lane == 0 && A.lse != nullptr) A.lse[at] = total == 0.f ? -INFINITY : (top + log2f(total)) * LN2;
}

}  // namespace svdp
