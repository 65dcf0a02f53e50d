// Attention of drafted tokens where a request has many rows (svdp_tree_attn.h holds the division of the work and the join).
//
// The waves of a block take different rows of the SAME tokens, 32 each: K and V come from memory once for 256 rows.
// Their tiles pass through LDS, in two stages of 64 KB that are filled straight from memory, one while the other is worked on, with
// one barrier a stage; each wave keeps its own rows' shift, denominator and sum, and nothing is exchanged between waves.
// Products are 32 x 32 x 16: S^T = K Q^T leaves a lane with 16 scores of one row (token of result register i in lane half f:
// 16 (i / 8) + 8 f + i % 8, by the choice of K rows), which are the tokens that O^T += V^T P^T wants of that lane.
// LDS: K rows of DIM channels, 16-byte chunk c of token i at slot c ^ swizzle(i), so that the tokens of an operand read lie in different
// banks; V as in memory, of which 32 lanes read consecutive 512 bytes.
// What bounds it: a tile of 32 tokens is 768 cycles of a SIMD's matrix unit for each of its two waves (the weights' two terms have a
// product with V each) and about as many of its vector unit (16 exponentials, two terms, some 110 other instructions).  A wave's products and
// its weights follow each other, so that the two waves of a SIMD run side by side only in part: by the counters the matrix unit is
// busy 46 % of the time and the vector unit 48; the reads of LDS take 15 %, without bank conflicts (in 16 bits; 8 bits below).  Trees of 64 with seven query heads
// a head over 27 000 to 32 768 tokens, 88 GFLOP without the second terms: 163 us (with weights of one term 127: 39 % and 41 %).  What a
// stage costs besides (its barrier, addresses, the first read of K) is why a stage is as large as LDS allows, and some 14 us are
// not stages: 2 for the lengths, 3 for the first pages, Q and K and V, and a part of 133 KB that every block writes and that leaves the
// caches at the end.  A call of one stage of 64 rows takes 12 us.
#pragma once

#include "svdp_tree_attn.h"

namespace svdp {

constexpr int TW_THREADS = 512, TW_WAVES = TW_THREADS / 64, TW_ROWS = 32 * TW_WAVES;
constexpr int TW_STAGE = 64 << 10, TW_LDS = 2 * TW_STAGE;
template <int DIM>
constexpr int tw_tiles() { return TW_STAGE / 2 / (TA_TILE * DIM * 2); }          // of a stage: 8 or 4
template <int DIM>
using WideCut = TreeCut<TW_ROWS, tw_tiles<DIM>(), 8, true>;
typedef float f32x16_t __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16_t mfma_32(const uint4 &a, const uint4 &b, const f32x16_t &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(ta_bf16x8, a), __builtin_bit_cast(ta_bf16x8, b), c, 0, 0, 0);
}

// Token (of 32) that row `at` of K's operand stands for, and what its chunks are moved by.
__device__ __forceinline__ int tw_token(int at) { return (at >> 4) * 16 + ((at >> 2) & 1) * 8 + ((at >> 3) & 1) * 4 + (at & 3); }
__device__ __forceinline__ int tw_swizzle(int token, int dim) { return dim == 64 ? token & 7 : token & 15; }

// A cache in 8 bits: its tiles come into LDS as they are, in two stages of 32 KB, and the block makes bf16 operands of one of them
// (K and V with their tokens' powers of two, exact) in the 64 KB that the products read, between two barriers.  The tree's own tokens,
// bf16 as ever, come straight to those 64 KB.  Made by each wave in registers, the operands would cost every wave what the block does once.
// Trees of 64 over 20 000 to 32 768 tokens, seven query heads a head: 163 to 179 us in a profile and a call 149 to 157, where the rows' tiles one
// after the other, 32 at a time, take 205; the matrix unit is busy 37 % of the time, the vector unit 51.  Of the cycles of LDS 17 % are bank
// conflicts: the operands are written in pieces of 16 bytes that lie 32 bytes apart from lane to lane.
constexpr int TW_CODED = TW_STAGE / 2, TW_SCALES = 1024;        // bytes of a stage: codes; scales of K and of V, and what a load fills besides

template <typename W, int DIM>
__global__ __launch_bounds__(TW_THREADS) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_tree_attn_wide(TreeAttnArgs A)
{
    using X = TreeTile<bf16, DIM>;
    constexpr bool CODED = sizeof(W) == 1;
    constexpr int TILES = tw_tiles<DIM>(), KC = DIM / 16, DT = DIM / 32, CHUNKS = DIM / 8;
    using Cut = WideCut<DIM>;
    constexpr int TILE_BYTES = TA_TILE * DIM * 2, V_AT = TW_STAGE / 2;
    static_assert(TILES * TA_TILE >= 64, "the tree's tokens are one stage");
    // a stage of the tree's tokens: K where it always is; V as it comes, then in packs (finite elements), and as it is in packs
    constexpr int OWN_RAW = V_AT, OWN_PACKS = V_AT + TW_STAGE / 4, OWN_ALL = TW_STAGE / 4;
    extern __shared__ __align__(16) char tw_smem[];
    __shared__ __align__(16) uint8_t s_scales[CODED ? 2 : 1][CODED ? TW_SCALES : 16];     // of a stage's tokens: K's, behind them V's
    __shared__ uint64_t s_sees[TW_WAVES * 32];                   // what a row sees of its tree
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), f = lane >> 5, m = lane & 31;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void_t *)tw_smem;
    const uint32_t scales0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t *)&s_scales[0][0]);

    TreeChunk<Cut> chunk;
    const int units = tree_units(A, lane, chunk);
    int u = tree_begin<Cut>(blockIdx.x, units);
    const int u1 = tree_begin<Cut>(blockIdx.x + 1, units);
    if (u >= u1) return;
    int rem, l = tree_request(A, u, lane, chunk, &rem);

    // where a lane's operands lie in a tile (chunk c of K: ^ 32 c)
    const int k_at = tw_token(m) * CHUNKS * 16 + ((f ^ tw_swizzle(tw_token(m), DIM)) * 16);
    const int v_at = (f * DIM + m) * 16;
    // what a wave brings of a stage, 1 KB eight times: 128 channels: K or V of a tile; 64 channels: K and V of a tile
    const int fill_tile = DIM == 128 ? wave >> 1 : wave;
    const int fill_k = (lane / CHUNKS) * CHUNKS * 16 + (((lane % CHUNKS) ^ tw_swizzle(lane / CHUNKS, DIM)) * 16);

    for (bool first = true; u < u1; ++l, rem = 0) {
        if (l == 64) {
            chunk.load(A, lane, chunk.first + 64);
            l = 0;
        }
        const TreeSpan S = chunk.span(A, l);
        if (S.units == 0) continue;
        const int r = chunk.first + l;
        const int cached_steps = (S.tiles + TILES - 1) / TILES, per_page = A.page_bits - 5;
        int task = rem / S.cuts, s0 = rem - task * S.cuts;
        for (; task < A.heads * S.row_tiles && u < u1; ++task, s0 = 0, first = false) {
            const int s1 = A.part_rows == 0 ? S.steps : min(S.steps, s0 + u1 - u), s_end = min(s1, cached_steps);
            const int h = task / S.row_tiles, rows = S.n * A.group, block_row0 = (task - h * S.row_tiles) * TW_ROWS;
            const int row0 = block_row0 + wave * 32;
            const bool whole = s0 == 0 && s1 == S.steps, active = row0 < rows;

            // Page ids: a lane each for 64 pages, read out per tile.  (Read one by one through the scalar cache, the wait for
            // them also holds up the reads from LDS.)
            int window = -64, window_ids = 0;
            bool window_whole = true;                            // no page of it is missing
            const auto request_pages = [&](int step) {
                window = (max(step - 1, s0) * TILES) >> per_page;                // the stage that is worked on as well
                return A.table[(size_t)r * A.max_pages + max(min(window + (tid & 63), (S.tiles - 1) >> per_page), 0)];
            };
            const auto see_pages = [&](int step) {
                if (min((step * TILES + TILES - 1) >> per_page, (S.tiles - 1) >> per_page) >= window + 64) {
                    window_ids = here(request_pages(step));
                    window_whole = __all((uint32_t)window_ids < (uint32_t)A.pages);
                }
            };
            const auto page_of = [&](int tile) {
                return __builtin_amdgcn_readlane(window_ids, (min(tile, S.tiles - 1) >> per_page) - window);
            };
            // codes of a stage: rows of K as they lie, packs of V as they lie; a wave brings 2 KB of each, and one of them the scales
            const auto fill_coded = [&](int step, int stage) {
                see_pages(step);
                const int lane = here(tid) & 63, which = stage == 0 ? 0 : 1;
                const uint32_t to = lds0 + TW_STAGE + which * TW_CODED;
                const auto token_at = [&](int tile, int id) {        // the first one of a tile
                    const int64_t page = (int64_t)((uint32_t)id < (uint32_t)A.pages ? id : 0) * A.heads + h;
                    return ((page << per_page) + (tile & ((1 << per_page) - 1))) * TA_TILE;
                };
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int piece = (wave * 2 + i) * 64, per = TA_TILE * DIM / 16;           // pieces of 16 bytes; of a tile
                    const int tile = min(step * TILES + piece / per, S.tiles - 1);
                    const int64_t at = token_at(tile, page_of(tile)) * DIM + (piece % per + lane) * 16;
                    load_to_lds(static_cast<const char *>(A.K) + at, to + piece * 16);
                    load_to_lds(static_cast<const char *>(A.V) + at, to + TW_CODED / 2 + piece * 16);
                }
                // 32 scales of a tile are two times 16 bytes: wave 0 brings all K's, behind them V's (lanes past them the last ones again)
                if (wave == 0) {
                    const int piece = min(lane, 4 * TILES - 1), of_v = piece >= 2 * TILES, tile = min(step * TILES + (piece >> 1) % TILES, S.tiles - 1);
                    load_to_lds((of_v ? A.V_scale : A.K_scale) + token_at(tile, __shfl(window_ids, (tile >> per_page) - window)) + (piece & 1) * 16,
                                scales0 + which * TW_SCALES);
                }
            };
            const auto fill = [&](int step, int stage) {
                if constexpr (CODED) {
                    fill_coded(step, stage);
                    return;
                }
                see_pages(step);
                const int tile = min(step * TILES + fill_tile, S.tiles - 1), id = page_of(tile);
                const int64_t page = (int64_t)((uint32_t)id < (uint32_t)A.pages ? id : 0) * A.heads + h;
                const int64_t at = ((page << per_page) + (tile & ((1 << per_page) - 1))) * TILE_BYTES;
                const uint32_t to = lds0 + stage + fill_tile * TILE_BYTES;
                if constexpr (DIM == 128) {
                    const char *from = static_cast<const char *>(wave & 1 ? A.V : A.K) + at;
                    const int off = wave & 1 ? lane * 16 : fill_k, turn = wave & 1 ? 0 : 64;     // rows of 16 chunks: four of them in 1 KB
#pragma unroll
                    for (int i = 0; i < 8; ++i) load_to_lds(from + i * 1024 + (off ^ ((i & 3) * turn)), to + (wave & 1 ? V_AT : 0) + i * 1024);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        load_to_lds(static_cast<const char *>(A.K) + at + i * 1024 + fill_k, to + i * 1024);
                        load_to_lds(static_cast<const char *>(A.V) + at + i * 1024 + lane * 16, to + V_AT + i * 1024);
                    }
                }
            };
            // the tree's own tokens: rows of K and of V as they are (those past the last one repeat it)
            const auto fill_own = [&](int stage) {
                const int lane = here(tid) & 63;
                for (int p0 = wave * 64; p0 < (S.n + TA_TILE - 1) / TA_TILE * TA_TILE * CHUNKS; p0 += TW_THREADS) {
                    const int p = p0 + lane, token = p / CHUNKS, slot = p % CHUNKS;
                    const int64_t row = S.start + min(token, S.n - 1);
                    const int piece = (slot ^ tw_swizzle(token, DIM)) * 8;
                    load_to_lds(static_cast<const bf16 *>(A.k) + row * A.k_stride + h * DIM + piece, lds0 + stage + p0 * 16);
                    load_to_lds(static_cast<const bf16 *>(A.v) + row * A.v_stride + h * DIM + slot * 8, lds0 + stage + OWN_RAW + p0 * 16);
                }
            };

            // The first pages' ids, then Q and what the rows see of their tree, then the first stage, each requested before the one in
            // front of it is waited for.
            const TreeScale scale(A.scale, X::SIGNS);
            uint4 q[KC], k[KC], v[DT][2];
            uint64_t sees;
            stage_barrier<0>();                                  // the last segment's stages and stores are done with
            window_ids = request_pages(s0);                      // a segment of the tree's own tokens only: not looked at
            {
                const int row = min(row0 + (here(lane) & 31), rows - 1), node = row / A.group, head = h * A.group + row - node * A.group;
                const bf16 *from = static_cast<const bf16 *>(A.q) + (S.start + node) * A.q_stride + (int64_t)head * DIM + f * 8;
                sees = A.tree != nullptr ? A.tree[S.start + node] : ~0ull >> (63 - node);
#pragma unroll
                for (int c = 0; c < KC; ++c) q[c] = load_raw(from + c * 16);
            }
            // codes of a stage into operands, where a stage of 16 bits would have been filled
            const auto widen_stage = [&](int stage) {
                const int which = stage == 0 ? 0 : 1;
                const char *from = tw_smem + TW_STAGE + which * TW_CODED;
                for (int p = here(tid); p < TILES * TA_TILE * DIM / 16; p += TW_THREADS) {
                    constexpr int PER = DIM / 16;                // pieces of 16 channels of a token
                    const int token = p / PER, piece = p % PER, in_tile = token & (TA_TILE - 1);
                    const uint4 raw = *reinterpret_cast<const uint4 *>(from + p * 16);
                    const float by = power_of(s_scales[which][token]);
                    char *to = tw_smem + token * DIM * 2;
                    *reinterpret_cast<uint4 *>(to + (((2 * piece) ^ tw_swizzle(in_tile, DIM)) * 16)) = widen_e4m3(raw.x, raw.y, by);
                    *reinterpret_cast<uint4 *>(to + (((2 * piece + 1) ^ tw_swizzle(in_tile, DIM)) * 16)) = widen_e4m3(raw.z, raw.w, by);
                }
                for (int p = here(tid); p < TILES * TA_TILE * DIM / 16; p += TW_THREADS) {
                    const int pack = p / (DIM / 2);              // two channels of eight tokens
                    const uint4 raw = *reinterpret_cast<const uint4 *>(from + TW_CODED / 2 + p * 16);
                    const uint64_t scales = *reinterpret_cast<const uint64_t *>(&s_scales[which][TILES * TA_TILE + pack * 8]);
                    *reinterpret_cast<uint4 *>(tw_smem + V_AT + p * 32) = TreeTile<e4m3, DIM>::decoded(raw.x, raw.y, scales);
                    *reinterpret_cast<uint4 *>(tw_smem + V_AT + p * 32 + 16) = TreeTile<e4m3, DIM>::decoded(raw.z, raw.w, scales);
                }
            };
            int stage = 0;
            if (s0 < s_end) {
                window_ids = here(window_ids);
                window_whole = __all((uint32_t)window_ids < (uint32_t)A.pages);
                fill(s0, 0);
            } else {
                fill_own(0);
            }
            if (f == 0) s_sees[wave * 32 + m] = sees;
#pragma unroll
            for (int c = 0; c < KC; ++c) q[c] = scale.of(q[c]);
            // as in TreeWave: sum, shift, denominator (the lane half's part), and what a score has to exceed for the shift to move
            f32x16_t o[DT];
            float shift = 0.f, total = 0.f, limit = -INFINITY;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;

            for (int step = s0; step < s1; ++step, stage ^= TW_STAGE) {
                const bool own_tokens = step >= cached_steps;    // the tree's
                stage_barrier<0>();
                const bool full = !own_tokens && window_whole && (step + 1) * TILES * TA_TILE <= S.len;
                uint64_t counts = 0;                             // where it is not full: tokens of each tile, eight bits each
                bool finite = true;
                if (!full) {
                    for (int j = 0; j < TILES; ++j) {
                        const int tile = step * TILES + j;
                        const int count = own_tokens ? S.n - j * TA_TILE : (uint32_t)page_of(tile) < (uint32_t)A.pages ? S.len - tile * TA_TILE : 0;
                        counts |= (uint64_t)min(max(count, 0), TA_TILE) << (8 * j);
                    }
                }
                const auto count_of = [&](int j) { return (int)(counts >> (8 * j)) & 0xff; };
                if constexpr (CODED) {
                    if (!own_tokens) {
                        widen_stage(stage);
                        if (step + 1 < s_end) fill(step + 1, stage ^ TW_STAGE);
                        lds_barrier();
                    } else if (step > s0) {                      // the operands' memory is free only now
                        fill_own(0);
                        stage_barrier<0>();
                    }
                } else {
                    if (step + 1 < s_end) fill(step + 1, stage ^ TW_STAGE);
                    else if (step + 1 < s1) fill_own(stage ^ TW_STAGE);
                }
                char *const lds = tw_smem + (CODED ? 0 : stage);
                const int n_tiles = own_tokens ? (S.n + TA_TILE - 1) / TA_TILE : min(TILES, S.tiles - step * TILES);
                if (own_tokens) {                                // V into packs
                    int odd = 0;
                    for (int e = here(tid); e < n_tiles * 4 * DIM; e += TW_THREADS) {
                        const int pack = e / DIM, c = e - pack * DIM;
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            uint32_t x = *reinterpret_cast<const uint16_t *>(lds + OWN_RAW + ((pack * 8 + i) * DIM + c) * 2);
                            x = pack * 8 + i < S.n ? x : 0u;
                            w[i >> 1] = i & 1 ? w[i >> 1] | x << 16 : x;
                        }
                        const uint4 all = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4 *>(lds + OWN_PACKS + e * 16) = only_finite<X>(all);
                        *reinterpret_cast<uint4 *>(lds + OWN_ALL + e * 16) = all;
                        odd |= X::finite(all) ? 0 : 1;
                    }
                    finite = __syncthreads_or(odd) == 0;
                } else if (!full) {                              // what lies behind the tokens in V must not be NaN
                    for (int j = 0; j < n_tiles; ++j) {
                        if (count_of(j) == TA_TILE) continue;
                        for (int e = here(tid); e < TILE_BYTES / 16; e += TW_THREADS) {
                            uint4 *at = reinterpret_cast<uint4 *>(lds + V_AT + j * TILE_BYTES) + e;
                            *at = X::first(*at, count_of(j) - e / DIM * 8);
                        }
                    }
                    __syncthreads();
                }
                if (!active) continue;

                // which of the lane's 16 tokens its row sees
                const auto mask_of = [&](int j) {
                    const int f = here(lane) >> 5, m = here(lane) & 31;
                    uint32_t seen = (uint32_t)((1ull << count_of(j)) - 1);
                    if (own_tokens) seen &= (uint32_t)(s_sees[wave * 32 + m] >> (j * TA_TILE));
                    return ((seen >> (8 * f)) & 0xffu) | ((seen >> (16 + 8 * f)) & 0xffu) << 8;
                };
                // A tile's operands are read ahead of their use by hand, V's while the weights are formed and the next tile's K
                // in front of the second product: left alone, the compiler reads each just before its products, and the
                // wave stands for the whole way to LDS every time.
                const char *v_from = lds + (own_tokens ? OWN_PACKS : V_AT) + v_at, *k_from[KC];
#pragma unroll
                for (int c = 0; c < KC; ++c) k_from[c] = lds + (k_at ^ (c * 32));
                const auto read_k = [&](int j) {
#pragma unroll
                    for (int c = 0; c < KC; ++c) k[c] = *reinterpret_cast<const uint4 *>(k_from[c] + j * TILE_BYTES);
                };
                read_k(0);
#pragma unroll
                for (int j = 0; j < TILES; ++j) {
                    if (j >= n_tiles) break;
                    f32x16_t s;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
                    for (int c = 0; c < KC; ++c) s = mfma_32(k[c], q[c], s);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int t = 0; t < 2; ++t) v[dt][t] = *reinterpret_cast<const uint4 *>(v_from + j * TILE_BYTES + (2 * t * DIM + dt * 32) * 16);
                    if (j + 1 < TILES) read_k(j + 1);
                    __builtin_amdgcn_sched_barrier(0);
                    float z[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[i] = fmaf(s[i], scale.unit, -shift);
                    if (!full) {
                        const uint32_t mask = mask_of(j);
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (!((mask >> i) & 1)) z[i] = -INFINITY;
                    }
                    float top = z[0];
#pragma unroll
                    for (int i = 1; i < 16; ++i) top = fmaxf(top, z[i]);
                    top = max_xor32(top);
                    if (__any(top > limit)) {
                        const float to = top > limit ? shift + top : shift;
                        const float down = to - shift, old = limit == -INFINITY ? 0.f : exp2_fast(-down);
                        shift = to;
                        limit = top > limit ? SLACK : limit;
                        total *= old;
#pragma unroll
                        for (int i = 0; i < 16; ++i) z[i] -= down;
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) o[dt] *= old;
                    }
                    float sum = 0.f;
                    typename X::Weights p[2];
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        float e[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) e[i] = exp2_fast(z[8 * t + i]);
                        sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
                        p[t] = X::pack_weights(e);
                    }
                    total += sum;
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) o[dt] = mfma_32(v[dt][t], p[t].hi, o[dt]);
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) o[dt] = mfma_32(v[dt][t], p[t].lo, o[dt]);
                }
                if (finite) continue;
                // infinities and NaN that a row sees (see TreeWave::add_special)
#pragma unroll 1
                for (int j = 0; j < n_tiles; ++j) {
                    const uint32_t mask = mask_of(j);
                    const char *from = lds + OWN_ALL + j * TILE_BYTES + v_at;
#pragma unroll 1
                    for (int kind = 0; kind < 3; ++kind)
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) {
                            f32x16_t count;
#pragma unroll
                            for (int i = 0; i < 16; ++i) count[i] = 0.f;
#pragma unroll
                            for (int t = 0; t < 2; ++t) {
                                float seen[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) seen[i] = (mask >> (8 * t + i)) & 1 ? 1.f : 0.f;
                                const uint4 all = *reinterpret_cast<const uint4 *>(from + (2 * t * DIM + dt * 32) * 16);
                                count = mfma_32(ones_of_kind<X>(all, kind), X::pack_weights(seen).hi, count);
                            }
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[dt][i] += count[i] > 0.f ? value_of_kind(kind) : 0.f;
                        }
                }
            }

            // result register i of a lane: channel 32 dt + 8 (i / 4) + 4 f + i % 4 of row m
            if (active) {
                const int f = here(lane) >> 5, row = row0 + (here(lane) & 31);
                const float all = add_xor32(total), up = limit == -INFINITY ? -INFINITY : shift;
                if (row < rows) {
                    if (whole) {
                        const float by = all == 0.f ? 0.f : 1.f / all;
                        const int node = row / A.group, head = h * A.group + row - node * A.group;
                        const int64_t at = (int64_t)(S.start + node) * A.heads * A.group + head;
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                            for (int b = 0; b < 4; ++b) {
                                bf16 to[4];
#pragma unroll
                                for (int c = 0; c < 4; ++c) from_f32(o[dt][4 * b + c] * by, to + c);
                                __builtin_memcpy(__builtin_assume_aligned(static_cast<bf16 *>(A.out) + at * DIM + dt * 32 + 8 * b + 4 * f, 8), to, 8);
                            }
                        if (f == 0 && A.lse != nullptr) A.lse[at] = all == 0.f ? -INFINITY : (up + log2f(all)) * LN2;
                    } else {
                        float *part = tree_part(A, blockIdx.x, first ? 0 : 1, DIM);
                        const int at = row - block_row0;
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                            for (int b = 0; b < 4; ++b)
                                *reinterpret_cast<float4 *>(part + (size_t)at * DIM + dt * 32 + 8 * b + 4 * f) =
                                    make_float4(o[dt][4 * b], o[dt][4 * b + 1], o[dt][4 * b + 2], o[dt][4 * b + 3]);
                        if (f == 0) *reinterpret_cast<float2 *>(part + (size_t)A.part_rows * DIM + 2 * at) = make_float2(up, all);
                    }
                }
            }
            u += A.part_rows == 0 ? 1 : s1 - s0;
        }
    }
}

}  // namespace svdp
