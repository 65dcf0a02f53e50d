// Kernels around the attention of drafted tokens: block tables and slots from lengths, the answers' tokens and the
// accepted branch, K and V of accepted tokens into their pages.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svdp_device.h"

namespace svdp {

// ---- block tables and slots -----------------------------------------------------------------------------------------------

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_WAVES = PLAN_THREADS / 64;
constexpr int PLAN_EACH = 4;                // requests of a thread, at most
// LDS of a block: starts [R + 1], then lens, limit and first [R] (below)
inline size_t plan_lds(int R) { return ((size_t)4 * R + 1) * 4; }

// Pages are handed out by a prefix sum of the requests' needs, and so are places at the ring's end for pages that come
// back.  Every block forms the whole sums (R <= 4096 lengths, a few microseconds' worth of arithmetic at most) and then does
// its share of table rows and of slots, so that nothing waits for another block and nothing but the inputs is read: a new entry
// of the table is taken from the ring again by the rows that lie in it.  Blocks for table rows and blocks for slots follow each
// other in the grid.  What bounds it is the chain of loads (lengths, then the ring or the table), not bytes: 3.4 us for 8
// requests, 7.2 us for 700 requests and 93 289 rows (7.8 us where a block does rows and then slots, 8.7 us with blocks of 256
// threads, whose threads have three requests each).
__global__ __launch_bounds__(PLAN_THREADS) void k_kv_plan(
    int32_t *table, int max_pages, int32_t *ring, int pages, int page_bits, const int32_t *pool, const int32_t *lens,
    const int32_t *add, const int32_t *starts, const int32_t *keep, int R, int T, int row_blocks, int64_t *slots,
    int32_t *lens_out, int32_t *pool_out, int32_t *refused)
{
    extern __shared__ __align__(16) char plan_smem[];
    int *s_starts = reinterpret_cast<int *>(plan_smem);
    int *s_lens = s_starts + R + 1;
    int *s_limit = s_lens + R;          // tokens that get a slot: 0 for a refused request, -1 for one that ends
    int *s_first = s_limit + R;         // pages that the requests before it take, or give back
    __shared__ int s_wave[2][PLAN_WAVES];
    __shared__ int s_taken;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int page = 1 << page_bits;
    const int per = (R + PLAN_THREADS - 1) / PLAN_THREADS, r0 = tid * per, mine = min(per, R - r0);
    int raw[PLAN_EACH], more[PLAN_EACH];
#pragma unroll
    for (int j = 0; j < PLAN_EACH; ++j) {
        if (j >= per) break;
        raw[j] = lens[min(r0 + j, R - 1)];
        more[j] = add[min(r0 + j, R - 1)];
    }
    const int free_pages = min(max(pool[1], 0), pages);
    const int head = (int)(((uint32_t)max(pool[0], 0)) % (uint32_t)pages);
    // slots of the blocks behind those that do the table's rows, and what is kept of the first of them
    const int64_t slot_step = (int64_t)(gridDim.x - row_blocks) * PLAN_THREADS;
    int64_t t = ((int64_t)blockIdx.x - row_blocks) * PLAN_THREADS + tid;
    int kept = t >= 0 && t < T && keep != nullptr ? keep[t] : 0;
    if (tid == 0) s_taken = 0;
    for (int r = tid; r <= R; r += PLAN_THREADS) s_starts[r] = starts[r];

    // pages held, and pages needed, of a request; more pages than the table is wide: refused
    const auto pages_of = [&](int n) { return (n + page - 1) >> page_bits; };
    int len[PLAN_EACH], need[PLAN_EACH], need_sum = 0, give_sum = 0;
    bool wide[PLAN_EACH];
#pragma unroll
    for (int j = 0; j < PLAN_EACH; ++j)
        if (j < mine) {
            len[j] = min(max(raw[j], 0), max_pages << page_bits);
            const int before = pages_of(len[j]);
            const bool ends = more[j] < 0;
            wide[j] = !ends && (int64_t)len[j] + more[j] > (int64_t)max_pages << page_bits;
            need[j] = ends || wide[j] ? 0 : pages_of(len[j] + more[j]) - before;
            s_lens[r0 + j] = len[j];
            need_sum += need[j];
            give_sum += ends ? before : 0;
        }
    const int need_upto = wave_inclusive_scan(need_sum), give_upto = wave_inclusive_scan(give_sum);
    if (lane == 63) {
        s_wave[0][wave] = need_upto;
        s_wave[1][wave] = give_upto;
    }
    __syncthreads();
    int taken_before = need_upto - need_sum, given_before = give_upto - give_sum, given = 0;
#pragma unroll
    for (int w = 0; w < PLAN_WAVES; ++w) {
        taken_before += w < wave ? s_wave[0][w] : 0;
        given_before += w < wave ? s_wave[1][w] : 0;
        given += s_wave[1][w];
    }
    int taken = 0;
#pragma unroll
    for (int j = 0; j < PLAN_EACH; ++j)
        if (j < mine) {
            const int r = r0 + j;
            const bool ends = more[j] < 0, no = wide[j] || (need[j] > 0 && taken_before + need[j] > free_pages);
            s_first[r] = ends ? given_before : taken_before;
            s_limit[r] = ends ? -1 : no ? 0 : more[j];
            taken_before += need[j];
            given_before += ends ? pages_of(len[j]) : 0;
            if (need[j] > 0 && !no) taken = taken_before;   // sums only grow: the last granted one is the largest
            if (blockIdx.x == 0) {
                lens_out[r] = ends ? 0 : no ? raw[j] : len[j] + more[j];
                refused[r] = no ? 1 : 0;
            }
        }
    if (taken > 0) atomicMax(&s_taken, taken);
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
        pool_out[0] = (int)(((uint32_t)head + (uint32_t)s_taken) % (uint32_t)pages);
        pool_out[1] = min(free_pages - s_taken + given, pages);
    }

    // table rows, one wave each: new entries in, or the pages of a request that ends to the ring's end
    if ((int)blockIdx.x < row_blocks) {
        for (int r = blockIdx.x * PLAN_WAVES + wave; r < R; r += row_blocks * PLAN_WAVES) {
            const int limit = s_limit[r], before = pages_of(s_lens[r]), first = s_first[r];
            int32_t *row = table + (size_t)r * max_pages;
            if (limit < 0) {
                for (int i = lane; i < before; i += 64)
                    if (first + i < pages - free_pages)     // no more than there are places for
                        ring[((uint32_t)head + (uint32_t)free_pages + (uint32_t)(first + i)) % (uint32_t)pages] = row[i];
            } else {
                const int after = pages_of(s_lens[r] + limit);
                for (int i = before + lane; i < after; i += 64)
                    row[i] = ring[((uint32_t)head + (uint32_t)(first + i - before)) % (uint32_t)pages];
            }
        }
        return;
    }

    // slots
    for (; t < T; t += slot_step, kept = t < T && keep != nullptr ? keep[t] : 0) {
        int lo = 0, hi = R;                                 // the last request that starts at or before t
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (s_starts[mid] <= (int)t) lo = mid;
            else hi = mid - 1;
        }
        int64_t slot = -1;
        if (lo < R) {
            const int place = keep != nullptr ? kept : (int)t - s_starts[lo];
            if (place >= 0 && place < s_limit[lo]) {
                const int at = s_lens[lo] + place, i = at >> page_bits, before = pages_of(s_lens[lo]);
                const int id = i < before
                                   ? table[(size_t)lo * max_pages + i]
                                   : ring[((uint32_t)head + (uint32_t)(s_first[lo] + i - before)) % (uint32_t)pages];
                if (id >= 0 && id < pages) slot = ((int64_t)id << page_bits) + (at & (page - 1));
            }
        }
        slots[t] = slot;
    }
}

// ---- the answers' tokens and the accepted branch --------------------------------------------------------------------------

constexpr int BEST_THREADS = 256;

// A word that grows with the value: NaN above all, -0 equal to 0; and one that then falls with the index.
__device__ __forceinline__ uint32_t best_order(float v)
{
    const uint32_t u = __float_as_uint(v + 0.f);
    return (u & 0x7fffffffu) > 0x7f800000u ? 0xffffffffu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t best_key(float v, uint32_t index)
{
    return ((uint64_t)best_order(v) << 32) | (0xffffffffu - index);
}
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v)
{
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)v, m);
        v = o > v ? o : v;
    }
    return v;
}

// The largest logit of a row's vectors [begin, end), of those that a lane takes (at, at + step, ...).  Vectors are counted from the
// aligned address at or before the row, whatever its own alignment.  A lane keeps its best vector by the largest of its values, a few
// operations for a vector, and looks for the place in it once, at the end.
template <int AHEAD, typename W>
__device__ __forceinline__ uint64_t best_of(const W *row, int V, int begin, int end, int at, int step)
{
    constexpr int VEC = Elem<W>::VEC;
    const int skew = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / Elem<W>::BYTES);
    // vectors that lie in the row as a whole
    const int inner = max(begin, skew > 0 ? 1 : 0), outer = min(end, (V + skew) / VEC);
    uint4 kept = make_uint4(0, 0, 0, 0);
    uint32_t top = 0;                                       // order of the largest value, above 0 once there is one
    int place = 0;
    for (int i0 = inner + at; i0 < outer; i0 += AHEAD * step) {
        uint4 in[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) in[a] = load_raw(row + (min(i0 + a * step, outer - 1) * VEC - skew));
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            float v[VEC];
            widen(in[a], v, row);
            float m = v[0];
            bool nan = false;
#pragma unroll
            for (int j = 0; j < VEC; j += 2) {
                m = fmaxf(m, fmaxf(v[j], v[j + 1]));
                nan |= __builtin_isunordered(v[j], v[j + 1]);
            }
            const uint32_t o = nan ? 0xffffffffu : best_order(m);
            if (o > top) {
                top = o;
                place = min(i0 + a * step, outer - 1);
                kept = in[a];
            }
        }
    }
    uint64_t best = 0;
    if (top > 0) {
        float v[VEC];
        widen(kept, v, row);
#pragma unroll
        for (int j = VEC - 1; j >= 0; --j)
            if (best_order(v[j]) == top) best = best_key(v[j], place * VEC - skew + j);
    }
    // the row's ends: the first and the last vector of the row, where they reach over it
    const auto edge = [&](int i) {
        if (i < begin || i >= end || at >= VEC) return;
        const int e = i * VEC - skew + at;
        if (e < 0 || e >= V) return;
        const uint64_t key = best_key(to_f32(row[e]), e);
        best = key > best ? key : best;
    };
    if (skew > 0) edge(0);
    if ((V + skew) % VEC != 0) edge((V + skew) / VEC);
    return wave_max_u64(best);
}
template <typename W>
__device__ __forceinline__ int best_vectors(const W *row, int V)
{
    return (V + (int)((reinterpret_cast<uintptr_t>(row) & 15u) / Elem<W>::BYTES) + Elem<W>::VEC - 1) / Elem<W>::VEC;
}

// Part blockIdx.y of row blockIdx.x: `per` vectors.  Bound by reading: 439 MB of bf16 logits in 76 us, 5.8 TB/s (90.7 us, by
// arithmetic, with an order and an index for every element); 8 rows of 32 000 in 3.4 us, by the latency of one load and the launch.
template <typename W>
__global__ __launch_bounds__(BEST_THREADS) void k_logits_best(const W *logits, int64_t stride, int V, int per, uint64_t *parts)
{
    __shared__ uint64_t s_best[BEST_THREADS / 64];
    const W *row = logits + (int64_t)blockIdx.x * stride;
    const int begin = blockIdx.y * per, end = min(begin + per, best_vectors(row, V));
    uint64_t best = best_of<4>(row, V, begin, end, threadIdx.x, BEST_THREADS);
    if ((threadIdx.x & 63) == 0) s_best[threadIdx.x >> 6] = best;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < BEST_THREADS / 64; ++w) best = s_best[w] > best ? s_best[w] : best;
        parts[(size_t)blockIdx.x * gridDim.y + blockIdx.y] = best;
    }
}

struct TreeWalk {
    const int32_t *tokens;
    const uint64_t *tree;
    const int32_t *starts;
    int32_t *keep, *counts, *next, *best;
    int R, T, max_nodes;
};
// Down the tree of request r, n nodes from row a on, a lane each, by the whole wave; mine: the answer of the lane's node.
__device__ __forceinline__ void walk_down(const TreeWalk &A, int r, int a, int n, int lane, int token, uint64_t sees, int mine)
{
    const bool node = lane < n;
    const uint64_t up = sees & ((1ull << lane) - 1);
    const int parent = node && up != 0 ? 63 - __clzll((long long)up) : -1;
    int place = lane == 0 ? 0 : -1, count = n > 0 ? 1 : 0, at = 0;
    while (count > 0) {                                     // at grows with every step
        const int answered = __builtin_amdgcn_readlane(mine, at);
        const uint64_t agree = __ballot(node && lane > at && parent == at && token == answered);
        if (agree == 0) break;
        at = __ffsll((unsigned long long)agree) - 1;
        if (lane == at) place = count;
        ++count;
    }
    const int following = __builtin_amdgcn_readlane(mine, at);
    if (node) A.keep[a + lane] = place;
    if (lane == 0) {
        A.counts[r] = count;
        A.next[r] = count > 0 ? following : -1;
    }
}
__device__ __forceinline__ int best_index(uint64_t key) { return (int)(0xffffffffu - (uint32_t)key); }

// One wave a request: the rows' answers from their parts, then down the tree; the last block has the padding.  Bound by the latency
// of two loads after each other: 2.1 us for one tree of 8, 5.1 us for 32 trees and 10 parts a row.
__global__ __launch_bounds__(64) void k_tree_walk(const uint64_t *parts, int n_parts, TreeWalk A)
{
    const int r = blockIdx.x, lane = threadIdx.x;
    const auto answer = [&](int t) {
        constexpr int AHEAD = 16;
        uint64_t k = 0;
        for (int p = 0; p < n_parts; p += AHEAD) {
            uint64_t o[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) o[i] = parts[(size_t)t * n_parts + min(p + i, n_parts - 1)];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) k = o[i] > k ? o[i] : k;
        }
        return best_index(k);
    };
    const int a = min(max(A.starts[r], 0), A.T), b = r < A.R ? min(max(A.starts[r + 1], a), A.T) : A.T;
    const int n = r < A.R ? min(b - a, A.max_nodes) : 0;
    int mine = -1, token = -2;
    uint64_t sees = 0;
    if (lane < n) {
        sees = A.tree != nullptr ? A.tree[a + lane] : ~0ull;
        token = A.tokens[a + lane];
        mine = answer(a + lane);
        A.best[a + lane] = mine;
    }
    if (r < A.R) walk_down(A, r, a, n, lane, token, sees, mine);
    for (int t = a + n + lane; t < b; t += 64) {            // rows that are no node
        A.best[t] = answer(t);
        A.keep[t] = -1;
    }
}

// Both in one launch, where a request's logits are few: a block has all rows of a request, as many of its waves as there are for
// a row, and blocks R on have the padding, max_nodes rows each (T <= R max_nodes).  Bound by the latency of a block that reads by
// itself: 8 rows of 8000 in 6.1 us, where the two launches take 3.3 + 1.6 and the host 3 us more; 500 KB a block take 15 us.
constexpr int SMALL_THREADS = 1024, SMALL_WAVES = SMALL_THREADS / 64;
template <typename W>
__global__ __launch_bounds__(SMALL_THREADS) void k_tree_accept(const W *logits, int64_t stride, int V, TreeWalk A)
{
    __shared__ uint64_t s_best[64][SMALL_WAVES];
    const int r = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int first = min(max(A.starts[min(r, A.R)], 0), A.T), a = r < A.R ? first : min(first + (r - A.R) * A.max_nodes, A.T);
    const int b = r < A.R ? min(max(A.starts[r + 1], a), A.T) : min(a + A.max_nodes, A.T);
    const int n = r < A.R ? min(b - a, A.max_nodes) : 0;
    int token = -2;
    uint64_t sees = 0;
    if (wave == 0 && lane < n) {
        sees = A.tree != nullptr ? A.tree[a + lane] : ~0ull;
        token = A.tokens[a + lane];
    }
    bool nodes = true;                                      // the nodes first, then rows that are none
    for (int t0 = a, rows = n; nodes || rows > 0; t0 += rows, rows = min(b - t0, 64), nodes = false) {
        int share = SMALL_WAVES;                            // waves of a row: a power of two
        while (share > 1 && share * rows > SMALL_WAVES) share >>= 1;
        const int sub = wave & (share - 1);
        for (int i = wave / share; i < rows; i += SMALL_WAVES / share) {
            const W *row = logits + (int64_t)(t0 + i) * stride;
            const uint64_t best = best_of<8>(row, V, 0, best_vectors(row, V), sub * 64 + lane, share * 64);
            if (lane == 0) s_best[i][sub] = best;
        }
        __syncthreads();
        if (wave == 0) {
            uint64_t k = 0;
            if (lane < rows)
                for (int w = 0; w < share; ++w) k = s_best[lane][w] > k ? s_best[lane][w] : k;
            const int mine = lane < rows ? best_index(k) : -1;
            if (lane < rows) A.best[t0 + lane] = mine;
            if (nodes && r < A.R) walk_down(A, r, a, n, lane, token, sees, mine);
            else if (lane < rows) A.keep[t0 + lane] = -1;
        }
        __syncthreads();
    }
}

// ---- K and V into their pages ---------------------------------------------------------------------------------------------

constexpr int COMMIT_THREADS = 256;
constexpr int COMMIT_ROWS = 8;
constexpr int COMMIT_CHANNELS = 256;        // the least a block has of them, unless a row has fewer

// Rows [8 blockIdx.x, + 8) of layer blockIdx.y, channels [c0, + channels) of all heads side by side with c0 = (blockIdx.z / 2)
// channels; even blockIdx.z: K, odd: V.  K is copied in 16-byte vectors.  V lies with e tokens of a channel side by side: where e
// rows in a row fill such a pack (prompts), they are read together and written as whole packs, by the row of the pack's first
// token; other rows (branches of a tree) write their elements one by one.  A lane has two channels of V, so that the packs of a
// wave lie side by side.  Bound by reading and writing: a prompt's 618 MB (half read, half written) in 112 us, 5.5 TB/s (144 us
// with eight channels a lane, packs 128 bytes apart); a branch of a tree of 8, in 32 layers, in 4.0 us, by latency, with its
// channels over many blocks (five rows of a branch 6.6 us, with one block for all channels 14.0); branches of 723 rows in 12 layers, 8.8 MB,
// in 6.4 us.
template <typename W>
__global__ __launch_bounds__(COMMIT_THREADS) void k_kv_commit(W *K, W *V, const W *k, int64_t k_layer, int64_t k_row,
                                                              const W *v, int64_t v_layer, int64_t v_row,
                                                              const int64_t *slots, int T, int pages, int page_bits, int heads,
                                                              int dim_bits, int channels)
{
    constexpr int E = Elem<W>::VEC, AHEAD = 4;
    __shared__ int64_t s_near[COMMIT_ROWS + 2 * E];         // slots from row t0 - E on
    __shared__ int s_rows[COMMIT_ROWS];                     // V: from the front those that write whole packs, from the back one token; K: all
    __shared__ int s_count[2];
    const int tid = threadIdx.x, t0 = blockIdx.x * COMMIT_ROWS, layer = blockIdx.y;
    const int64_t all = (int64_t)pages << page_bits;
    if (tid < COMMIT_ROWS + 2 * E) {
        const int t = t0 - E + tid;
        const int64_t s = t >= 0 && t < T ? slots[t] : -1;
        s_near[tid] = s < all ? s : -1;
    }
    __syncthreads();
    const int page = 1 << page_bits, c0 = (int)(blockIdx.z >> 1) * channels, cn = min(channels, (heads << dim_bits) - c0);
    k += (int64_t)layer * k_layer + (int64_t)t0 * k_row + c0;
    v += (int64_t)layer * v_layer + (int64_t)t0 * v_row + c0;
    const int64_t layer_at = (int64_t)layer * pages * heads;
    // element of the cache at which channel c of a slot's head begins its page
    const auto page_at = [&](int64_t slot, int c) {
        return (((layer_at + (slot >> page_bits) * heads + (c >> dim_bits)) << page_bits) << dim_bits);
    };
    const int mask = (1 << dim_bits) - 1;
    const bool of_v = blockIdx.z & 1;
    if (tid < 64) {
        bool real = false, whole = false, first = false;
        if (tid < COMMIT_ROWS) {
            const int64_t s = s_near[E + tid];
            const int j = (int)(s & (E - 1));
            real = whole = s >= 0;
            first = j == 0;
#pragma unroll
            for (int i = 0; i < E; ++i) whole &= s_near[E + tid - j + i] == s - j + i;
        }
        const bool in_front = real && (!of_v || (whole && first)), behind = real && of_v && !whole;
        const uint64_t front = __ballot(in_front), back = __ballot(behind), before = (1ull << tid) - 1;
        if (in_front) s_rows[__popcll(front & before)] = tid;
        if (behind) s_rows[COMMIT_ROWS - 1 - __popcll(back & before)] = tid;
        if (tid == 0) {
            s_count[0] = __popcll(front);
            s_count[1] = __popcll(back);
        }
    }
    __syncthreads();
    if (!of_v) {
        const int vectors = cn / E, items = s_count[0] * vectors;
        for (int i0 = tid; i0 < items; i0 += AHEAD * COMMIT_THREADS) {
            uint4 in[AHEAD];
            W *to[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {                // no branch around a load: they are on their way together
                const int i = min(i0 + a * COMMIT_THREADS, items - 1), job = i / vectors, c = (i - job * vectors) * E, row = s_rows[job];
                const int64_t slot = s_near[E + row];
                in[a] = load_raw(k + (int64_t)row * k_row + c);
                to[a] = K + page_at(slot, c0 + c) + (((slot & (page - 1)) << dim_bits) + ((c0 + c) & mask));
            }
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                if (i0 + a * COMMIT_THREADS >= items) break;
                *reinterpret_cast<uint4 *>(to[a]) = in[a];
            }
        }
        return;
    }
    const int pairs = cn / 2, whole_items = s_count[0] * pairs, one_items = s_count[1] * pairs;
    const auto place_of = [&](int64_t slot, int c) {             // where V's pack of a slot and channel lies
        return V + page_at(slot, c0 + c) + ((((slot & (page - 1)) / E << dim_bits) + ((c0 + c) & mask)) * E);
    };
    for (int i = tid; i < whole_items; i += COMMIT_THREADS) {
        const int job = i / pairs, c = (i - job * pairs) * 2, row = s_rows[job];
        const W *from = v + (int64_t)row * v_row + c;
        W in[E][2], out[2][E];
#pragma unroll
        for (int j = 0; j < E; ++j) __builtin_memcpy(in[j], __builtin_assume_aligned(from + j * v_row, sizeof(in[j])), sizeof(in[j]));
#pragma unroll
        for (int j = 0; j < E; ++j) {
            out[0][j] = in[j][0];
            out[1][j] = in[j][1];
        }
        __builtin_memcpy(__builtin_assume_aligned(place_of(s_near[E + row], c), 16), out, sizeof(out));
    }
    for (int i0 = tid; i0 < one_items; i0 += AHEAD * COMMIT_THREADS) {
        W in[AHEAD][2], *to[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int i = min(i0 + a * COMMIT_THREADS, one_items - 1), job = i / pairs, c = (i - job * pairs) * 2, row = s_rows[COMMIT_ROWS - 1 - job];
            const int64_t slot = s_near[E + row];
            __builtin_memcpy(in[a], __builtin_assume_aligned(v + (int64_t)row * v_row + c, sizeof(in[a])), sizeof(in[a]));
            to[a] = place_of(slot, c) + (slot & (E - 1));
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (i0 + a * COMMIT_THREADS >= one_items) break;
            to[a][0] = in[a][0];
            to[a][E] = in[a][1];
        }
    }
}

}  // namespace svdp
