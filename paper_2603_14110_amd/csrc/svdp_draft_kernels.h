// Kernels around the attention of drafted tokens: block tables and slots from lengths, the answers' tokens and the
// accepted branch, K and V of accepted tokens into their pages.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svdp_device.h"

namespace svdp {

// ---- block tables and slots -----------------------------------------------------------------------------------------------

constexpr int PLAN_THREADS = 256;
constexpr int PLAN_WAVES = PLAN_THREADS / 64;
// LDS of a block: starts [R + 1], then lens, limit and first [R] (below)
inline size_t plan_lds(int R) { return ((size_t)4 * R + 1) * 4; }

// Pages are handed out by a prefix sum of the requests' needs, and so are places at the ring's end for pages that come
// back.  Every block forms the whole sums (R <= 4096 lengths, a few microseconds' worth of arithmetic at most) and then does
// its share of table rows and of slots, so that nothing waits for another block and nothing but the inputs is read: a new entry
// of the table is taken from the ring again by the rows that lie in it.
__global__ __launch_bounds__(PLAN_THREADS) void k_kv_plan(
    int32_t *table, int max_pages, int32_t *ring, int pages, int page_bits, const int32_t *pool, const int32_t *lens,
    const int32_t *add, const int32_t *starts, const int32_t *keep, int R, int T, int64_t *slots, int32_t *lens_out,
    int32_t *pool_out, int32_t *refused)
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
    const int free_pages = min(max(pool[1], 0), pages);
    const int head = (int)(((uint32_t)max(pool[0], 0)) % (uint32_t)pages);
    if (tid == 0) s_taken = 0;
    for (int r = tid; r <= R; r += PLAN_THREADS) s_starts[r] = starts[r];

    // pages held, and pages needed, of request r; more pages than the table is wide: refused (need 0)
    const auto pages_of = [&](int n) { return (n + page - 1) >> page_bits; };
    const int per = (R + PLAN_THREADS - 1) / PLAN_THREADS, r0 = min(tid * per, R), r1 = min(r0 + per, R);
    int need_sum = 0, give_sum = 0;
    for (int r = r0; r < r1; ++r) {
        const int len = min(max(lens[r], 0), max_pages << page_bits), a = add[r];
        const int before = pages_of(len);
        const bool ends = a < 0, wide = (int64_t)len + a > (int64_t)max_pages << page_bits;
        const int need = ends || wide ? 0 : pages_of(len + a) - before;
        s_lens[r] = len;
        s_limit[r] = ends ? -1 : wide ? -2 : need;          // until the sums are known
        need_sum += need;
        give_sum += ends ? before : 0;
    }
    const int need_upto = wave_inclusive_scan(need_sum), give_upto = wave_inclusive_scan(give_sum);
    if (lane == 63) {
        s_wave[0][wave] = need_upto;
        s_wave[1][wave] = give_upto;
    }
    __syncthreads();
    int taken_before = need_upto - need_sum, given_before = give_upto - give_sum, given = 0;
    for (int w = 0; w < PLAN_WAVES; ++w) {
        taken_before += w < wave ? s_wave[0][w] : 0;
        given_before += w < wave ? s_wave[1][w] : 0;
        given += s_wave[1][w];
    }
    int taken = 0;
    for (int r = r0; r < r1; ++r) {
        const int kind = s_limit[r], len = s_lens[r];
        const bool ends = kind == -1;
        const int need = max(kind, 0);
        const bool no = kind == -2 || (need > 0 && taken_before + need > free_pages);
        s_first[r] = ends ? given_before : taken_before;
        s_limit[r] = ends ? -1 : no ? 0 : add[r];
        taken_before += need;
        given_before += ends ? pages_of(len) : 0;
        if (need > 0 && !no) taken = taken_before;          // sums only grow: the last granted one is the largest
        if (blockIdx.x == 0) {
            lens_out[r] = ends ? 0 : no ? lens[r] : len + add[r];
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
    for (int r = blockIdx.x * PLAN_WAVES + wave; r < R; r += gridDim.x * PLAN_WAVES) {
        const int limit = s_limit[r], before = pages_of(s_lens[r]), first = s_first[r];
        int32_t *row = table + (size_t)r * max_pages;
        if (limit < 0) {
            for (int i = lane; i < before; i += 64)
                if (first + i < pages - free_pages)         // no more than there are places for
                    ring[((uint32_t)head + (uint32_t)free_pages + (uint32_t)(first + i)) % (uint32_t)pages] = row[i];
        } else {
            const int after = pages_of(s_lens[r] + limit);
            for (int i = before + lane; i < after; i += 64)
                row[i] = ring[((uint32_t)head + (uint32_t)(first + i - before)) % (uint32_t)pages];
        }
    }

    // slots
    for (int64_t t = (int64_t)blockIdx.x * PLAN_THREADS + tid; t < T; t += (int64_t)gridDim.x * PLAN_THREADS) {
        int lo = 0, hi = R;                                 // the last request that starts at or before t
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (s_starts[mid] <= (int)t) lo = mid;
            else hi = mid - 1;
        }
        int64_t slot = -1;
        if (lo < R) {
            const int place = keep != nullptr ? keep[t] : (int)t - s_starts[lo];
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

// A value and its index as one word that grows with the value and falls with the index: NaN above all, -0 equal to 0.
__device__ __forceinline__ uint64_t best_key(float v, uint32_t index)
{
    const uint32_t u = __float_as_uint(v + 0.f);
    const uint32_t o = (u & 0x7fffffffu) > 0x7f800000u ? 0xffffffffu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
    return ((uint64_t)o << 32) | (0xffffffffu - index);
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

// The largest logit of a part of a row.  A row is cut where 16-byte vectors begin, whatever its own alignment: part p has the
// vectors [p per, (p + 1) per) counted from the aligned address at or before the row.
template <typename W>
__global__ __launch_bounds__(BEST_THREADS) void k_logits_best(const W *logits, int64_t stride, int V, int per, uint64_t *parts)
{
    constexpr int VEC = Elem<W>::VEC;
    __shared__ uint64_t s_best[BEST_THREADS / 64];
    const W *row = logits + (int64_t)blockIdx.x * stride;
    const int skew = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / Elem<W>::BYTES);
    const int vectors = (V + skew + VEC - 1) / VEC;
    const int end = min((int)(blockIdx.y + 1) * per, vectors);
    uint64_t best = 0;
    for (int i = blockIdx.y * per + threadIdx.x; i < end; i += BEST_THREADS) {
        const int at = i * VEC - skew;
        if (at >= 0 && at + VEC <= V) {
            float v[VEC];
            load_vec(row + at, v);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const uint64_t key = best_key(v[j], at + j);
                best = key > best ? key : best;
            }
        } else {
            for (int j = max(at, 0); j < min(at + VEC, V); ++j) {
                const uint64_t key = best_key(to_f32(row[j]), j);
                best = key > best ? key : best;
            }
        }
    }
    best = wave_max_u64(best);
    if ((threadIdx.x & 63) == 0) s_best[threadIdx.x >> 6] = best;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < BEST_THREADS / 64; ++w) best = s_best[w] > best ? s_best[w] : best;
        parts[(size_t)blockIdx.x * gridDim.y + blockIdx.y] = best;
    }
}

// One wave a request, a lane a node: the rows' answers from their parts, then down the tree; the last block has the padding.
__global__ __launch_bounds__(64) void k_tree_walk(const uint64_t *parts, int n_parts, const int32_t *tokens, const uint64_t *tree,
                                                  const int32_t *starts, int R, int T, int max_nodes, int32_t *keep,
                                                  int32_t *counts, int32_t *next, int32_t *best)
{
    const int r = blockIdx.x, lane = threadIdx.x;
    const auto answer = [&](int t) {
        uint64_t k = 0;
        for (int p = 0; p < n_parts; ++p) {
            const uint64_t o = parts[(size_t)t * n_parts + p];
            k = o > k ? o : k;
        }
        return (int)(0xffffffffu - (uint32_t)k);
    };
    const int a = min(max(starts[r], 0), T), b = r < R ? min(max(starts[r + 1], a), T) : T;
    const int n = r < R ? min(b - a, max_nodes) : 0;
    const bool node = lane < n;
    int mine = -1, token = -2, parent = -1;
    if (node) {
        mine = answer(a + lane);
        best[a + lane] = mine;
        token = tokens[a + lane];
        const uint64_t before = (1ull << lane) - 1;
        const uint64_t up = tree != nullptr ? tree[a + lane] & before : before;
        parent = up != 0 ? 63 - __clzll((long long)up) : -1;
    }
    if (r < R) {
        int place = lane == 0 ? 0 : -1, count = n > 0 ? 1 : 0, at = 0;
        while (count > 0) {                                 // at grows with every step
            const int answered = __shfl(mine, at);
            const uint64_t agree = __ballot(node && lane > at && parent == at && token == answered);
            if (agree == 0) break;
            at = __ffsll((unsigned long long)agree) - 1;
            if (lane == at) place = count;
            ++count;
        }
        const int following = __shfl(mine, at);
        if (node) keep[a + lane] = place;
        if (lane == 0) {
            counts[r] = count;
            next[r] = count > 0 ? following : -1;
        }
    }
    for (int t = a + n + lane; t < b; t += 64) {            // rows that are no node
        best[t] = answer(t);
        keep[t] = -1;
    }
}

// ---- K and V into their pages ---------------------------------------------------------------------------------------------

constexpr int COMMIT_THREADS = 256;
constexpr int COMMIT_ROWS = 8;

// Rows [8 blockIdx.x, + 8) of layer blockIdx.y.  K is copied in 16-byte vectors.  V lies with e tokens of a channel side by side:
// where e rows in a row fill such a pack (prompts), their elements are exchanged between registers and written as whole
// packs by the rows of the pack's first token; other rows (branches of a tree) write their elements one by one.
template <typename W>
__global__ __launch_bounds__(COMMIT_THREADS) void k_kv_commit(W *K, W *V, const W *k, int64_t k_layer, int64_t k_row,
                                                              const W *v, int64_t v_layer, int64_t v_row,
                                                              const int64_t *slots, int T, int pages, int page_bits, int heads,
                                                              int dim)
{
    constexpr int E = Elem<W>::VEC;
    __shared__ int64_t s_slot[COMMIT_ROWS];
    __shared__ int s_whole[COMMIT_ROWS];          // 0: element by element, 1: writes a pack, 2: another row writes it
    const int tid = threadIdx.x, t0 = blockIdx.x * COMMIT_ROWS, layer = blockIdx.y;
    const int64_t all = (int64_t)pages << page_bits;
    if (tid < COMMIT_ROWS) {
        const int t = t0 + tid;
        const int64_t s = t < T ? slots[t] : -1;
        const bool real = s >= 0 && s < all;
        const int j = (int)(s & (E - 1)), first = t - j;
        bool whole = real && first >= 0 && first + E <= T;
        for (int i = 0; i < E && whole; ++i) whole = slots[first + i] == s - j + i;
        s_slot[tid] = real ? s : -1;
        s_whole[tid] = whole ? (j == 0 ? 1 : 2) : 0;
    }
    __syncthreads();
    const int page = 1 << page_bits, vectors = heads * dim / E;
    k += (int64_t)layer * k_layer;
    v += (int64_t)layer * v_layer;
    const int64_t layer_at = (int64_t)layer * pages * heads;
    for (int i = tid; i < COMMIT_ROWS * vectors; i += COMMIT_THREADS) {
        const int row = i / vectors, at = (i - row * vectors) * E, h = at / dim, c = at - h * dim;
        const int64_t slot = s_slot[row];
        if (slot < 0) continue;
        const int t = t0 + row, place = (int)(slot & (page - 1));
        const int64_t base = ((layer_at + (slot >> page_bits) * heads + h) << page_bits) * dim;
        *reinterpret_cast<uint4 *>(K + base + (int64_t)place * dim + c) = load_raw(k + t * k_row + at);
        W *to = V + base + ((int64_t)(place / E) * dim + c) * E;
        if (s_whole[row] == 1) {
            W in[E][E];
#pragma unroll
            for (int j = 0; j < E; ++j) __builtin_memcpy(in[j], __builtin_assume_aligned(v + (t + j) * v_row + at, 16), 16);
#pragma unroll
            for (int d = 0; d < E; ++d) {
                W out[E];
#pragma unroll
                for (int j = 0; j < E; ++j) out[j] = in[j][d];
                __builtin_memcpy(__builtin_assume_aligned(to + d * E, 16), out, 16);
            }
        } else if (s_whole[row] == 0) {
            W in[E];
            __builtin_memcpy(in, __builtin_assume_aligned(v + t * v_row + at, 16), 16);
#pragma unroll
            for (int d = 0; d < E; ++d) to[d * E + (place & (E - 1))] = in[d];
        }
    }
}

}  // namespace svdp
