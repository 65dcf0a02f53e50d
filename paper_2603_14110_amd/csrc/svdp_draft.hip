// C-ABI entry points of decoding with drafted tokens (see include/svdp.h): host-side validation and kernel launches.  No
// allocation, no synchronisation, no state kept between calls.
#include "../../include/svdp.h"

#include <hip/hip_runtime.h>

#include "svdp_draft_kernels.h"
#include "svdp_host.h"
#include "svdp_kv8.h"
#include "svdp_tree_attn.h"
#include "svdp_tree_wide.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace {

using namespace svdp;

constexpr int64_t INT_LIMIT = (int64_t)1 << 31;

template <typename T>
struct Type {
    using type = T;
};
// f(W tag) for a storage type
template <typename F>
auto on_type(int dt, F &&f)
{
    return dt == SVDP_F32 ? f(Type<float>{}) : f(Type<bf16>{});
}

// of the cache: its own types, or codes with powers of two
template <typename F>
auto on_cache_type(int dt, F &&f)
{
    return dt == SVDP_E4M3 ? f(Type<e4m3>{}) : on_type(dt, f);
}

inline int row_type(int dt) { return dt == SVDP_E4M3 ? SVDP_BF16 : dt; }             // of q, k, v and out
inline int bytes_of(int dt) { return dt == SVDP_F32 ? 4 : dt == SVDP_BF16 ? 2 : 1; }
inline bool aligned_to(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline bool whole_vectors(int64_t stride, int dt) { return stride % (16 / bytes_of(dt)) == 0; }
inline bool good_page(int page) { return page == 32 || page == 64 || page == 128 || page == 256; }
inline int bits_of(int n) { return n == 32 ? 5 : n == 64 ? 6 : n == 128 ? 7 : 8; }
inline int tiles(int64_t n, int per) { return (int)((n + per - 1) / per); }

bool overlap(const void *a, size_t an, const void *b, size_t bn)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return an > 0 && bn > 0 && x < y + bn && y < x + an;
}

svdp_status check_cache(const svdp_kv_cache *c)
{
    if (c == nullptr || c->layers < 1 || c->pages < 1 || c->heads < 1) return SVDP_ERR_INVALID_ARG;
    if (c->dtype != SVDP_F32 && c->dtype != SVDP_BF16 && c->dtype != SVDP_E4M3) return SVDP_ERR_UNSUPPORTED;
    if (!good_page(c->page) || (c->dim != 64 && c->dim != 128 && c->dim != 256)) return SVDP_ERR_UNSUPPORTED;
    if ((int64_t)c->pages * c->page >= INT_LIMIT || c->heads > 65535 || c->layers > 65535) return SVDP_ERR_UNSUPPORTED;
    return SVDP_OK;
}
svdp_status check_cache_memory(const svdp_kv_cache *c)
{
    if (!c->K || !c->V || !aligned16(c->K) || !aligned16(c->V)) return SVDP_ERR_INVALID_ARG;
    if (c->dtype == SVDP_E4M3 && (!c->K_scale || !c->V_scale || !aligned16(c->K_scale) || !aligned16(c->V_scale))) return SVDP_ERR_INVALID_ARG;
    return SVDP_OK;
}
svdp_status check_requests(int R, int T, int max_nodes)
{
    if (R < 1 || T < 0 || max_nodes < 1) return SVDP_ERR_INVALID_ARG;
    if (R > SVDP_MAX_REQUESTS || T > SVDP_MAX_ROWS || max_nodes > SVDP_MAX_NODES) return SVDP_ERR_UNSUPPORTED;
    return SVDP_OK;
}
svdp_status check_table(int R, int max_pages, int page)
{
    if (max_pages < 1) return SVDP_ERR_INVALID_ARG;
    if ((int64_t)R * max_pages >= INT_LIMIT || (int64_t)max_pages * page >= INT_LIMIT) return SVDP_ERR_UNSUPPORTED;
    return SVDP_OK;
}
svdp_status check_ws(void *ws, size_t ws_bytes, size_t need)
{
    return ws == nullptr || !aligned_to(ws, ALIGN) || ws_bytes < need ? SVDP_ERR_WORKSPACE : SVDP_OK;
}

// Which attention kernel: rows are the nodes of a request times the query heads that share a head of K and V.
struct AttnPlan {
    bool wide;              // rows over the waves of a block (k_tree_attn_wide), or tokens (k_tree_attn)
    int nt;                 // row tiles of 16 in k_tree_attn
    int block_bits, part_rows;      // part_rows 0: nothing is cut, no second launch
    int64_t steps, tasks;   // units of a request and head, and requests times heads times row tiles, at most
    size_t bytes;
};
template <typename F>
void on_dim(int dim, F &&f)
{
    if (dim == 64) f(std::integral_constant<int, 64>{});
    else if (dim == 128) f(std::integral_constant<int, 128>{});
    else f(std::integral_constant<int, 256>{});
}
// f(W tag, DIM, cut) of the kernel that a plan takes
template <typename F>
void on_kernel(const AttnPlan &p, int dt, int dim, F &&f)
{
    on_dim(dim, [&](auto dc) {
        constexpr int DIM = decltype(dc)::value;
        if constexpr (DIM <= 128)
            if (p.wide) return dt == SVDP_E4M3 ? f(Type<e4m3>{}, dc, WideCut<DIM>{}) : f(Type<bf16>{}, dc, WideCut<DIM>{});
        on_cache_type(dt, [&](auto wt) {
            using W = typename decltype(wt)::type;
            if constexpr (DIM <= 128)
                if (p.nt == 2) return f(wt, dc, NarrowCut<W, DIM, 2>{});
            f(wt, dc, NarrowCut<W, DIM, 1>{});
        });
    });
}
// Units of a request and head up to which a block takes them all and there is nothing to join, if no block has two of them: one row,
// 250 tokens: 9.7 us and a call 12.3, cut 7.2 + 3.6 and 15.7; 20 requests of 32 rows 15.2 us, cut 17.4 + 4.4; seven units 14.1 us, cut
// 7.6 + 3.7.  Rows over the waves, 120 tokens: 64 rows 14.0 us and a call 13.8, cut 10.6 + 3.5 and 15.0; 20 requests of 64 rows 15.2,
// cut 19.6 + 7.1; 448 rows of one request, the other way round, 19.8 and 19.5, cut 14.8 + 4.0 and 17.6.
constexpr int UNCUT = 4, UNCUT_WIDE = 2;
AttnPlan attn_plan(const svdp_kv_cache *c, int heads_q, int R, int max_pages, int max_nodes)
{
    const int dt = c->dtype, dim = c->dim, group = heads_q / c->heads;
    const int64_t rows = (int64_t)group * max_nodes, room = (int64_t)max_pages * c->page / TA_TILE, own = tiles(max_nodes, TA_TILE);
    AttnPlan p;
    // More than 32 rows: over the waves, 32 each (eight requests of 4096 tokens, 135 MB: 36 and 64 rows 36 us, where k_tree_attn, with
    // two row tiles after each other, takes 48).  At 32 rows k_tree_attn is ahead: 26.4 us for one request of 30 000 tokens and 13.4
    // for 24 of 150, where rows over the waves took 32.0 and 16.6 + 4.4.
    // An 8-bit cache: more than 64, as reading K and V once more costs half (eight requests of 4096 tokens: 36 rows 31.5 us, over the
    // waves 44.3; 64 rows 36.1 and 45.8; 100 rows 47.8 and 48.0; 128 rows 56.3 and 49.9; 24 requests of 150 tokens and 98 rows 25.0 and 20.2).
    p.wide = dim <= 128 && (dt == SVDP_BF16 ? rows > 32 : dt == SVDP_E4M3 && rows > 64);
    // Two row tiles of 16 read K and V once for 32 rows (8 requests of 4096 tokens, 135 MB: 29.6 us, one after the other 45.2); with
    // 256 channels a second one does not fit the registers.
    p.nt = rows <= 16 || dim == 256 ? 1 : 2;
    int unit, block_rows;
    on_kernel(p, dt, dim, [&](auto, auto, auto cut) {
        using Cut = decltype(cut);
        unit = Cut::UNIT;
        block_rows = Cut::ROWS;
        p.block_bits = Cut::BITS;
    });
    p.steps = p.wide ? tiles(room, unit) + tiles(own, unit) : tiles(room + own, unit);
    p.tasks = (rows + block_rows - 1) / block_rows * c->heads * R;
    const bool uncut = p.steps <= 1 || (p.steps <= (p.wide ? UNCUT_WIDE : UNCUT) && p.tasks <= 1 << p.block_bits);
    p.part_rows = uncut ? 0 : (int)std::min<int64_t>(rows, block_rows);
    p.bytes = std::max(align_up(((size_t)2 << p.block_bits) * tree_part_floats(p.part_rows, dim) * 4), ALIGN);
    return p;
}
// Rows and heads from which the join has a wave for each, whatever the parts (12 288 of 24 requests: 7.1 us, with a block each 33.6; 256
// of one request, with 32 parts: 7.4 us, with a block each 4.0; in between it depends on the parts: 512 with 32 of them 7.8 and 4.8, 2048
// with few 4.6 and 5.4).
constexpr int JOIN_WAVES = 512;
// K and V of few rows: fewer channels a block, until there are so many blocks (five rows of 4096 channels in 32 layers: 6.6 us, with
// one block for all channels 14.0; 500 rows of 1024 channels in 32 layers: 21.6 us, up to 16 384 blocks 23.4).
constexpr int COMMIT_BLOCKS = 4096;
// Heads of a block that writes or reads 8-bit rows (reads any): fewer, until there are so many blocks (a row of 32 heads in 32 layers stored
// in 3.6 us, up to 4096 blocks 4.5; 40 rows of 8 heads 6.3 and 7.3; five rows of 32 heads 5.2, with all heads in a block 18.9).
constexpr int KV_BLOCKS = 1024;

// Rows of K and V, as a commit reads and a read writes them.
svdp_status check_rows(const svdp_kv_cache *c, const int64_t *slots, int T, const void *k, int64_t k_layer, int64_t k_row, const void *v, int64_t v_layer,
                       int64_t v_row)
{
    if (T < 0) return SVDP_ERR_INVALID_ARG;
    if (T > SVDP_MAX_ROWS) return SVDP_ERR_UNSUPPORTED;
    if (T == 0) return SVDP_OK;
    const int rt = row_type(c->dtype);
    const int64_t row = (int64_t)c->heads * c->dim;
    if (!k || !v || !slots || !aligned16(k) || !aligned16(v) || !aligned_to(slots, 8) || k_row < row || v_row < row || k_layer < 0 || v_layer < 0 ||
        !whole_vectors(k_row, rt) || !whole_vectors(v_row, rt) || !whole_vectors(k_layer, rt) || !whole_vectors(v_layer, rt))
        return SVDP_ERR_INVALID_ARG;
    return SVDP_OK;
}
// Rows of `row` elements at l * layer + t * step, l < layers, t < T, step >= row.  Whether one of them and one of the same rows moved by `apart`
// elements have an element in common (apart 0: two different rows).  For each difference of layers only the two nearest of rows can.
bool rows_meet(int64_t apart, int layers, int T, int64_t layer, int64_t step, int64_t row)
{
    if (layers == 1) layer = 0;
    if (T == 1) step = row;
    const int64_t far = apart < 0 ? -apart : apart;
    // one layer after the other, and between two rows of the one there is room for one of the other
    if ((layers == 1 || layer >= (T - 1) * step + far + row) && (apart == 0 || (far >= row && far + row <= step))) return false;
    for (int l = apart == 0 ? 1 : 1 - layers; l < layers; ++l) {
        const int64_t at = apart + l * layer, t = at / step;                // rows at - t step + (-1, 0, 1) step apart
        for (int64_t i = t - 1; i <= t + 1; ++i)
            if (i > -T && i < T && at - i * step > -row && at - i * step < row) return true;
    }
    return false;
}
// What is written: no row may overlap another one.  K's rows and V's are compared where their strides are the same, else their first ones.
bool rows_apart(const svdp_kv_cache *c, int T, const void *k, int64_t k_layer, int64_t k_row, const void *v, int64_t v_layer, int64_t v_row)
{
    const int64_t row = (int64_t)c->heads * c->dim, apart = ((intptr_t)v - (intptr_t)k) / bytes_of(row_type(c->dtype));
    constexpr int64_t MOST = (int64_t)1 << 46;                              // elements: more than any memory has; what follows stays in range
    if (std::max(k_layer, v_layer) >= MOST / c->layers && c->layers > 1) return false;
    if (std::max(k_row, v_row) >= MOST / T && T > 1) return false;
    if (rows_meet(0, c->layers, T, k_layer, k_row, row) || rows_meet(0, c->layers, T, v_layer, v_row, row)) return false;
    if (apart > -row && apart < row) return false;
    const auto extent = [&](int64_t layer, int64_t step) { return (c->layers > 1 ? (c->layers - 1) * layer : 0) + (T > 1 ? (T - 1) * step : 0) + row; };
    if (apart >= extent(k_layer, k_row) || -apart >= extent(v_layer, v_row)) return true;
    const bool alike = (c->layers == 1 || k_layer == v_layer) && (T == 1 || k_row == v_row);
    return !alike || !rows_meet(apart, c->layers, T, k_layer, k_row, row);
}
KvArgs kv_args(const svdp_kv_cache *c, const int64_t *slots, int T, const void *k, int64_t k_layer, int64_t k_row, const void *v, int64_t v_layer,
               int64_t v_row)
{
    // heads of a block: fewer, until there are so many blocks
    int each = c->heads;
    while (each > 1 && (int64_t)tiles(T, KV_ROWS) * c->layers * 2 * tiles(c->heads, each) < KV_BLOCKS) each = (each + 1) / 2;
    return {c->K, c->V, c->K_scale, c->V_scale, const_cast<void *>(k), const_cast<void *>(v), k_layer, k_row, v_layer, v_row, slots, T, c->pages,
            bits_of(c->page), c->heads, each};
}
dim3 kv_grid(const svdp_kv_cache *c, const KvArgs &A) { return dim3(tiles(A.T, KV_ROWS), c->layers, 2 * tiles(A.heads, A.heads_each)); }

// Bytes of a request's logits up to which one block reads them and walks, in one launch (125 KB: a call 9.6 us and 6.1 on the GPU,
// in two launches 12.4 and 3.3 + 1.6; 250 KB: 9.6 and 8.9, in two 12.3 and 3.3 + 1.7, so a caller who waits loses; 500 KB: 15.1, in two 12.2).
constexpr int64_t ACCEPT_SMALL = 128 << 10;

constexpr int BEST_ROWS = 1 << 23;        // of a launch: its threads are counted in 32 bits
static_assert((int64_t)BEST_ROWS * BEST_THREADS < (int64_t)1 << 32);

// Parts that a row of logits is cut into: about a thousand blocks altogether, each of 8 to 32 KB.
int best_parts(int T, int V, int dt)
{
    const int64_t row = (int64_t)V * bytes_of(dt);
    const int64_t part = std::min<int64_t>(std::max<int64_t>(row * T / 1024, 8 << 10), 32 << 10);
    return (int)std::min<int64_t>((row + part - 1) / part, 65535);
}

}  // namespace

extern "C" {

size_t svdp_tree_attn_workspace_bytes(const svdp_kv_cache *cache, int32_t heads_q, int32_t R, int32_t max_pages,
                                      int32_t max_nodes)
{
    if (check_cache(cache) != SVDP_OK || check_requests(R, 0, max_nodes) != SVDP_OK ||
        check_table(R, max_pages, cache->page) != SVDP_OK || heads_q < 1 || heads_q % cache->heads != 0)
        return 0;
    const AttnPlan plan = attn_plan(cache, heads_q, R, max_pages, max_nodes);
    return plan.steps * plan.tasks < INT_LIMIT ? plan.bytes : 0;
}

svdp_status svdp_tree_attn(const svdp_kv_cache *cache, int32_t layer, const void *q, int64_t q_stride, const void *k,
                           int64_t k_stride, const void *v, int64_t v_stride, const uint64_t *tree, const int32_t *table,
                           int32_t max_pages, const int32_t *lens, const int32_t *starts, int32_t R, int32_t T,
                           int32_t max_nodes, int32_t heads_q, float scale, void *out, float *lse, void *ws,
                           size_t ws_bytes, void *stream)
{
    svdp_status st = check_cache(cache);
    if (st == SVDP_OK) st = check_cache_memory(cache);
    if (st == SVDP_OK) st = check_requests(R, T, max_nodes);
    if (st == SVDP_OK) st = check_table(R, max_pages, cache->page);
    if (st != SVDP_OK) return st;
    const int dt = cache->dtype, rt = row_type(dt), dim = cache->dim;
    if (layer < 0 || layer >= cache->layers || heads_q < 1 || heads_q % cache->heads != 0 || !std::isfinite(scale * LOG2E))
        return SVDP_ERR_INVALID_ARG;
    if ((int64_t)T * heads_q >= 1 << 26) return SVDP_ERR_UNSUPPORTED;        // a wave each in the join: threads of a grid
    if (T == 0) return SVDP_OK;
    if (!q || !k || !v || !out || !table || !lens || !starts || !aligned16(q) || !aligned16(k) || !aligned16(v) ||
        !aligned16(out) || !aligned_to(table, 4) || !aligned_to(lens, 4) || !aligned_to(starts, 4) ||
        !aligned_to(tree, 8) || !aligned_to(lse, 4))
        return SVDP_ERR_INVALID_ARG;
    if (q_stride < (int64_t)heads_q * dim || k_stride < (int64_t)cache->heads * dim ||
        v_stride < (int64_t)cache->heads * dim || !whole_vectors(q_stride, rt) || !whole_vectors(k_stride, rt) ||
        !whole_vectors(v_stride, rt))
        return SVDP_ERR_INVALID_ARG;
    const AttnPlan plan = attn_plan(cache, heads_q, R, max_pages, max_nodes);
    if (plan.steps * plan.tasks >= INT_LIMIT) return SVDP_ERR_UNSUPPORTED;
    st = check_ws(ws, ws_bytes, plan.bytes);
    if (st != SVDP_OK) return st;
    const size_t layer_bytes = (size_t)cache->pages * cache->heads * cache->page * dim * bytes_of(dt);
    TreeAttnArgs A{};
    A.K = static_cast<const char *>(cache->K) + layer * layer_bytes;
    A.V = static_cast<const char *>(cache->V) + layer * layer_bytes;
    if (dt == SVDP_E4M3) {
        A.K_scale = cache->K_scale + layer * (layer_bytes / dim);
        A.V_scale = cache->V_scale + layer * (layer_bytes / dim);
    }
    A.q = q;
    A.k = k;
    A.v = v;
    A.q_stride = q_stride;
    A.k_stride = k_stride;
    A.v_stride = v_stride;
    A.tree = tree;
    A.table = table;
    A.lens = lens;
    A.starts = starts;
    A.out = out;
    A.lse = lse;
    A.scale = scale;
    A.room = max_pages << bits_of(cache->page);
    A.max_pages = max_pages;
    A.pages = cache->pages;
    A.page_bits = bits_of(cache->page);
    A.heads = cache->heads;
    A.group = heads_q / cache->heads;
    A.R = R;
    A.T = T;
    A.max_nodes = (uint16_t)max_nodes;
    A.parts = static_cast<float *>(ws);
    A.part_rows = (uint16_t)plan.part_rows;
    const TreeJoinArgs J = A;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const dim3 blocks(1 << plan.block_bits);
    bool granted = true;
    // A row has at most blocks / heads parts and two more: up to eight, which a wave reads at
    // once, or many rows, a wave each.
    const int items = T * heads_q;
    const bool shared = items < JOIN_WAVES && (1 << plan.block_bits) / cache->heads + 2 > 8;
    on_kernel(plan, dt, dim, [&](auto wt, auto dc, auto cut) {
        using W = typename decltype(wt)::type;
        using Cut = decltype(cut);
        constexpr int DIM = decltype(dc)::value;
        if constexpr (Cut::ROWS == TW_ROWS) {
            granted = grant_lds<k_tree_attn_wide<W, DIM>>(TW_LDS);
            if (!granted) return;
            launch((k_tree_attn_wide<W, DIM>), blocks, dim3(TW_THREADS), TW_LDS, hs, A);
        } else {
            launch((k_tree_attn<W, DIM, Cut::ROWS / 16>), blocks, dim3(TA_THREADS), 0, hs, A);
        }
        if (plan.part_rows == 0) return;
        if (shared) launch((k_tree_join<W, DIM, Cut, true>), dim3(items), dim3(64 * tj_waves<true>()), 0, hs, J);
        else launch((k_tree_join<W, DIM, Cut, false>), dim3(tiles(items, tj_waves<false>())), dim3(64 * tj_waves<false>()), 0, hs, J);
    });
    return granted ? hip_status(hipSuccess) : SVDP_ERR_UNSUPPORTED;
}

size_t svdp_tree_accept_workspace_bytes(int32_t T, int32_t V, int32_t dtype)
{
    if (T < 0 || T > SVDP_MAX_ROWS || V < 1 || (dtype != SVDP_F32 && dtype != SVDP_BF16)) return 0;
    return std::max(align_up((size_t)T * best_parts(T, V, dtype) * 8), ALIGN);
}

svdp_status svdp_tree_accept(const void *logits, int64_t stride, int32_t dtype, int32_t V, const int32_t *tokens,
                             const uint64_t *tree, const int32_t *starts, int32_t R, int32_t T, int32_t max_nodes,
                             int32_t *keep, int32_t *counts, int32_t *next, int32_t *best, void *ws, size_t ws_bytes,
                             void *stream)
{
    svdp_status st = check_requests(R, T, max_nodes);
    if (st != SVDP_OK) return st;
    if (V < 1 || stride < V) return SVDP_ERR_INVALID_ARG;
    if (dtype != SVDP_F32 && dtype != SVDP_BF16) return SVDP_ERR_UNSUPPORTED;
    if (V > (1 << 30)) return SVDP_ERR_UNSUPPORTED;
    if (!starts || !counts || !next || !aligned_to(starts, 4) || !aligned_to(counts, 4) || !aligned_to(next, 4))
        return SVDP_ERR_INVALID_ARG;
    if (T > 0 && (!logits || !tokens || !keep || !best || !aligned_to(logits, bytes_of(dtype)) || !aligned_to(tokens, 4) ||
                  !aligned_to(tree, 8) || !aligned_to(keep, 4) || !aligned_to(best, 4)))
        return SVDP_ERR_INVALID_ARG;
    st = check_ws(ws, ws_bytes, svdp_tree_accept_workspace_bytes(T, V, dtype));
    if (st != SVDP_OK) return st;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const TreeWalk A{tokens, tree, starts, keep, counts, next, best, R, T, max_nodes};
    on_type(dtype, [&](auto wt) {
        using W = typename decltype(wt)::type;
        const W *rows = static_cast<const W *>(logits);
        if ((int64_t)max_nodes * V * bytes_of(dtype) <= ACCEPT_SMALL && T <= (int64_t)R * max_nodes) {
            launch(k_tree_accept<W>, dim3(2 * R), dim3(SMALL_THREADS), 0, hs, rows, stride, V, A);
            return;
        }
        uint64_t *parts = static_cast<uint64_t *>(ws);
        const int n_parts = best_parts(T, V, dtype);
        // one vector more than the row has where it begins between two of them
        const int per = tiles(tiles(V, Elem<W>::VEC) + 1, n_parts);
        for (int t = 0; t < T; t += BEST_ROWS)
            launch(k_logits_best<W>, dim3(std::min(T - t, BEST_ROWS), n_parts), dim3(BEST_THREADS), 0, hs, rows + t * stride, stride, V, per,
                   parts + (size_t)t * n_parts);
        launch(k_tree_walk, dim3(R + 1), dim3(64), 0, hs, parts, n_parts, A);
    });
    return hip_status(hipSuccess);
}

svdp_status svdp_kv_plan(int32_t *table, int32_t max_pages, int32_t *ring, int32_t pages, int32_t page, const int32_t *pool,
                         const int32_t *lens, const int32_t *add, const int32_t *starts, const int32_t *keep, int32_t R,
                         int32_t T, int64_t *slots, int32_t *lens_out, int32_t *pool_out, int32_t *refused, void *stream)
{
    svdp_status st = check_requests(R, T, 1);
    if (st != SVDP_OK) return st;
    if (pages < 1) return SVDP_ERR_INVALID_ARG;
    if (!good_page(page) || (int64_t)pages * page >= INT_LIMIT) return SVDP_ERR_UNSUPPORTED;
    st = check_table(R, max_pages, page);
    if (st != SVDP_OK) return st;
    const void *words[] = {table, ring, pool, lens, add, starts, lens_out, pool_out, refused};
    for (const void *p : words)
        if (p == nullptr || !aligned_to(p, 4)) return SVDP_ERR_INVALID_ARG;
    if (!aligned_to(keep, 4) || (T > 0 && slots == nullptr) || !aligned_to(slots, 8)) return SVDP_ERR_INVALID_ARG;
    // blocks do not wait for each other: what one of them writes no other may read, nor write
    const size_t rows = (size_t)R * 4;
    const struct {
        const void *at;
        size_t bytes;
        bool written;
    } arrays[] = {{slots, (size_t)T * 8, true}, {lens_out, rows, true}, {refused, rows, true}, {pool_out, 8, true},
                  {table, rows * max_pages, true}, {ring, (size_t)pages * 4, true}, {pool, 8, false}, {lens, rows, false},
                  {add, rows, false}, {starts, rows + 4, false}, {keep, keep != nullptr ? (size_t)T * 4 : 0, false}};
    for (const auto &o : arrays)
        for (const auto &i : arrays)
            if (o.written && &o != &i && overlap(o.at, o.bytes, i.at, i.bytes)) return SVDP_ERR_INVALID_ARG;
    static_assert(SVDP_MAX_REQUESTS <= PLAN_EACH * PLAN_THREADS, "every request has a thread");
    const size_t lds = plan_lds(R);
    if (!grant_lds<k_kv_plan>(lds)) return SVDP_ERR_UNSUPPORTED;
    const int row_blocks = tiles(R, PLAN_WAVES), slot_blocks = std::min(tiles(T, PLAN_THREADS), 256);
    launch(k_kv_plan, dim3(row_blocks + slot_blocks), dim3(PLAN_THREADS), lds, static_cast<hipStream_t>(stream), table, max_pages, ring, pages,
           bits_of(page), pool, lens, add, starts, keep, R, T, row_blocks, slots, lens_out, pool_out,
           refused);
    return hip_status(hipSuccess);
}

svdp_status svdp_tree_walk(const int32_t *answers, const int32_t *tokens, const uint64_t *tree, const int32_t *starts, int32_t R, int32_t T,
                           int32_t max_nodes, int32_t *keep, int32_t *counts, int32_t *next, void *stream)
{
    svdp_status st = check_requests(R, T, max_nodes);
    if (st != SVDP_OK) return st;
    if (!starts || !counts || !next || !aligned_to(starts, 4) || !aligned_to(counts, 4) || !aligned_to(next, 4)) return SVDP_ERR_INVALID_ARG;
    if (T > 0 && (!answers || !tokens || !keep || !aligned_to(answers, 4) || !aligned_to(tokens, 4) || !aligned_to(tree, 8) || !aligned_to(keep, 4)))
        return SVDP_ERR_INVALID_ARG;
    const TreeWalk A{tokens, tree, starts, keep, counts, next, const_cast<int32_t *>(answers), R, T, max_nodes};
    launch(k_tree_walk_given, dim3(R + 1), dim3(64), 0, static_cast<hipStream_t>(stream), A);
    return hip_status(hipSuccess);
}

svdp_status svdp_kv_commit(const svdp_kv_cache *cache, const void *k, int64_t k_layer_stride, int64_t k_row_stride,
                           const void *v, int64_t v_layer_stride, int64_t v_row_stride, const int64_t *slots, int32_t T,
                           void *stream)
{
    svdp_status st = check_cache(cache);
    if (st == SVDP_OK) st = check_cache_memory(cache);
    if (st == SVDP_OK) st = check_rows(cache, slots, T, k, k_layer_stride, k_row_stride, v, v_layer_stride, v_row_stride);
    if (st != SVDP_OK || T == 0) return st;
    const int dt = cache->dtype;
    if (dt == SVDP_E4M3) {
        const KvArgs A = kv_args(cache, slots, T, k, k_layer_stride, k_row_stride, v, v_layer_stride, v_row_stride);
        on_dim(cache->dim, [&](auto dc) {
            launch(k_kv_commit8<decltype(dc)::value>, kv_grid(cache, A), dim3(KV_THREADS), 0, static_cast<hipStream_t>(stream), A);
        });
        return hip_status(hipSuccess);
    }
    const int64_t row = (int64_t)cache->heads * cache->dim;
    const int groups = tiles(T, COMMIT_ROWS);
    int channels = (int)row;
    while (channels > COMMIT_CHANNELS && tiles(row, channels) < COMMIT_BLOCKS / (2 * (int64_t)groups * cache->layers))
        channels = tiles(channels, 2 * COMMIT_CHANNELS) * COMMIT_CHANNELS;
    return on_type(dt, [&](auto wt) {
        using W = typename decltype(wt)::type;
        launch(k_kv_commit<W>, dim3(groups, cache->layers, 2 * tiles(row, channels)), dim3(COMMIT_THREADS), 0,
               static_cast<hipStream_t>(stream), static_cast<W *>(cache->K), static_cast<W *>(cache->V),
               static_cast<const W *>(k), k_layer_stride, k_row_stride, static_cast<const W *>(v), v_layer_stride,
               v_row_stride, slots, T, cache->pages, bits_of(cache->page), cache->heads, bits_of(cache->dim), channels);
        return hip_status(hipSuccess);
    });
}

svdp_status svdp_kv_read(const svdp_kv_cache *cache, const int64_t *slots, int32_t T, void *k, int64_t k_layer_stride, int64_t k_row_stride, void *v,
                         int64_t v_layer_stride, int64_t v_row_stride, void *stream)
{
    svdp_status st = check_cache(cache);
    if (st == SVDP_OK) st = check_cache_memory(cache);
    if (st == SVDP_OK) st = check_rows(cache, slots, T, k, k_layer_stride, k_row_stride, v, v_layer_stride, v_row_stride);
    if (st != SVDP_OK || T == 0) return st;
    if (!rows_apart(cache, T, k, k_layer_stride, k_row_stride, v, v_layer_stride, v_row_stride)) return SVDP_ERR_INVALID_ARG;
    const KvArgs A = kv_args(cache, slots, T, k, k_layer_stride, k_row_stride, v, v_layer_stride, v_row_stride);
    on_cache_type(cache->dtype, [&](auto wt) {
        on_dim(cache->dim, [&](auto dc) {
            launch((k_kv_read<typename decltype(wt)::type, decltype(dc)::value>), kv_grid(cache, A), dim3(KV_THREADS), 0, static_cast<hipStream_t>(stream), A);
        });
    });
    return hip_status(hipSuccess);
}

}  // extern "C"
