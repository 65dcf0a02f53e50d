// Attention of drafted tokens over paged K and V and over their own tree.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svdp_device.h"

namespace svdp {

struct TreeAttnArgs {
    const void *K, *V;                  // of the layer
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    const uint64_t *tree;
    const int32_t *table, *lens, *starts;
    void *out;
    float *lse;
    float scale;
    int max_pages, pages, page_bits, heads, group, R, T, max_nodes;
};

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
    return v;
}

// One wave a row and query head: 64 tokens at a time, a lane a token for the scores and a lane every 64th channel for the sum.
template <typename W, int DIM>
__global__ __launch_bounds__(64) void k_tree_attn(TreeAttnArgs A)
{
    constexpr int E = Elem<W>::VEC, PER = DIM / 64;
    const int lane = threadIdx.x, t = blockIdx.x, hq = blockIdx.y, h = hq / A.group;
    int lo = 0, hi = A.R;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (A.starts[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    if (lo >= A.R) return;
    const int a = max(A.starts[lo], 0), n = min(min(A.starts[lo + 1], A.T) - a, A.max_nodes), node = t - a;
    if (node < 0 || node >= n) return;
    const int page = 1 << A.page_bits, len = min(max(A.lens[lo], 0), A.max_pages << A.page_bits);
    const int heads_q = A.heads * A.group;
    const W *q = static_cast<const W *>(A.q) + t * A.q_stride + (int64_t)hq * DIM;
    const W *K = static_cast<const W *>(A.K), *V = static_cast<const W *>(A.V);
    const int32_t *table = A.table + (size_t)lo * A.max_pages;
    const uint64_t sees = A.tree != nullptr ? A.tree[t] : ~0ull >> (63 - node);
    float top = -INFINITY, total = 0.f, acc[PER] = {};
    for (int at = 0; at < len + n; at += 64) {
        const int j = at + lane;
        const W *key = nullptr, *value = nullptr;
        int64_t value_step = 0;
        if (j < len) {
            const int id = table[j >> A.page_bits];
            if (id >= 0 && id < A.pages) {
                const int place = j & (page - 1);
                const int64_t base = (((int64_t)id * A.heads + h) << A.page_bits) * DIM;
                key = K + base + (int64_t)place * DIM;
                value = V + base + (int64_t)(place / E) * DIM * E + (place & (E - 1));
                value_step = E;
            }
        } else if (j < len + n && ((sees >> (j - len)) & 1)) {
            key = static_cast<const W *>(A.k) + (a + j - len) * A.k_stride + (int64_t)h * DIM;
            value = static_cast<const W *>(A.v) + (a + j - len) * A.v_stride + (int64_t)h * DIM;
            value_step = 1;
        }
        float s = -INFINITY;
        if (key != nullptr) {
            s = 0.f;
            for (int c = 0; c < DIM; ++c) s = fmaf(to_f32(q[c]), to_f32(key[c]), s);
            s *= A.scale;
        }
        const float next = fmaxf(top, wave_max(s)), shift = next == -INFINITY ? 0.f : next;
        const float p = key != nullptr ? __expf(s - shift) : 0.f, old = __expf(top - shift);
        top = next;
        total = total * old + wave_sum(p);
#pragma unroll
        for (int i = 0; i < PER; ++i) acc[i] *= old;
        for (int o = 0; o < 64; ++o) {
            const W *from = reinterpret_cast<const W *>(__shfl((unsigned long long)(uintptr_t)value, o));
            const int64_t step = __shfl(value_step, o);
            const float w = __shfl(p, o);
            if (from == nullptr) continue;
#pragma unroll
            for (int i = 0; i < PER; ++i) acc[i] = fmaf(w, to_f32(from[(lane + 64 * i) * step]), acc[i]);
        }
    }
    W *out = static_cast<W *>(A.out) + ((int64_t)t * heads_q + hq) * DIM;
#pragma unroll
    for (int i = 0; i < PER; ++i) from_f32(total == 0.f ? 0.f : acc[i] / total, out + lane + 64 * i);
    if (A.lse != nullptr && lane == 0)
        A.lse[(int64_t)t * heads_q + hq] = total == 0.f ? -INFINITY : top + logf(total);
}

}  // namespace svdp
