// K and V of a cache in 8 bits as they are written, and K and V of any cache read back as rows.
//
// The dim elements x of a token's head become codes x / 2^b, rounded to e4m3 (to the nearest, ties to even), where b >= KV8_LEAST is
// the least whole number with max |x| <= 448 2^b, 448 being the largest e4m3 number.  A power of two costs no precision beside any other
// scale (at most one of the fifteen binades at the lower end), makes x / 2^b and code 2^b exact, and is one byte.
// Infinities and NaN become NaN and do not count for the maximum.  At the largest power, 2^120, codes end at 240 instead of 448: from 256 2^120
// on there is no bf16 number, and what was finite would come back infinite; 255 2^120, the largest one, is off by less than half a step.
//
// What bounds both: reading and writing.  A prompt of 2357 tokens, 32 layers of 8 heads of 128, 465 MB, stored in 87 us, 5.3 TB/s (111 us
// with a wave that has two channels a lane of every token, in 4-byte loads and with a maximum over 64 lanes each); 3400 tokens of the
// same, 892 MB, read in 162 us, 5.5 TB/s.  A branch of five rows in 32 layers of 32 heads: 5.4 us; 77 tokens read: 4.9 us, by latency.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svdp_device.h"

namespace svdp {

constexpr int KV_THREADS = 256, KV_WAVES = KV_THREADS / 64;
constexpr int KV_ROWS = 8;                 // rows of a block: a pack's tokens at the most
constexpr int KV8_LEAST = -96;
constexpr uint32_t KV8_MOST = 120 + 127;   // as it is kept
constexpr float KV8_MOST_CODE = 240.f;

// Biased exponent (b + 127) for the largest magnitude of a token's head.
__device__ __forceinline__ uint32_t kv8_exponent(float top)
{
    const uint32_t u = __float_as_uint(top);
    const int b = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);        // 448 = 1.75 2^8
    return (uint32_t)max(b, KV8_LEAST + 127);
}
// 2^-b
__device__ __forceinline__ float kv8_inverse(uint32_t biased) { return __uint_as_float((254u - biased) << 23); }
__device__ __forceinline__ float kv8_magnitude(float x)
{
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? __uint_as_float(u) : 0.f;
}
__device__ __forceinline__ float kv8_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? NAN : x; }
// What is rounded to codes: x times 2^-b.
template <int N>
__device__ __forceinline__ void kv8_scale(float (&x)[N], uint32_t biased)
{
    const float by = kv8_inverse(biased);
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = kv8_finite(x[j]) * by;
    if (biased == KV8_MOST) {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = fabsf(x[j]) > KV8_MOST_CODE ? copysignf(KV8_MOST_CODE, x[j]) : x[j];      // NaN stays
    }
}
// Four codes in a word.
__device__ __forceinline__ uint32_t kv8_codes(float a, float b, float c, float d)
{
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true);
}

struct KvArgs {
    void *K, *V;
    uint8_t *K_scale, *V_scale;
    void *k, *v;                            // rows: read by the commit, written by the other
    int64_t k_layer, k_row, v_layer, v_row;
    const int64_t *slots;
    int T, pages, page_bits, heads, heads_each;     // heads_each: of a block
};

// What a block knows of its rows [t0, t0 + KV_ROWS): their slots and those around them (-1: none), and for V which of them begin a pack
// whose tokens are all there (whole), and which are on their own.
template <int E>
struct KvRows {
    int64_t near[KV_ROWS + 2 * E];
    int rows[KV_ROWS];                      // whole from the front, alone from the back
    int whole, alone;
    // ALL: rows without a slot are on their own too.
    template <bool ALL>
    __device__ __forceinline__ void look(const KvArgs &A, int t0, int tid)
    {
        const int64_t all = (int64_t)A.pages << A.page_bits;
        if (tid < KV_ROWS + 2 * E) {
            const int t = t0 - E + tid;
            const int64_t s = t >= 0 && t < A.T ? A.slots[t] : -1;
            near[tid] = s >= 0 && s < all ? s : -1;
        }
        __syncthreads();
        if (tid < 64) {
            bool in = false, pack = false, first = false;
            if (tid < KV_ROWS) {
                const int64_t s = near[E + tid];
                const int j = (int)(s & (E - 1));
                in = t0 + tid < A.T && (ALL || s >= 0);
                pack = s >= 0;
                first = j == 0;
#pragma unroll
                for (int i = 0; i < E; ++i) pack = pack && near[E + tid - j + i] == s - j + i;
            }
            const uint64_t front = __ballot(pack && first), back = __ballot(in && !pack), before = (1ull << tid) - 1;
            if (pack && first) rows[__popcll(front & before)] = tid;
            if (in && !pack) rows[KV_ROWS - 1 - __popcll(back & before)] = tid;
            if (tid == 0) {
                whole = __popcll(front);
                alone = __popcll(back);
            }
        }
        __syncthreads();
    }
    __device__ __forceinline__ int64_t slot(int row) const { return near[E + row]; }
};

// Rows [8 blockIdx.x, + 8) of layer blockIdx.y, heads [z / 2 heads_each, + heads_each); even z: K, odd z: V.
// K: dim / 8 lanes a head, eight channels each.  V: where a pack's eight tokens are rows of the step (prompts), a wave takes them all; a token
// on its own is written byte by byte.
template <int DIM>
__global__ __launch_bounds__(KV_THREADS) void k_kv_commit8(KvArgs A)
{
    constexpr int E = 8, LANES = DIM / 8, LOG2 = DIM == 64 ? 3 : DIM == 128 ? 4 : 5, C = DIM / 64;
    __shared__ KvRows<E> s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, t0 = blockIdx.x * KV_ROWS, layer = blockIdx.y;
    const int h0 = (int)(blockIdx.z >> 1) * A.heads_each, hn = min(A.heads_each, A.heads - h0), page = 1 << A.page_bits;
    s.look<false>(A, t0, tid);
    const int64_t layer_at = (int64_t)layer * A.pages * A.heads;
    // token of a slot's head, counted from the cache's beginning
    const auto token_of = [&](int64_t slot, int h) {
        return ((layer_at + (slot >> A.page_bits) * A.heads + h) << A.page_bits) + (slot & (page - 1));
    };
    if (!(blockIdx.z & 1)) {
        const bf16 *k = static_cast<const bf16 *>(A.k) + layer * A.k_layer + t0 * A.k_row + (int64_t)h0 * DIM;
        const int rows = min(KV_ROWS, A.T - t0), items = rows * hn, c = tid % LANES * 8;
        for (int i0 = tid / LANES; i0 - tid / LANES < items; i0 += KV_THREADS / LANES) {
            const int i = min(i0, items - 1), row = i / hn, h = i - row * hn;
            const uint4 raw = load_raw(k + row * A.k_row + (int64_t)h * DIM + c);
            float x[8], top = 0.f;
            widen(raw, x, (const bf16 *)nullptr);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, kv8_magnitude(x[j]));
            const uint32_t by = kv8_exponent(group_max<LOG2>(top));
            kv8_scale(x, by);
            const int64_t slot = s.slot(row);
            if (i0 >= items || slot < 0) continue;
            const int64_t token = token_of(slot, h0 + h);
            *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(A.K) + token * DIM + c) = make_uint2(kv8_codes(x[0], x[1], x[2], x[3]), kv8_codes(x[4], x[5], x[6], x[7]));
            if (c == 0) A.K_scale[token] = (uint8_t)by;
        }
        return;
    }
    const bf16 *v = static_cast<const bf16 *>(A.v) + layer * A.v_layer + t0 * A.v_row + (int64_t)h0 * DIM;
    // Whole packs: a quarter of the wave has two of the tokens, a lane eight of 128 channels (two heads of 64, or 256 twice), in 16-byte loads;
    // the quarters then exchange words of two channels and two tokens, so that a lane has all tokens of two channels.
    constexpr int SIDE = DIM == 64 ? 2 : 1, PIECES = DIM == 256 ? 2 : 1;      // heads, pieces of 128 channels
    const int g = lane >> 4, c8 = (lane & 15) * 8, side = c8 / DIM, groups = (hn + SIDE - 1) / SIDE;
    for (int i = wave; i < s.whole * groups; i += KV_WAVES) {
        const int job = i / groups, h = (i - job * groups) * SIDE + side, row = s.rows[job], channel = c8 - side * DIM;
        const bf16 *from = v + (int64_t)(row + 2 * g) * A.v_row + (int64_t)min(h, hn - 1) * DIM + channel;
        uint4 raw[2][PIECES];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int p = 0; p < PIECES; ++p) raw[t][p] = load_raw(from + t * A.v_row + p * 128);
        float x[2][PIECES][8];
        uint32_t by[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float top = 0.f;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                widen(raw[t][p], x[t][p], (const bf16 *)nullptr);
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, kv8_magnitude(x[t][p][j]));
            }
            by[t] = kv8_exponent(group_max<DIM == 64 ? 3 : 4>(top));
#pragma unroll
            for (int p = 0; p < PIECES; ++p) kv8_scale(x[t][p], by[t]);
        }
        const int64_t token = token_of(s.slot(row), h0 + min(h, hn - 1));                    // the pack's first
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = kv8_codes(x[0][p][2 * q], x[1][p][2 * q], x[0][p][2 * q + 1], x[1][p][2 * q + 1]);
            const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
            const auto front = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), back = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
            // words of tokens 0 and 1, 2 and 3, 4 and 5, 6 and 7 of channels 2 g and 2 g + 1 of the lane's eight
            const uint4 out = make_uint4(__builtin_amdgcn_perm(front[1], front[0], 0x05040100u), __builtin_amdgcn_perm(back[1], back[0], 0x05040100u),
                                         __builtin_amdgcn_perm(front[1], front[0], 0x07060302u), __builtin_amdgcn_perm(back[1], back[0], 0x07060302u));
            if (h < hn) *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(A.V) + token * DIM + (channel + p * 128 + 2 * g) * E) = out;
        }
        if (h < hn && channel == 0) *reinterpret_cast<uint16_t *>(A.V_scale + token + 2 * g) = (uint16_t)(by[0] | by[1] << 8);
    }
    // tokens on their own: C channels a lane
    for (int i = wave; i < s.alone * hn; i += KV_WAVES) {
        const int job = i / hn, h = i - job * hn, row = s.rows[KV_ROWS - 1 - job];
        bf16 in[C];
        __builtin_memcpy(in, __builtin_assume_aligned(v + row * A.v_row + (int64_t)h * DIM + lane * C, sizeof(in)), sizeof(in));
        float x[C], top = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            x[c] = to_f32(in[c]);
            top = fmaxf(top, kv8_magnitude(x[c]));
        }
        const uint32_t by = kv8_exponent(group_max<6>(top));
        kv8_scale(x, by);
        const int64_t token = token_of(s.slot(row), h0 + h);
        const int in_pack = (int)(token & (E - 1));
        uint8_t *to = static_cast<uint8_t *>(A.V) + (token - in_pack) * DIM + in_pack;
#pragma unroll
        for (int c = 0; c < C; ++c) to[(lane * C + c) * E] = (uint8_t)kv8_codes(x[c], 0.f, 0.f, 0.f);
        if (lane == 0) A.V_scale[token] = (uint8_t)by;
    }
}

// The same rows, the other way: K and V of slots as rows of the cache's type (8 bits: bf16, exact for all that the commit writes).  Rows without a
// slot become zeros.
template <typename W, int DIM>
__global__ __launch_bounds__(KV_THREADS) void k_kv_read(KvArgs A)
{
    using Row = typename RowOf<W>::type;
    constexpr bool CODED = sizeof(W) == 1;
    constexpr int E = CODED ? 8 : 16 / (int)sizeof(W), VEC = Elem<Row>::VEC, LANES = DIM / VEC, C = DIM / 64;
    __shared__ KvRows<E> s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, t0 = blockIdx.x * KV_ROWS, layer = blockIdx.y;
    const int h0 = (int)(blockIdx.z >> 1) * A.heads_each, hn = min(A.heads_each, A.heads - h0), page = 1 << A.page_bits;
    s.template look<true>(A, t0, tid);
    const int64_t layer_at = (int64_t)layer * A.pages * A.heads;
    const auto token_of = [&](int64_t slot, int h) {
        return ((layer_at + (slot >> A.page_bits) * A.heads + h) << A.page_bits) + (slot & (page - 1));
    };
    if (!(blockIdx.z & 1)) {
        Row *k = static_cast<Row *>(A.k) + layer * A.k_layer + t0 * A.k_row + (int64_t)h0 * DIM;
        const int items = min(KV_ROWS, A.T - t0) * hn, c = tid % LANES * VEC;
        for (int i = tid / LANES; i < items; i += KV_THREADS / LANES) {
            const int row = i / hn, h = i - row * hn;
            const int64_t slot = s.slot(row), token = token_of(max(slot, (int64_t)0), h0 + h);
            uint4 out;
            if constexpr (CODED) {
                const uint2 raw = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(A.K) + token * DIM + c);
                out = widen_e4m3(raw.x, raw.y, power_of(A.K_scale[token]));
            } else {
                out = load_raw(static_cast<const W *>(A.K) + token * DIM + c);
            }
            *reinterpret_cast<uint4 *>(k + row * A.k_row + (int64_t)h * DIM + c) = slot < 0 ? make_uint4(0, 0, 0, 0) : out;
        }
        return;
    }
    Row *v = static_cast<Row *>(A.v) + layer * A.v_layer + t0 * A.v_row + (int64_t)h0 * DIM;
    const auto write = [&](int64_t row, int h, const Row (&out)[C]) {
        __builtin_memcpy(__builtin_assume_aligned(v + row * A.v_row + (int64_t)h * DIM + lane * C, sizeof(out)), out, sizeof(out));
    };
    for (int i = wave; i < s.whole * hn; i += KV_WAVES) {
        const int job = i / hn, h = i - job * hn, row = s.rows[job];
        const int64_t token = token_of(s.slot(row), h0 + h);
        Row out[E][C];
        W in[C][E];
        __builtin_memcpy(in, __builtin_assume_aligned(static_cast<const W *>(A.V) + token * DIM + lane * C * E, C * E * sizeof(W) < 16 ? 8 : 16), sizeof(in));
        if constexpr (CODED) {
            uint8_t by[E];
            __builtin_memcpy(by, __builtin_assume_aligned(A.V_scale + token, 8), 8);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                uint32_t raw[2];
                __builtin_memcpy(raw, in[c], 8);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const auto low = __builtin_amdgcn_cvt_pk_f32_fp8(raw[w], false), high = __builtin_amdgcn_cvt_pk_f32_fp8(raw[w], true);
                    const float x[4] = {low[0], low[1], high[0], high[1]};
#pragma unroll
                    for (int t = 0; t < 4; ++t) from_f32(x[t] * power_of(by[4 * w + t]), &out[4 * w + t][c]);
                }
            }
        } else {
#pragma unroll
            for (int t = 0; t < E; ++t)
#pragma unroll
                for (int c = 0; c < C; ++c) out[t][c] = in[c][t];
        }
#pragma unroll
        for (int t = 0; t < E; ++t) write(row + t, h, out[t]);
    }
    for (int i = wave; i < s.alone * hn; i += KV_WAVES) {
        const int job = i / hn, h = i - job * hn, row = s.rows[KV_ROWS - 1 - job];
        const int64_t slot = s.slot(row), token = token_of(max(slot, (int64_t)0), h0 + h);
        const int in_pack = (int)(token & (E - 1));
        const W *from = static_cast<const W *>(A.V) + (token - in_pack) * DIM + in_pack;
        Row out[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const W x = from[(lane * C + c) * E];
            if constexpr (CODED) from_f32(slot < 0 ? 0.f : __builtin_amdgcn_cvt_f32_fp8(x.bits, 0) * power_of(A.V_scale[token]), &out[c]);
            else if (slot < 0) from_f32(0.f, &out[c]);
            else out[c] = x;
        }
        write(row, h, out);
    }
}

}  // namespace svdp
