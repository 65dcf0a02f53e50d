// Norms of the heads of queries and keys, and their rotation by the row's position, in one pass:
//   y = x / sqrt(mean(x^2) + eps) * weight,   (a, b) -> (a cos - b sin, b cos + a sin),   angle = position * inv_freq[i]
// for the pairs (a, b) of the first 2 half channels: i and half + i, or (INTER) 2 i and 2 i + 1.  Channels behind them are not turned.
//
// A head is dim / 2 P lanes with P pairs each, so that both elements of a pair are in a lane, and a wave has 128 P / dim heads of one row at
// a time; its angles are computed once.  An angle is taken in turns in 64 bits, of which the whole ones are dropped: positions of a
// million lose nothing.  All else is fp32, rounded once.
//
// What bounds it: reading and writing.  19 001 rows of 40 heads of 128 in bf16, 389 MB, in 79 us, 4.9 TB/s (a copy of 1 GiB reaches 5.1, rows read
// back from a cache 5.5); one row of 64 heads in 3.2 us, by the latency of position, angles and row.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svdp_device.h"

namespace svdp {

constexpr int ROPE_THREADS = 256, ROPE_WAVES = ROPE_THREADS / 64;

struct RopeArgs {
    const int32_t *places;
    const float *inv_freq;
    const void *q, *k;
    void *q_out, *k_out;
    const float *q_weight, *k_weight;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;
    int T, heads_q, heads, half;
    int q_each, k_each;                     // floats from one head's weights to the next one's
    int each;                               // rounds of a wave (128 P / dim heads each)
    float eps;
};

template <int N, typename W>
__device__ __forceinline__ void load_some(const W *p, float (&x)[N])
{
    W in[N];
    __builtin_memcpy(in, __builtin_assume_aligned(p, sizeof(in) < 16 ? sizeof(in) : 16), sizeof(in));
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = to_f32(in[j]);
}
template <int N, typename W>
__device__ __forceinline__ void store_some(W *p, const float (&x)[N])
{
    W out[N];
#pragma unroll
    for (int j = 0; j < N; ++j) from_f32(x[j], out + j);
    __builtin_memcpy(__builtin_assume_aligned(p, sizeof(out) < 16 ? sizeof(out) : 16), out, sizeof(out));
}

template <typename W, int DIM, int P, bool INTER, bool NORM>
__global__ __launch_bounds__(ROPE_THREADS) void k_qk_rope(RopeArgs A)
{
    constexpr int LANES = DIM / 2 / P, LOG2 = LANES == 4 ? 2 : LANES == 8 ? 3 : LANES == 16 ? 4 : 5, HEADS = 64 / LANES;
    static_assert(LANES == 1 << LOG2);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = A.heads_q + A.heads;
    const int rounds = (heads + HEADS - 1) / HEADS, parts = (rounds + A.each - 1) / A.each;
    const int64_t job = (int64_t)blockIdx.x * ROPE_WAVES + wave;
    const int t = (int)(job / parts);
    if (t >= A.T) return;
    const int h0 = (int)(job - (int64_t)t * parts) * A.each * HEADS, h1 = min(h0 + A.each * HEADS, heads);
    const int i0 = (lane % LANES) * P, rot = 2 * A.half;
    const bool turned = i0 < A.half;
    // the lane's channels: two times P
    const int at0 = !turned ? rot + 2 * (i0 - A.half) : INTER ? 2 * i0 : i0, at1 = turned && !INTER ? A.half + i0 : at0 + P;
    float sin[P], cos[P];
    if (turned) {
        const double place = A.places[t];
        float freq[P];
#pragma unroll
        for (int j = 0; j < P; ++j) freq[j] = A.inv_freq[i0 + j];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const double turns = place * ((double)freq[j] * 0.15915494309189533577);
            sincospif(2.f * (float)(turns - rint(turns)), &sin[j], &cos[j]);
        }
    }
    for (int h = h0; h < h1; h += HEADS) {
        const int mine = h + lane / LANES, head = min(mine, heads - 1), of_k = head >= A.heads_q, local = of_k ? head - A.heads_q : head;
        const W *from = static_cast<const W *>(of_k ? A.k : A.q) + t * (of_k ? A.k_stride : A.q_stride) + (int64_t)local * DIM;
        float x[2][P];
        load_some(from + at0, x[0]);
        load_some(from + at1, x[1]);
        if constexpr (NORM) {
            const float *weight = of_k ? A.k_weight : A.q_weight;
            float square = 0.f;
#pragma unroll
            for (int j = 0; j < P; ++j) square += x[0][j] * x[0][j] + x[1][j] * x[1][j];
            const float by = 1.f / sqrtf(group_sum<LOG2>(square) * (1.f / DIM) + A.eps);
            float w[2][P];
#pragma unroll
            for (int j = 0; j < P; ++j) w[0][j] = w[1][j] = 1.f;
            if (weight != nullptr) {
                weight += (int64_t)local * (of_k ? A.k_each : A.q_each);
                load_some(weight + at0, w[0]);
                load_some(weight + at1, w[1]);
            }
#pragma unroll
            for (int j = 0; j < P; ++j) {
                x[0][j] = x[0][j] * by * w[0][j];
                x[1][j] = x[1][j] * by * w[1][j];
            }
        }
        if (turned) {
            const auto turn = [](float &a, float &b, float c, float s) {
                const float y = a * c - b * s;
                b = b * c + a * s;
                a = y;
            };
            if constexpr (INTER) {
#pragma unroll
                for (int j = 0; j < P / 2; ++j) {
                    turn(x[0][2 * j], x[0][2 * j + 1], cos[j], sin[j]);
                    turn(x[1][2 * j], x[1][2 * j + 1], cos[P / 2 + j], sin[P / 2 + j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < P; ++j) turn(x[0][j], x[1][j], cos[j], sin[j]);
            }
        }
        if (mine >= h1) continue;
        W *to = static_cast<W *>(of_k ? A.k_out : A.q_out) + t * (of_k ? A.k_out_stride : A.q_out_stride) + (int64_t)local * DIM;
        store_some(to + at0, x[0]);
        store_some(to + at1, x[1]);
    }
}

}  // namespace svdp
