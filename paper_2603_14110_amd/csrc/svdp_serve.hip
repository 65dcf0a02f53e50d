// C-ABI entry points of a decode step around attention and logits (see include/svdp.h): norms and rotation of heads, tokens from
// logits.  Host-side validation and kernel launches; no allocation, no synchronisation, no state kept between calls.
#include "../../include/svdp.h"

#include <hip/hip_runtime.h>

#include "svdp_host.h"
#include "svdp_rope.h"
#include "svdp_sample.h"

#include <algorithm>
#include <cmath>

namespace {

using namespace svdp;

inline int bytes_of(int dt) { return dt == SVDP_F32 ? 4 : 2; }
inline bool aligned_to(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// T rows of `written` elements, and T rows of `other` elements: whether one of the first has an element in common with one of the second.
// Looked at where both have the same stride.
bool rows_meet(int T, const void *a, int64_t a_stride, int64_t written, const void *b, int64_t b_stride, int64_t other, int bytes)
{
    if (T > 1 && a_stride != b_stride) return false;
    const int64_t by = ((intptr_t)b - (intptr_t)a) / bytes, last = written - 1 - by;         // b's rows are at by + i a_stride of a's, |i| < T
    int64_t i = 0;                                                                           // the largest i that does not lie behind the row
    if (T > 1) i = std::min<int64_t>(last >= 0 ? last / a_stride : -((-last + a_stride - 1) / a_stride), T - 1);
    return i > -T && by + i * a_stride < written && by + i * a_stride > -other;
}
template <SampleWays WAYS>
using Ways = std::integral_constant<SampleWays, WAYS>;
template <bool B>
using Flag = std::integral_constant<bool, B>;
template <typename F>
void on_flag(bool b, F &&f)
{
    if (b) f(Flag<true>{});
    else f(Flag<false>{});
}
template <typename W, int DIM>
void launch_rope(const RopeArgs &A, bool eight, bool inter, bool norm, dim3 grid, hipStream_t hs)
{
    on_flag(inter, [&](auto i) {
        on_flag(norm, [&](auto n) {
            constexpr bool INTER = decltype(i)::value, NORM = decltype(n)::value;
            if constexpr (sizeof(W) == 2)
                if (eight) return launch(k_qk_rope<W, DIM, 8, INTER, NORM>, grid, dim3(ROPE_THREADS), 0, hs, A);
            launch(k_qk_rope<W, DIM, 4, INTER, NORM>, grid, dim3(ROPE_THREADS), 0, hs, A);
        });
    });
}

// Rows of bf16 up to which one launch does all, a block of 1024 threads for each compute unit: 256 of 152 064 logits 33.2 us, in two launches
// 39.4, 256 of 32 000 19.2 and 21.6.  Beyond, blocks of 512 threads that do not carry the other way's registers, and a launch for
// the rows they left: 400 rows 50.0 us, in one launch 51.8; 768 rows 69.9 and 83.4, of 32 000 logits 34.6 and 49.0.
constexpr int SAMPLE_ONE_LAUNCH = 256;
// Heads (of all rows) from which a lane of bf16 has eight pairs, in 16-byte accesses: 16 384 rows of 40 heads 71.0 us, with four pairs
// 74.5; 1024 of them 8.4 and 9.4.  Few heads are bound by the chain of a wave, which four pairs shorten: one row of 64 heads 3.0 us,
// with eight 3.65.  In fp32 four are 16 bytes already (16 384 rows of 6 heads of 64: 12.5 us, with eight 16.9).
constexpr int64_t ROPE_EIGHT = 16384;

}  // namespace

extern "C" {

svdp_status svdp_qk_rope(int32_t dtype, int32_t dim, int32_t T, const void *q, int64_t q_stride, int32_t heads_q, const void *k, int64_t k_stride,
                         int32_t heads, const int32_t *places, const float *inv_freq, int32_t rot, uint32_t flags, const float *q_weight,
                         const float *k_weight, float eps, void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride, void *stream)
{
    if (T < 0 || heads_q < 1 || heads < 0 || rot < 0) return SVDP_ERR_INVALID_ARG;
    if ((flags & ~(uint32_t)(SVDP_ROPE_INTERLEAVED | SVDP_ROPE_NORM | SVDP_ROPE_WEIGHT_EACH)) != 0) return SVDP_ERR_INVALID_ARG;
    if (dtype != SVDP_F32 && dtype != SVDP_BF16) return SVDP_ERR_UNSUPPORTED;
    if ((dim != 64 && dim != 128 && dim != 256) || rot % 8 != 0 || heads_q > 65535 || heads > 65535 || T > SVDP_MAX_ROWS) return SVDP_ERR_UNSUPPORTED;
    if (rot > dim) return SVDP_ERR_INVALID_ARG;
    const bool norm = flags & SVDP_ROPE_NORM;
    if (norm ? !(eps >= 0.f) || !std::isfinite(eps) : q_weight != nullptr || k_weight != nullptr || (flags & SVDP_ROPE_WEIGHT_EACH)) return SVDP_ERR_INVALID_ARG;
    if (T == 0) return SVDP_OK;
    const int vec = 16 / bytes_of(dtype);
    const auto rows_ok = [&](const void *p, int64_t stride, int n) {
        return p != nullptr && aligned16(p) && stride >= (int64_t)n * dim && stride % vec == 0 && stride < (int64_t)1 << 40;
    };
    if (!rows_ok(q, q_stride, heads_q) || !rows_ok(q_out, q_out_stride, heads_q)) return SVDP_ERR_INVALID_ARG;
    if (heads > 0 && (!rows_ok(k, k_stride, heads) || !rows_ok(k_out, k_out_stride, heads))) return SVDP_ERR_INVALID_ARG;
    if ((q == q_out && q_stride != q_out_stride) || (heads > 0 && k == k_out && k_stride != k_out_stride)) return SVDP_ERR_INVALID_ARG;
    const int bytes = bytes_of(dtype);
    const int64_t q_row = (int64_t)heads_q * dim, k_row = (int64_t)heads * dim;
    if (q != q_out && rows_meet(T, q_out, q_out_stride, q_row, q, q_stride, q_row, bytes)) return SVDP_ERR_INVALID_ARG;
    if (heads > 0 && ((k != k_out && rows_meet(T, k_out, k_out_stride, k_row, k, k_stride, k_row, bytes)) ||
                      rows_meet(T, q_out, q_out_stride, q_row, k_out, k_out_stride, k_row, bytes) ||
                      rows_meet(T, q_out, q_out_stride, q_row, k, k_stride, k_row, bytes) || rows_meet(T, k_out, k_out_stride, k_row, q, q_stride, q_row, bytes)))
        return SVDP_ERR_INVALID_ARG;
    if ((rot > 0 && (!places || !inv_freq)) || !aligned_to(places, 4) || !aligned_to(inv_freq, 4) || !aligned16(q_weight) || !aligned16(k_weight))
        return SVDP_ERR_INVALID_ARG;
    RopeArgs A{};
    A.q = q;
    A.k = k;
    A.q_out = q_out;
    A.k_out = k_out;
    A.q_stride = q_stride;
    A.k_stride = k_stride;
    A.q_out_stride = q_out_stride;
    A.k_out_stride = k_out_stride;
    A.places = places;
    A.inv_freq = inv_freq;
    A.q_weight = q_weight;
    A.k_weight = k_weight;
    A.T = T;
    A.heads_q = heads_q;
    A.heads = heads;
    A.half = rot / 2;
    A.q_each = A.k_each = flags & SVDP_ROPE_WEIGHT_EACH ? dim : 0;
    A.eps = eps;
    const bool eight = dtype == SVDP_BF16 && rot % 16 == 0 && (int64_t)T * (heads_q + heads) >= ROPE_EIGHT;
    const int per = (eight ? 1024 : 512) / dim, rounds = (heads_q + heads + per - 1) / per;
    A.each = (int)std::min<int64_t>(rounds, std::max<int64_t>(1, (int64_t)T * rounds / 16384));
    const int64_t waves = (int64_t)T * ((rounds + A.each - 1) / A.each), blocks = (waves + ROPE_WAVES - 1) / ROPE_WAVES;
    if (blocks * ROPE_THREADS >= (int64_t)1 << 32) return SVDP_ERR_UNSUPPORTED;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    const auto of = [&](auto dc) {
        constexpr int DIM = decltype(dc)::value;
        if (dtype == SVDP_F32) launch_rope<float, DIM>(A, eight, flags & SVDP_ROPE_INTERLEAVED, norm, dim3((uint32_t)blocks), hs);
        else launch_rope<bf16, DIM>(A, eight, flags & SVDP_ROPE_INTERLEAVED, norm, dim3((uint32_t)blocks), hs);
    };
    if (dim == 64) of(std::integral_constant<int, 64>{});
    else if (dim == 128) of(std::integral_constant<int, 128>{});
    else of(std::integral_constant<int, 256>{});
    return hip_status(hipSuccess);
}

svdp_status svdp_sample(const void *logits, int64_t stride, int32_t dtype, int32_t V, const float *u, const float *temperature, const int32_t *top_k,
                        const float *top_p, const float *min_p, int32_t T, int32_t *answers, float *logp, void *stream)
{
    static_assert(SAMPLE_MAX_V == SVDP_MAX_VOCABULARY);
    if (T < 0 || V < 1 || (stride != 0 && stride < V)) return SVDP_ERR_INVALID_ARG;
    if (dtype != SVDP_F32 && dtype != SVDP_BF16) return SVDP_ERR_UNSUPPORTED;
    if (T > SVDP_MAX_ROWS || V > SVDP_MAX_VOCABULARY) return SVDP_ERR_UNSUPPORTED;
    if (T == 0) return SVDP_OK;
    if (!logits || !u || !answers || !aligned_to(logits, bytes_of(dtype)) || !aligned_to(u, 4) || !aligned_to(temperature, 4) || !aligned_to(top_k, 4) ||
        !aligned_to(top_p, 4) || !aligned_to(min_p, 4) || !aligned_to(answers, 4) || !aligned_to(logp, 4))
        return SVDP_ERR_INVALID_ARG;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    constexpr int ROWS = 1 << 21;            // of a launch: its threads are counted in 32 bits
    static_assert((int64_t)ROWS * SAMPLE_THREADS < (int64_t)1 << 32);
    // before anything is enqueued (the kernel by value alone needs no grant)
    if (!(dtype == SVDP_F32 ? grant_lds<k_sample<float, SampleWays::ALL>>(sample_lds<float, SampleWays::ALL>())
          : T <= SAMPLE_ONE_LAUNCH ? grant_lds<k_sample<bf16, SampleWays::ALL>>(sample_lds<bf16, SampleWays::ALL>())
                                   : grant_lds<k_sample<bf16, SampleWays::LEFT>>(sample_lds<bf16, SampleWays::LEFT>())))
        return SVDP_ERR_UNSUPPORTED;
    static_assert(sample_lds<bf16, SampleWays::VALUE>() <= LDS_DEFAULT);
    for (int t = 0; t < T; t += ROWS) {
        const auto from = [&](auto *p) { return p != nullptr ? p + t : p; };
        const SampleArgs A{static_cast<const char *>(logits) + (int64_t)t * stride * bytes_of(dtype), stride, from(u), from(temperature), from(top_k),
                           from(top_p), from(min_p), from(answers), from(logp), V};
        const auto with = [&](auto wt, auto ways) {
            using W = decltype(wt);
            constexpr SampleWays WAYS = decltype(ways)::value;
            launch(k_sample<W, WAYS>, dim3(std::min(T - t, ROWS)), dim3(sample_threads<W, WAYS>()), sample_lds<W, WAYS>(), hs, A);
        };
        if (dtype == SVDP_F32) {
            with(float{}, Ways<SampleWays::ALL>{});
        } else if (T <= SAMPLE_ONE_LAUNCH) {
            with(bf16{}, Ways<SampleWays::ALL>{});
        } else {
            with(bf16{}, Ways<SampleWays::VALUE>{});
            with(bf16{}, Ways<SampleWays::LEFT>{});
        }
    }
    return hip_status(hipSuccess);
}

}  // extern "C"
