// Log probabilities of given experts with log-sum-exp, entropy and the most likely experts of every row, and their gradient.
//
// One pass over a row, in powers of two: the largest logit, then total = sum 2^y and dot = sum 2^y y from the values in registers (y <= 0: relative to the
// largest).  lse = largest / tau + ln 2 log2 total, entropy = ln 2 (log2 total - dot / total) (no cancellation: both terms are >= 0), and the picks' logits
// are read again, from the cache.  It has to read the logits and picks and to write 8 bytes a row, 4 a pick and 8 an alternative: fp32 rows are bound by that
// (2^20 x 256 with 8 picks: 1.15 GB in 207 us, 5.6 TB/s; 2^20 x 64: 61 us), rows of the short types and alternatives by the instructions (2^20 x 256 bf16: 112 us for
// 0.6 GB; with 8 alternatives fp32 226 us for 1.22 GB, bf16 184 for 0.68).  The gradient reads and writes every logit: 2^23 x 8 117 us, 2^20 x 256 348, 6.2 TB/s.
#include "router_core.hpp"

namespace rs {

// How the most likely experts of a row are found: not at all, one round over the row each, or by stage 1's lists of 8 or 16.
enum { ALT_NONE = 0, ALT_ROUNDS = 1, ALT_LISTS_8 = 8, ALT_LISTS_16 = 16 };

template <int LANES>
__device__ __forceinline__ int row_min(int v)
{
    if constexpr (LANES <= 16) v = group_min<LANES>(v);
    else {
        v = group_min<16>(v);
        v = min(v, xlane<16>(v));
        if constexpr (LANES == 64) v = min(v, xlane<32>(v));
    }
    return v;
}

// The m largest logits of the row, one round each: emit(sel, expert, logit) in every lane of the row, INT_MAX once only -infinity is left (and NaN, which is
// never taken).  The winners are taken out of x.
template <int LANES, int VPL, bool VEC, typename F>
__device__ __forceinline__ void row_rounds(float (&x)[VPL], int m, int q, F emit)
{
    for (int sel = 0; sel < m; ++sel) {
        float best = x[0];
#pragma unroll
        for (int j = 1; j < VPL; ++j) best = fmaxf(best, x[j]);
        best = row_max<LANES>(best);
        int slot = VPL;
#pragma unroll
        for (int j = VPL - 1; j >= 0; --j) slot = x[j] == best ? j : slot;
        const int mine = slot < VPL && best > -INFINITY ? slot_index<LANES, VPL, VEC>(q, slot) : INT_MAX;
        const int winner = row_min<LANES>(mine);
        const int gone = winner == mine ? slot : VPL;
#pragma unroll
        for (int j = 0; j < VPL; ++j) x[j] = j == gone ? -INFINITY : x[j];
        emit(sel, winner, best);
    }
}

template <typename T, int LANES, int VPL, bool VEC, int ALT, int L>
__global__ __launch_bounds__(256) void route_logprobs_kernel(const T *__restrict__ logits, int64_t rows, int E, int64_t ld, float inv_tau,
                                                             const uint8_t *__restrict__ row_mask, const int32_t *__restrict__ topk_idx,
                                                             int k, int m, float *__restrict__ logp, float *__restrict__ lse,
                                                             float *__restrict__ entropy, int32_t *__restrict__ alt_idx,
                                                             float *__restrict__ alt_logp)
{
    constexpr int ROWS_PER_BLOCK = 256 / LANES;
    const int q = threadIdx.x % LANES;
    const float c = inv_tau * kLog2e;
    const int64_t first = first_row(ROWS_PER_BLOCK);
    if (first >= rows) return;
    const RowAt at_row = row_at(threadIdx.x / LANES, rows - first, row_mask, first);
    const bool there = at_row.there;
    const int64_t row = first + threadIdx.x / LANES;
    const T *__restrict__ from = row_of(logits + first * ld, at_row.slot, ld);
    const int32_t *__restrict__ ask = topk_idx + first * k + at_row.slot * k;
    int pick = -1;
    if (k > 0) pick = ask[q < k ? q : 0];                // a lane's first pick is fetched with the row, its logit before the row is waited for
    RowRaw<T, VPL, VEC> raw;
    row_fetch<true, T, LANES, VPL, VEC>(from, E, q, raw);
    pick = pick < E ? pick : -1;
    float x[VPL], dot;
    // The lists give experts, not logits: rows of up to 32 KiB a workgroup wait for them in LDS.  By the time they are known the row has left the L2: fetched again,
    // eight alternatives of 2^20 x 256 cost half a GiB of reads on top of one.  The picks of such a kernel are taken from there too.
    constexpr bool keep = ALT >= ALT_LISTS_8 && 256 * VPL * sizeof(T) <= 32768;
    __shared__ __align__(16) T lds[keep ? 256 * VPL : 1];
    T *mine = lds + (keep ? threadIdx.x / LANES * (LANES * VPL) : 0);
    auto kept_at = [&](int at) { return at < (E & ~3) || at >= E ? at : at + (-E & 3); };      // the last values, if they are no whole four, stand at its end
    T picked;
    if constexpr (keep) {
#pragma unroll
        for (int i = 0; i < VPL / 4; ++i) *reinterpret_cast<typename RowRaw<T, VPL, VEC>::four *>(mine + 4 * (q + LANES * i)) = raw.v[i];
        lds_order();
        picked = mine[kept_at(pick < 0 ? 0 : pick)];
    } else {
        picked = from[pick < 0 ? 0 : pick];
    }
    auto kept = [&](int at) { return keep ? mine[kept_at(at)] : from[at < E ? at : 0]; };
    row_take<T, LANES, VPL, VEC>(raw, E, q, x);
    const RowSoft soft = row_sums<LANES, VPL>(x, c, dot);
    const bool counts = at_row.live && soft.total != 0.0f;
    const float log_total = log2_of(soft.total);
    if (there && q == 0) {
        if (lse) lse[row] = counts ? fmaf(soft.largest, inv_tau, kLn2 * log_total) : 0.0f;
        if (entropy) entropy[row] = counts ? kLn2 * (log_total - dot * inverse(soft.total)) : 0.0f;
    }
    if (there && q < k) logp[row * k + q] = counts && pick >= 0 ? kLn2 * (soft.y((float)picked, c) - log_total) : 0.0f;
    if (there) {
        for (int j = q + LANES; j < k; j += LANES) {
            const int at = ask[j];
            const bool good = counts && at >= 0 && at < E;
            logp[row * k + j] = good ? kLn2 * (soft.y((float)from[at], c) - log_total) : 0.0f;
        }
    }
    if constexpr (ALT != ALT_NONE) {
        auto put = [&](int sel, int at, float v) {
            const bool good = counts && at < E && v != -INFINITY;
            alt_idx[row * m + sel] = good ? at : -1;
            alt_logp[row * m + sel] = good ? kLn2 * (soft.y(v, c) - log_total) : counts ? -INFINITY : 0.0f;
        };
        auto each = [&](int sel, int at, float v) {
            if (there && q == sel % LANES) put(sel, at, v);
        };
        if constexpr (ALT == ALT_ROUNDS) {
            row_rounds<LANES, VPL, VEC>(x, m, q, each);
        } else {
            constexpr int KM = ALT;
            constexpr unsigned MASK = (unsigned)(LANES * VPL) - 1u;
            float4 v[VPL / 4];
#pragma unroll
            for (int i = 0; i < VPL / 4; ++i) v[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
            int own[L];
            unsigned bits, u[KM];
            lane_best<LANES, VPL, L, false>(v, E, q, own, bits);
            // a NaN has a place among the keys, above or below all numbers, but none in the order: a row with one (its total is NaN) goes by rounds, as narrow rows do
            const bool bad = row_best<LANES, VPL, L, KM>(own, bits, m, u) || soft.total != soft.total;
            if (__ballot(there && bad) == 0ull) {
#pragma unroll
                for (int r = 0; r < (KM + LANES - 1) / LANES; ++r) {     // alternatives q, q + LANES, ... of this lane
                    unsigned sel = 0;
#pragma unroll
                    for (int j = r * LANES; j < KM && j < (r + 1) * LANES; ++j) sel = j == q + r * LANES ? u[j] : sel;
                    const int at = (int)key_index<MASK>(sel);
                    if (there && q + r * LANES < m) put(q + r * LANES, at, (float)kept(at));
                }
            } else {
                row_rounds<LANES, VPL, VEC>(x, m, q, each);
            }
        }
    }
}

// d_logits[e] = (sum of d_logp over the slots of e - p_e (sum of d_logp - d_lse + d_entropy (log p_e + entropy))) / tau, where log p_e + entropy is
// ln 2 (y_e - sum p y): the logarithm of the total is in both.  The slots' gradients reach the lanes that hold their experts through a row in LDS.
template <typename T, int LANES, int VPL, bool VEC, int NK>
__global__ __launch_bounds__(256) void route_logprobs_backward_kernel(const T *__restrict__ logits, int64_t rows, int E, int64_t ld,
                                                                      float inv_tau, const uint8_t *__restrict__ row_mask,
                                                                      const int32_t *__restrict__ topk_idx, int k,
                                                                      const float *__restrict__ d_logp, const float *__restrict__ d_lse,
                                                                      const float *__restrict__ d_entropy, int add, T *__restrict__ d_logits,
                                                                      int64_t ld_d)
{
    constexpr int ROWS_PER_BLOCK = 256 / LANES;
    __shared__ __align__(16) float lds[ROWS_PER_BLOCK * LANES * VPL];
    const int q = threadIdx.x % LANES;
    float *mine = lds + threadIdx.x / LANES * (LANES * VPL);
    const int64_t first = first_row(ROWS_PER_BLOCK);
    if (first >= rows) return;
    const RowAt at_row = row_at(threadIdx.x / LANES, rows - first, row_mask, first);
    // NK entries a lane at a time; the first ones are asked for before the row, as they are waited for first
    const int64_t entry0 = first * k + at_row.slot * k;
    int at[NK];
    float g[NK];
    auto entries = [&](int j0) {
#pragma unroll
        for (int r = 0; r < NK; ++r) {
            const int j = j0 + q + LANES * r;
            const int64_t entry = entry0 + (j < k ? j : 0);
            at[r] = topk_idx[entry];
            g[r] = d_logp[entry];
        }
    };
    if (d_logp) entries(0);
    const float along = d_lse ? d_lse[first + at_row.slot] : 0.0f;
    const float spread = d_entropy ? kLn2 * d_entropy[first + at_row.slot] : 0.0f;
    RowRaw<T, VPL, VEC> raw;
    row_fetch<false, T, LANES, VPL, VEC>(row_of(logits + first * ld, at_row.slot, ld), E, q, raw);

    float dx[VPL], sum = 0.0f;
#pragma unroll
    for (int j = 0; j < VPL; ++j) dx[j] = 0.0f;
    if (d_logp) {
        for (int j0 = 0; j0 < k; j0 += LANES * NK) {
            bool again[NK];
            float part[VPL];
            if (j0 > 0) entries(j0);
#pragma unroll
            for (int r = 0; r < NK; ++r) {
                const bool good = j0 + q + LANES * r < k && at[r] >= 0 && at[r] < E;
                at[r] = good ? at[r] : -1;
                g[r] = good ? g[r] : 0.0f;
                sum += g[r];
            }
            lds_fill<LANES, VPL, VEC>(mine, q, 0.0f);
            lds_order();
            lds_mark<LANES, NK>(mine, q, k - j0, at, again);
            lds_put<LANES, NK>(mine, q, k - j0, at, again, g);
            lds_values<LANES, VPL, VEC>(mine, q, part);
            lds_order();
#pragma unroll
            for (int j = 0; j < VPL; ++j) dx[j] += part[j];
        }
        sum = row_sum<LANES>(sum);
    }
    float y[VPL], e[VPL];
    row_take<T, LANES, VPL, VEC>(raw, E, q, y);
    const RowSoft soft = row_softmax<LANES, VPL>(y, e, inv_tau * kLog2e);
    const bool counts = at_row.live && soft.total != 0.0f;
    const float scale = inverse(soft.total), pull = sum - along;
    if (d_entropy) {
        // p goes into the difference before d_entropy does: an expert that is out, or nearly, has p (y - mean) small however far y is, where d_entropy (y - mean) may overflow
        const float mean = row_dot<LANES, VPL>(y, e) * scale;
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const float p = e[j] * scale;
            dx[j] -= p * pull + spread * (p * (fmaxf(y[j], -1e30f) - mean));
        }
    } else {
#pragma unroll
        for (int j = 0; j < VPL; ++j) dx[j] -= e[j] * scale * pull;
    }
#pragma unroll
    for (int j = 0; j < VPL; ++j) dx[j] = counts ? dx[j] * inv_tau : 0.0f;
    if (at_row.there && (counts || !add)) row_store<T, LANES, VPL, VEC>(d_logits + (first + threadIdx.x / LANES) * ld_d, E, q, add != 0, dx);
}

template <typename T, int LANES, int VPL, bool VEC, int ALT, int L, typename... A>
static int launch_logprobs(const T *logits, int64_t rows, hipStream_t st, A... rest)
{
    hipLaunchKernelGGL((route_logprobs_kernel<T, LANES, VPL, VEC, ALT, L>), row_grid(rows, 256 / LANES), dim3(256), 0, st, logits, rows, rest...);
    return launch_status();
}
template <typename T, int LANES, int VPL, bool VEC, int NK, typename... A>
static int launch_logprobs_backward(const T *logits, int64_t rows, hipStream_t st, A... rest)
{
    hipLaunchKernelGGL((route_logprobs_backward_kernel<T, LANES, VPL, VEC, NK>), row_grid(rows, 256 / LANES), dim3(256), 0, st, logits, rows, rest...);
    return launch_status();
}

}  // namespace rs

extern "C" int railsched_route_logprobs(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, float temperature,
                                        const uint8_t *row_mask, const int32_t *topk_idx, int32_t k, int32_t m, float *logp, float *lse,
                                        float *entropy, int32_t *alt_idx, float *alt_logp, void *stream)
{
    using namespace rs;
    if (int rc = check_router(logits, dtype, rows, E, ld, temperature)) return rc;
    if (k < 0 || k > E || m < 0 || m > E) return RAILSCHED_ERR_INVALID_ARG;
    if (m > kMaxListed) return RAILSCHED_ERR_UNSUPPORTED;
    if (rows == 0) return RAILSCHED_OK;
    if ((k > 0 && (!topk_idx || !logp)) || (m > 0 && (!alt_idx || !alt_logp))) return RAILSCHED_ERR_NULL_PTR;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return by_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto s, auto alt, auto length) {
            using S = decltype(s);
            return launch_logprobs<T, S::LANES, S::VPL, S::VEC, decltype(alt)::value, decltype(length)::value>(
                static_cast<const T *>(logits), rows, st, E, ld, 1.0f / temperature, row_mask, topk_idx, k, m, logp, lse, entropy, alt_idx, alt_logp);
        };
        // Up to 16 alternatives come from stage 1's lists, in lengths that leave a lane whose whole list is taken as rare: up to eight of rows of more than 32 logits,
        // more of rows of more than 64 (2^20 x 256 with 16: about 700 us by rounds, 302 so).  These kernels are bound by their instructions, most of which a row of
        // fewer lanes shares among more rows: 2^20 x 256 with 8 takes 226 us with 8 lanes, 261 with 16; bf16 184 and 240; but 2^20 x 128 with 4 lanes half as long again
        // as with 8.
        if (E > 32 && m > 0 && m <= 8) {
            constexpr std::integral_constant<int, ALT_LISTS_8> lists;
            if (E <= 64) return go(Shape<4, 16, true>(), lists, std::integral_constant<int, 8>());
            if (E <= 128) return go(Shape<8, 16, true>(), lists, std::integral_constant<int, 6>());
            if (E <= 256) return go(Shape<8, 32, true>(), lists, std::integral_constant<int, 6>());
            if (E <= 512) return go(Shape<16, 32, true>(), lists, std::integral_constant<int, 5>());
            return go(Shape<16, 64, true>(), lists, std::integral_constant<int, 5>());
        }
        if (E > 64 && m > 8 && m <= 16) {
            constexpr std::integral_constant<int, ALT_LISTS_16> lists;
            if (E <= 128) return go(Shape<8, 16, true>(), lists, std::integral_constant<int, 8>());
            if (E <= 256) return go(Shape<8, 32, true>(), lists, std::integral_constant<int, 8>());
            if (E <= 512) return go(Shape<16, 32, true>(), lists, std::integral_constant<int, 7>());
            return go(Shape<16, 64, true>(), lists, std::integral_constant<int, 7>());
        }
        return by_shape<false, T>(E, [&](auto s) {
            if (m > 0) return go(s, std::integral_constant<int, ALT_ROUNDS>(), std::integral_constant<int, 0>());
            return go(s, std::integral_constant<int, ALT_NONE>(), std::integral_constant<int, 0>());
        });
    });
}

extern "C" int railsched_route_logprobs_backward(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, float temperature,
                                                 const uint8_t *row_mask, const int32_t *topk_idx, int32_t k, const float *d_logp,
                                                 const float *d_lse, const float *d_entropy, int32_t accumulate, void *d_logits,
                                                 int64_t ld_d, void *stream)
{
    using namespace rs;
    if (int rc = check_router(logits, dtype, rows, E, ld, temperature)) return rc;
    if (int rc = check_gradient(logits, d_logits, rows, E, ld_d, accumulate)) return rc;
    if (k < 0 || k > E) return RAILSCHED_ERR_INVALID_ARG;
    if (rows == 0) return RAILSCHED_OK;
    if (d_logp && k > 0 && !topk_idx) return RAILSCHED_ERR_NULL_PTR;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return by_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        return by_shape<true, T>(E, [&](auto s) {
            using S = decltype(s);
            return launch_logprobs_backward<T, S::LANES, S::VPL, S::VEC, 1>(static_cast<const T *>(logits), rows, st, E, ld, 1.0f / temperature, row_mask,
                                                                            topk_idx, k, k > 0 ? d_logp : nullptr, d_lse, d_entropy, accumulate,
                                                                            static_cast<T *>(d_logits), ld_d);
        });
    });
}
