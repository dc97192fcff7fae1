// Log probabilities of given experts with log-sum-exp, entropy and the most likely experts of every row, and their gradient.
//
// One pass over a row, in powers of two: the largest logit, then total = sum 2^y and dot = sum 2^y y from the values in registers (y <= 0: relative to the
// largest).  lse = largest / tau + ln 2 log2 total, entropy = ln 2 (log2 total - dot / total) (no cancellation: both terms are >= 0), and the picks' logits
// are read again, from the cache.
#include "router_core.h"

namespace rs {

template <typename T, int LANES, int VPL, bool VEC>
__global__ __launch_bounds__(256) void route_logprobs_kernel(const T *__restrict__ logits, int64_t rows, int E, int64_t ld, float inv_tau,
                                                             const uint8_t *__restrict__ row_mask, const int32_t *__restrict__ topk_idx,
                                                             int k, int m, float *__restrict__ logp, float *__restrict__ lse,
                                                             float *__restrict__ entropy, int32_t *__restrict__ alt_idx,
                                                             float *__restrict__ alt_logp)
{
    constexpr int ROWS_PER_BLOCK = 256 / LANES;
    const int q = threadIdx.x % LANES;
    const int64_t stride = (int64_t)gridDim.x * ROWS_PER_BLOCK;
    for (int64_t w0 = (int64_t)blockIdx.x * ROWS_PER_BLOCK; w0 < rows; w0 += stride) {          // the same for every lane
        const int64_t row = w0 + threadIdx.x / LANES;
        const bool there = row < rows;
        const bool live = there && (!row_mask || row_mask[row] != 0);
        const T *__restrict__ from = logits + row * ld;
        float raw[VPL], y[VPL], e[VPL];
        row_values<T, LANES, VPL, VEC>(from, live, E, q, raw);
#pragma unroll
        for (int j = 0; j < VPL; ++j) y[j] = raw[j];
        const float c = inv_tau * kLog2e;
        const RowSoft soft = row_softmax<LANES, VPL>(y, e, c);
        const float dot = row_dot<LANES, VPL>(y, e);
        const bool counts = soft.total != 0.0f;
        const float log_total = log2_of(soft.total);
        if (there && q == 0) {
            if (lse) lse[row] = counts ? fmaf(soft.largest, inv_tau, kLn2 * log_total) : 0.0f;
            if (entropy) entropy[row] = counts ? kLn2 * (log_total - dot * inverse(soft.total)) : 0.0f;
        }
        if (there) {
            for (int j = q; j < k; j += LANES) {
                const int at = topk_idx[row * k + j];
                const bool good = counts && at >= 0 && at < E;
                logp[row * k + j] = good ? kLn2 * (soft.y((float)from[at], c) - log_total) : 0.0f;
            }
        }
        for (int sel = 0; sel < m; ++sel) {
            float best = -INFINITY;
            int at = INT_MAX;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                const bool better = raw[j] > best;
                best = better ? raw[j] : best;
                at = better ? slot_index<LANES, VPL, VEC>(q, j) : at;
            }
            group_argmax<LANES>(best, at);
#pragma unroll
            for (int j = 0; j < VPL; ++j) raw[j] = slot_index<LANES, VPL, VEC>(q, j) == at ? -INFINITY : raw[j];
            if (there && q == sel % LANES) {
                alt_idx[row * m + sel] = at < E ? at : -1;
                alt_logp[row * m + sel] = !counts ? 0.0f : at < E ? kLn2 * (soft.y(best, c) - log_total) : -INFINITY;
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
    const int64_t stride = (int64_t)gridDim.x * ROWS_PER_BLOCK;
    for (int64_t w0 = (int64_t)blockIdx.x * ROWS_PER_BLOCK; w0 < rows; w0 += stride) {
        const int64_t row = w0 + threadIdx.x / LANES;
        const bool there = row < rows;
        const bool live = there && (!row_mask || row_mask[row] != 0);
        float y[VPL], e[VPL];
        row_values<T, LANES, VPL, VEC>(logits + row * ld, live, E, q, y);
        const RowSoft soft = row_softmax<LANES, VPL>(y, e, inv_tau * kLog2e);
        const bool counts = soft.total != 0.0f;

        float dx[VPL], sum = 0.0f;
#pragma unroll
        for (int j = 0; j < VPL; ++j) dx[j] = 0.0f;
        if (d_logp) {
            for (int first = 0; first < k; first += LANES * NK) {            // NK entries a lane at a time
                int at[NK];
                bool again[NK];
                float g[NK], part[VPL];
#pragma unroll
                for (int r = 0; r < NK; ++r) {
                    const int j = first + q + LANES * r;
                    at[r] = live && j < k ? topk_idx[row * k + j] : -1;
                    if (at[r] >= E) at[r] = -1;
                    g[r] = at[r] >= 0 ? d_logp[row * k + j] : 0.0f;
                    sum += g[r];
                }
                lds_fill<LANES, VPL, VEC>(mine, q, 0.0f);
                lds_order();
                lds_mark<LANES, NK>(mine, q, k - first, at, again);
                lds_put<LANES, NK>(mine, q, k - first, at, again, g);
                lds_values<LANES, VPL, VEC>(mine, q, part);
                lds_order();
#pragma unroll
                for (int j = 0; j < VPL; ++j) dx[j] += part[j];
            }
            sum = row_sum<LANES>(sum);
        }
        const float pull = sum - (d_lse && live ? d_lse[row] : 0.0f);
        const float scale = inverse(soft.total);
        if (d_entropy) {
            const float mean = row_dot<LANES, VPL>(y, e) * scale;
            const float gh = live ? kLn2 * d_entropy[row] : 0.0f;
#pragma unroll
            for (int j = 0; j < VPL; ++j) dx[j] -= e[j] * scale * (pull + gh * (fmaxf(y[j], -1e30f) - mean));
        } else {
#pragma unroll
            for (int j = 0; j < VPL; ++j) dx[j] -= e[j] * scale * pull;
        }
#pragma unroll
        for (int j = 0; j < VPL; ++j) dx[j] = counts ? dx[j] * inv_tau : 0.0f;
        if (there && (counts || !add)) row_store<T, LANES, VPL, VEC>(d_logits + row * ld_d, E, q, add != 0, dx);
    }
}

template <typename T, int LANES, int VPL, bool VEC, typename... A>
static int launch_logprobs(const T *logits, int64_t rows, hipStream_t st, A... rest)
{
    const int64_t blocks = (rows + 256 / LANES - 1) / (256 / LANES);
    hipLaunchKernelGGL((route_logprobs_kernel<T, LANES, VPL, VEC>), dim3((unsigned)(blocks < (1 << 22) ? blocks : 1 << 22)), dim3(256), 0, st, logits, rows,
                       rest...);
    return launch_status();
}
template <typename T, int LANES, int VPL, bool VEC, int NK, typename... A>
static int launch_logprobs_backward(const T *logits, int64_t rows, hipStream_t st, A... rest)
{
    const int64_t blocks = (rows + 256 / LANES - 1) / (256 / LANES);
    hipLaunchKernelGGL((route_logprobs_backward_kernel<T, LANES, VPL, VEC, NK>), dim3((unsigned)(blocks < (1 << 22) ? blocks : 1 << 22)), dim3(256), 0, st,
                       logits, rows, rest...);
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
        return by_shape(E, in_fours<T>(logits, E, ld), [&](auto s) {
            using S = decltype(s);
            return launch_logprobs<T, S::LANES, S::VPL, S::VEC>(static_cast<const T *>(logits), rows, st, E, ld, 1.0f / temperature, row_mask, topk_idx, k,
                                                                m, logp, lse, entropy, alt_idx, alt_logp);
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
        return by_shape(E, in_fours<T>(logits, E, ld) && in_fours<T>(d_logits, E, ld_d), [&](auto s) {
            using S = decltype(s);
            return launch_logprobs_backward<T, S::LANES, S::VPL, S::VEC, 1>(static_cast<const T *>(logits), rows, st, E, ld, 1.0f / temperature, row_mask,
                                                                            topk_idx, k, k > 0 ? d_logp : nullptr, d_lse, d_entropy, accumulate,
                                                                            static_cast<T *>(d_logits), ld_d);
        });
    });
}
