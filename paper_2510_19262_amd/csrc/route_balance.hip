// Balance loss of groups of rows with the counts of picks per expert, and its gradient.
//
// The rows are cut into slices, a workgroup each.  A slice holds parts of one or several groups; for each part the workgroup adds up the
// probabilities of its rows (fp32, a lane its own experts) and counts its picks (LDS), and writes one record.  Slices and groups are both in
// row order, so the part of group g in slice s can take the record s + g: no two parts share it.  A second kernel adds the records of a group up
// in their order (fp64) and forms the loss.  No floating-point atomics: equal inputs give equal bits.
#include "router_core.h"

namespace rs {

// rows of group g, kept within [0, rows]
struct Groups {
    const int64_t *off;     // NULL: equal parts of `each` rows
    int64_t each, rows;
    int n;
    __device__ __forceinline__ int64_t begin(int g) const
    {
        const int64_t b = off ? off[g] : g * each;
        return b < 0 ? 0 : b < rows ? b : rows;
    }
    // the first group that can hold a row >= r; by all lanes of a wavefront
    __device__ __forceinline__ int first(int64_t r) const
    {
        if (!off) return (int)(r / each);
        return off[0] > r ? 0 : wave_last_le(off, n, r);
    }
};

struct Record {             // of a part: E sums, E counts, the rows that count
    static __host__ __device__ int64_t words(int E) { return 2 * (int64_t)E + 1; }
};

template <typename T, int LANES, int VPL, bool VEC>
__global__ __launch_bounds__(256) void route_balance_kernel(const T *__restrict__ logits, int E, int64_t ld, const uint8_t *__restrict__ row_mask,
                                                            const int32_t *__restrict__ topk_idx, int k, Groups groups, int64_t slice_rows,
                                                            float *__restrict__ records)
{
    constexpr int ROWS_PER_BLOCK = 256 / LANES;
    __shared__ __align__(16) float sums[ROWS_PER_BLOCK * LANES * VPL];
    __shared__ unsigned picks[kMaxExperts];
    __shared__ unsigned counted;
    const int q = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int64_t r0 = blockIdx.x * slice_rows;
    const int64_t r1 = r0 + slice_rows < groups.rows ? r0 + slice_rows : groups.rows;
    for (int g = groups.first(r0); g < groups.n; ++g) {
        const int64_t gb = groups.begin(g), ge = groups.begin(g + 1);
        if (gb >= r1) break;
        const int64_t lo = gb > r0 ? gb : r0, hi = ge < r1 ? ge : r1;
        if (lo >= hi) continue;
        for (int i = threadIdx.x; i < E; i += 256) picks[i] = 0;
        if (threadIdx.x == 0) counted = 0;
        __syncthreads();
        float acc[VPL];
#pragma unroll
        for (int j = 0; j < VPL; ++j) acc[j] = 0.0f;
        unsigned here = 0;
        for (int64_t w0 = lo; w0 < hi; w0 += ROWS_PER_BLOCK) {
            const int64_t row = w0 + slot;
            const bool live = row < hi && (!row_mask || row_mask[row] != 0);
            float t[VPL], e[VPL];
            row_values<T, LANES, VPL, VEC>(logits + row * ld, live, E, q, t);
            const RowSoft soft = row_softmax<LANES, VPL>(t, e, kLog2e);
            if (soft.total != 0.0f) {
                const float scale = 1.0f / soft.total;
#pragma unroll
                for (int j = 0; j < VPL; ++j) acc[j] += e[j] * scale;
                here += q == 0;
                for (int j = q; j < k; j += LANES) {
                    const int at = topk_idx[row * k + j];
                    if (at >= 0 && at < E) atomicAdd(&picks[at], 1u);
                }
            }
        }
        if (here) atomicAdd(&counted, here);
#pragma unroll
        for (int j = 0; j < VPL; ++j) sums[slot * (LANES * VPL) + slot_index<LANES, VPL, VEC>(q, j)] = acc[j];
        __syncthreads();
        float *rec = records + (blockIdx.x + (int64_t)g) * Record::words(E);
        for (int i = threadIdx.x; i < E; i += 256) {
            float s = 0.0f;
            for (int r = 0; r < ROWS_PER_BLOCK; ++r) s += sums[r * (LANES * VPL) + i];
            rec[i] = s;
            reinterpret_cast<unsigned *>(rec)[E + i] = picks[i];
        }
        if (threadIdx.x == 0) reinterpret_cast<unsigned *>(rec)[2 * E] = counted;
        __syncthreads();
    }
}

__global__ __launch_bounds__(256) void route_balance_join_kernel(const float *__restrict__ records, int E, int k, Groups groups, int64_t slice_rows,
                                                                 float coef, int64_t *__restrict__ counts, int64_t *__restrict__ tokens,
                                                                 float *__restrict__ prob_sum, float *__restrict__ loss)
{
    __shared__ double part[256];
    const int g = blockIdx.x;
    const int64_t gb = groups.begin(g), ge = groups.begin(g + 1);
    const int64_t s0 = gb / slice_rows, s1 = gb < ge ? (ge - 1) / slice_rows + 1 : s0;
    const int64_t words = Record::words(E);
    double dot = 0.0;
    for (int i = threadIdx.x; i < E; i += 256) {
        double s = 0.0;
        int64_t c = 0;
        for (int64_t r = s0; r < s1; ++r) {
            const float *rec = records + (r + g) * words;
            s += rec[i];
            c += reinterpret_cast<const unsigned *>(rec)[E + i];
        }
        prob_sum[(int64_t)g * E + i] = (float)s;
        counts[(int64_t)g * E + i] = c;
        dot += s * (double)c;
    }
    part[threadIdx.x] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
        double sum = 0.0;
        for (int i = 0; i < 256; ++i) sum += part[i];
        int64_t n = 0;
        for (int64_t r = s0; r < s1; ++r) n += reinterpret_cast<const unsigned *>(records + (r + g) * words)[2 * E];
        tokens[g] = n;
        loss[g] = n ? (float)((double)coef * E / ((double)k * n * n) * sum) : 0.0f;
    }
}

// d_logits[e] = p_e (a_e - sum_f a_f p_f), a_e = d_loss coef E c_e / (k n^2).  The gradient does not change with a constant added to a: the mean
// count is taken off first (fp64), so that nothing is lost where the counts are nearly equal.
template <typename T, int LANES, int VPL, bool VEC>
__global__ __launch_bounds__(256) void route_balance_backward_kernel(const T *__restrict__ logits, int E, int64_t ld,
                                                                     const uint8_t *__restrict__ row_mask, int k, Groups groups,
                                                                     int64_t slice_rows, float coef, const int64_t *__restrict__ counts,
                                                                     const int64_t *__restrict__ tokens, const float *__restrict__ d_loss,
                                                                     int add, T *__restrict__ d_logits, int64_t ld_d)
{
    constexpr int ROWS_PER_BLOCK = 256 / LANES;
    __shared__ double part[256];
    __shared__ float weight[kMaxExperts];
    const int q = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int64_t r0 = blockIdx.x * slice_rows;
    const int64_t r1 = r0 + slice_rows < groups.rows ? r0 + slice_rows : groups.rows;
    for (int g = groups.first(r0); g < groups.n; ++g) {
        const int64_t gb = groups.begin(g), ge = groups.begin(g + 1);
        if (gb >= r1) break;
        const int64_t lo = gb > r0 ? gb : r0, hi = ge < r1 ? ge : r1;
        if (lo >= hi) continue;
        const int64_t *__restrict__ c = counts + (int64_t)g * E;
        double sum = 0.0;
        for (int i = threadIdx.x; i < E; i += 256) sum += (double)c[i];
        part[threadIdx.x] = sum;
        __syncthreads();
#pragma unroll
        for (int w = 128; w >= 1; w /= 2) {
            if (threadIdx.x < w) part[threadIdx.x] += part[threadIdx.x + w];
            __syncthreads();
        }
        const double mean = part[0] / E, n = (double)tokens[g];
        const double unit = n > 0.0 ? (double)d_loss[g] * coef * E / ((double)k * n * n) : 0.0;
        for (int i = threadIdx.x; i < E; i += 256) weight[i] = (float)(unit * ((double)c[i] - mean));
        __syncthreads();
        float a[VPL];
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int i = slot_index<LANES, VPL, VEC>(q, j);
            a[j] = i < E ? weight[i] : 0.0f;
        }
        for (int64_t w0 = lo; w0 < hi; w0 += ROWS_PER_BLOCK) {
            const int64_t row = w0 + slot;
            const bool there = row < hi;
            const bool live = there && (!row_mask || row_mask[row] != 0);
            float t[VPL], e[VPL];
            row_values<T, LANES, VPL, VEC>(logits + row * ld, live, E, q, t);
            const RowSoft soft = row_softmax<LANES, VPL>(t, e, kLog2e);
            const bool counts_here = soft.total != 0.0f;
            const float scale = 1.0f / soft.total;
            float ap = 0.0f;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                e[j] *= scale;
                ap += a[j] * e[j];
            }
            ap = row_sum<LANES>(ap);
#pragma unroll
            for (int j = 0; j < VPL; ++j) t[j] = counts_here ? e[j] * (a[j] - ap) : 0.0f;
            if (there && (counts_here || !add)) row_store<T, LANES, VPL, VEC>(d_logits + row * ld_d, E, q, add != 0, t);
        }
        __syncthreads();
    }
}

// rows of a slice: 2048 slices fill the GPU eight workgroups to a CU; no fewer than the rows that a workgroup has in hand at once, nor than 64, so that
// the records stay few against the logits
static int64_t balance_slice_rows(int64_t rows, int E)
{
    const int64_t r = (rows + 2047) / 2048, least = E <= 8 ? 128 : 64;
    return r > least ? r : least;
}
static int64_t balance_slices(int64_t rows, int E) { return (rows + balance_slice_rows(rows, E) - 1) / balance_slice_rows(rows, E); }

static int check_groups(int64_t rows, const int64_t *group_off, int32_t groups)
{
    if (groups < 0 || (!group_off && (groups == 0 ? rows != 0 : rows % groups != 0))) return RAILSCHED_ERR_INVALID_ARG;
    return RAILSCHED_OK;
}
static Groups make_groups(int64_t rows, const int64_t *group_off, int32_t groups)
{
    Groups g;
    g.off = group_off;
    g.each = groups > 0 && rows / groups > 0 ? rows / groups : 1;
    g.rows = rows;
    g.n = groups;
    return g;
}

}  // namespace rs

extern "C" size_t railsched_route_balance_workspace_bytes(int64_t rows, int32_t groups, int32_t E)
{
    using namespace rs;
    if (rows < 0 || rows > 0x7FFFFFFFll || groups < 0 || E < 1 || E > kMaxExperts) return 0;
    return align_up((size_t)(balance_slices(rows, E) + groups + 1) * Record::words(E) * sizeof(float), 256);
}

extern "C" int railsched_route_balance(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, const uint8_t *row_mask,
                                       const int32_t *topk_idx, int32_t k, const int64_t *group_off, int32_t groups, float coef,
                                       int64_t *counts, int64_t *tokens, float *prob_sum, float *loss, void *ws, size_t ws_bytes,
                                       void *stream)
{
    using namespace rs;
    if (int rc = check_router(logits, dtype, rows, E, ld, 1.0f)) return rc;
    if (k < 1 || k > E) return RAILSCHED_ERR_INVALID_ARG;
    if (int rc = check_groups(rows, group_off, groups)) return rc;
    if (groups == 0) return RAILSCHED_OK;
    if ((rows > 0 && !topk_idx) || !counts || !tokens || !prob_sum || !loss) return RAILSCHED_ERR_NULL_PTR;
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 != 0 || ws_bytes < railsched_route_balance_workspace_bytes(rows, groups, E)) return RAILSCHED_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const Groups gr = make_groups(rows, group_off, groups);
    const int64_t slice_rows = balance_slice_rows(rows, E);
    float *records = static_cast<float *>(ws);
    if (rows > 0) {
        const int rc = by_dtype(dtype, [&](auto t) {
            using T = decltype(t);
            return by_shape(E, in_fours<T>(logits, E, ld), [&](auto s) {
                using S = decltype(s);
                hipLaunchKernelGGL((route_balance_kernel<T, S::LANES, S::VPL, S::VEC>), dim3((unsigned)balance_slices(rows, E)), dim3(256), 0, st,
                                   static_cast<const T *>(logits), E, ld, row_mask, topk_idx, k, gr, slice_rows, records);
                return launch_status();
            });
        });
        if (rc) return rc;
    }
    hipLaunchKernelGGL(route_balance_join_kernel, dim3((unsigned)groups), dim3(256), 0, st, records, E, k, gr, slice_rows, coef, counts, tokens, prob_sum,
                       loss);
    return launch_status();
}

extern "C" int railsched_route_balance_backward(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, const uint8_t *row_mask,
                                                int32_t k, const int64_t *group_off, int32_t groups, float coef, const int64_t *counts,
                                                const int64_t *tokens, const float *d_loss, int32_t accumulate, void *d_logits,
                                                int64_t ld_d, void *stream)
{
    using namespace rs;
    if (int rc = check_router(logits, dtype, rows, E, ld, 1.0f)) return rc;
    if (int rc = check_gradient(logits, d_logits, rows, E, ld_d, accumulate)) return rc;
    if (k < 1 || k > E) return RAILSCHED_ERR_INVALID_ARG;
    if (int rc = check_groups(rows, group_off, groups)) return rc;
    if (groups == 0 || rows == 0) return RAILSCHED_OK;
    if (!counts || !tokens || !d_loss) return RAILSCHED_ERR_NULL_PTR;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const Groups gr = make_groups(rows, group_off, groups);
    return by_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        return by_shape(E, in_fours<T>(logits, E, ld) && in_fours<T>(d_logits, E, ld_d), [&](auto s) {
            using S = decltype(s);
            hipLaunchKernelGGL((route_balance_backward_kernel<T, S::LANES, S::VPL, S::VEC>), dim3((unsigned)balance_slices(rows, E)), dim3(256), 0, st,
                               static_cast<const T *>(logits), E, ld, row_mask, k, gr, balance_slice_rows(rows, E), coef, counts, tokens, d_loss,
                               accumulate, static_cast<T *>(d_logits), ld_d);
            return launch_status();
        });
    });
}
