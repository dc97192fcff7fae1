// Distillation of a router from the top logits of a teacher, and its gradient.
//
// Per row: the student's softmax from one read of its logits; the teacher's entries, one to a lane, their probabilities q, and the row in LDS
// that marks the listed experts, so that the student's probability outside the list is a sum of its own terms (1 minus the listed ones would lose
// it where the list holds nearly everything).
//
// The loss is formed as  sum_j (q log(q/p) - q + p) + rest + (sum of q and p outside these terms):  every term is >= 0 and of second order where
// p is near q, where sum q (log q - log p) would be a difference of larger terms.  With d = log p - log q:  q log(q/p) - q + p = q (e^d - 1 - d), so that an error of
// d, a few 2^-24 of 1 + |logit - t_logit| / tau, costs |p - q| times that.
//
// The loss reads the logits and 8 bytes an entry: bound by the instructions where the logits are short (2^20 x 64 bf16 with 6 entries: 41 us for 0.19 GB, 390 vector
// instructions for 16 rows), nearly by the reads where they are not (2^20 x 256 fp32: 179 us for 1.15 GB).  Lists of more than two entries a lane take
// registers: with 16 entries a lane 86 scalar ones are spilled and 4 wavefronts a SIMD are left of 8 (800393 x 64 fp16 with 32 entries: 138 us for 0.31 GB).  The gradient reads and writes every logit: 2^20 x 256 with 8 entries
// and the tail 369 us, 6.0 TB/s.
#include "router_core.hpp"

namespace rs {

// e^a for a few values, a <= 0 or near it: the product with log2 e is carried on to a second float, as its rounding alone is 2^-24 |a| of the result.  low is what fl(a fl(log2 e)) leaves,
// and a times what log2 e has behind its fp32 value
__device__ __forceinline__ float exp_of(float a)
{
    const float y = a * kLog2e, low = fmaf(a, 0x1.4ae0c0p-26f, fmaf(a, kLog2e, -y));
    return pow2(y) * (fabsf(low) < 1.0f ? fmaf(low, kLn2, 1.0f) : 1.0f);      // NaN where a is infinite
}
// a - log v of a normal v = m 2^k: k log 2 goes off in two parts, the first of them without rounding, as its sum with log m would be rounded at k.  The first part is log 2 to nine bits, whose
// product with an exponent of at most eight is exact, the second the rest of log 2 (the splitting of Cody and Waite, Software Manual for the Elementary Functions, 1980)
__device__ __forceinline__ float less_log(float a, float v)
{
    const float k = (float)__builtin_amdgcn_frexp_expf(v), m = __builtin_amdgcn_frexp_mantf(v);
    return fmaf(k, -0x1.63p-1f, a) - fmaf(k, -0x1.bd0106p-13f, kLn2 * log2_of(m));
}
// e^d - 1 - d: a series near 0, where the difference cancels.  |d| < 1/2: d^2/2 (1 + d/3 (1 + d/4 (... (1 + d/10)))), next term below 2^-27 of it
__device__ __forceinline__ float exp_above(float d)
{
    float s = fmaf(d, 1.0f / 10, 1.0f);
    s = fmaf(d * (1.0f / 9), s, 1.0f);
    s = fmaf(d * (1.0f / 8), s, 1.0f);
    s = fmaf(d * (1.0f / 7), s, 1.0f);
    s = fmaf(d * (1.0f / 6), s, 1.0f);
    s = fmaf(d * (1.0f / 5), s, 1.0f);
    s = fmaf(d * (1.0f / 4), s, 1.0f);
    s = fmaf(d * (1.0f / 3), s, 1.0f);
    s *= 0.5f * d * d;
    return fabsf(d) < 0.5f ? s : pow2(d * kLog2e) - 1.0f - d;
}
// x - log(1 + x), x > -1, the same way: with w = x / (2 + x), log(1 + x) = 2 (w + w^3/3 + w^5/5 + ...) and x - 2 w = x w.  |x| < 1/2: w^2 < 1/9, next
// term below 2^-26 of it.  Further off 1 + x is given, as x near -1 has lost it.
__device__ __forceinline__ float above_log(float x, float one_more)
{
    const float w = x * inverse(2.0f + x), v = w * w;
    float s = fmaf(v, 1.0f / 15, 1.0f / 13);
    s = fmaf(v, s, 1.0f / 11);
    s = fmaf(v, s, 1.0f / 9);
    s = fmaf(v, s, 1.0f / 7);
    s = fmaf(v, s, 1.0f / 5);
    s = fmaf(v, s, 1.0f / 3);
    return fabsf(x) < 0.5f ? w * (x - 2.0f * v * s) : x - kLn2 * log2_of(one_more);
}

// What both passes need of a row.
template <int LANES, int VPL, int NK>
struct Distilled {
    float y[VPL], e[VPL];        // the student: y, 2^y
    RowSoft soft;
    int at[NK];                  // this lane's entries: expert or -1
    bool again[NK];              // an entry whose expert another entry of the list names too
    float q[NK], p[NK];          // the teacher's and the student's probability
    float d[NK];                 // log p - log q
    float less[NK];              // for the gradient: q - p as q (1 - e^d), which does not cancel where p is near q; q alone where p is another entry's
    float mass;                  // sum of q (1 without t_lse)
    float gap;                   // sum of q - p over the entries (p of every expert once): with a tail p_r - q_r
    float rest_q, rest_p;
    bool listed;                 // whether the row has entries at all
};

// The row `at_row` of the rows from `first` on.
template <bool GRAD, typename T, int LANES, int VPL, bool VEC, int NK>
__device__ __forceinline__ void distill_row(const T *__restrict__ logits, int64_t first, const RowAt &at_row, int E, int64_t ld, float inv_tau,
                                            const int32_t *__restrict__ t_idx, const float *__restrict__ t_logit,
                                            const float *__restrict__ t_lse, int K, int q0, float *mine, Distilled<LANES, VPL, NK> &o)
{
    const T *__restrict__ from = row_of(logits + first * ld, at_row.slot, ld);
    const int entry0 = at_row.slot * K;
    t_idx += first * K;
    t_logit += first * K;
    // Everything is asked for before anything is waited for: the entries first, whose experts' logits are the next thing to ask for.  Entries that no lane
    // has cost nothing: the condition is the same for every lane, and there is none where one or two entries a lane are all there are.
    auto has = [&](int r) { return NK <= 2 || LANES * r < K; };
    int at[NK];
    float tl[NK];
#pragma unroll
    for (int r = 0; r < NK; ++r) {
        at[r] = -1;
        tl[r] = -INFINITY;
        if (has(r)) {
            const int j = q0 + LANES * r;
            at[r] = t_idx[entry0 + (j < K ? j : 0)];
            tl[r] = t_logit[entry0 + (j < K ? j : 0)];
        }
    }
    const float teacher = t_lse ? t_lse[first + at_row.slot] : 0.0f;
    RowRaw<T, VPL, VEC> raw;
    row_fetch<true, T, LANES, VPL, VEC>(from, E, q0, raw);
    T listed[NK];
    float best = -INFINITY;
    bool any = false;
#pragma unroll
    for (int r = 0; r < NK; ++r) {
        const bool good = q0 + LANES * r < K && at[r] >= 0 && at[r] < E && tl[r] != -INFINITY;
        o.at[r] = good ? at[r] : -1;
        tl[r] = good ? tl[r] : -INFINITY;
        listed[r] = T(0.0f);
        if (has(r)) listed[r] = from[good ? at[r] : 0];
        best = fmaxf(best, tl[r]);
        any |= good;
    }
    o.listed = row_any<LANES>(any);
    lds_fill<LANES, VPL, VEC>(mine, q0, -INFINITY);
    lds_order();
    lds_mark<LANES, NK>(mine, q0, K, o.at, o.again);
    const float c = inv_tau * kLog2e;
    row_take<T, LANES, VPL, VEC>(raw, E, q0, o.y);
    o.soft = row_softmax<LANES, VPL>(o.y, o.e, c);
    const float scale = inverse(o.soft.total);
    // q, and the teacher's log total mass less the student's
    float shift;
    if (t_lse) {
        shift = less_log(fmaf(-o.soft.largest, inv_tau, teacher), o.soft.total);
#pragma unroll
        for (int r = 0; r < NK; ++r) o.q[r] = has(r) && o.at[r] >= 0 ? exp_of(fmaf(tl[r], inv_tau, -teacher)) : 0.0f;
    } else {
        best = row_max<LANES>(best);
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < NK; ++r) {
            o.q[r] = has(r) && o.at[r] >= 0 ? pow2(c * (tl[r] - best)) : 0.0f;
            s += o.q[r];
        }
        s = row_sum<LANES>(s);
        const float share = inverse(s);
        shift = fmaf(best - o.soft.largest, inv_tau, kLn2 * log2_of(s * scale));
#pragma unroll
        for (int r = 0; r < NK; ++r) o.q[r] = has(r) && o.at[r] >= 0 ? o.q[r] * share : 0.0f;
    }
    float mass = 0.0f, gap = 0.0f;
#pragma unroll
    for (int r = 0; r < NK; ++r) {
        o.p[r] = o.d[r] = o.less[r] = 0.0f;
        if (has(r)) {
            const float x = (float)listed[r];
            o.p[r] = o.at[r] >= 0 ? pow2(o.soft.y(x, c)) * scale : 0.0f;
            o.d[r] = fmaf(x - tl[r], inv_tau, shift);
            mass += o.q[r];
            float less = o.q[r] - (o.again[r] ? 0.0f : o.p[r]);
            if (GRAD) {
                if (!o.again[r] && fabsf(o.d[r]) < 0.5f) less = -o.q[r] * (exp_above(o.d[r]) + o.d[r]);
                o.less[r] = less;
            }
            gap += less;
        }
    }
    o.mass = t_lse ? row_sum<LANES>(mass) : 1.0f;
    o.gap = t_lse ? row_sum<LANES>(gap) : 0.0f;
    float marks[VPL], outside = 0.0f;
    lds_values<LANES, VPL, VEC>(mine, q0, marks);
#pragma unroll
    for (int j = 0; j < VPL; ++j) outside += marks[j] < 0.0f ? o.e[j] : 0.0f;
    o.rest_p = row_sum<LANES>(outside) * scale;
    o.rest_q = t_lse && o.rest_p >= 0x1p-126f ? fmaxf(1.0f - o.mass, 0.0f) : 0.0f;
}

template <typename T, int LANES, int VPL, bool VEC, int NK>
__global__ __launch_bounds__(256) void route_distill_kernel(const T *__restrict__ logits, int64_t rows, int E, int64_t ld, float tau, float inv_tau,
                                                            const uint8_t *__restrict__ row_mask, const int32_t *__restrict__ t_idx,
                                                            const float *__restrict__ t_logit, const float *__restrict__ t_lse, int K,
                                                            float *__restrict__ loss)
{
    constexpr int ROWS_PER_BLOCK = 256 / LANES;
    __shared__ __align__(16) float lds[ROWS_PER_BLOCK * LANES * VPL];
    const int q0 = threadIdx.x % LANES;
    float *mine = lds + threadIdx.x / LANES * (LANES * VPL);
    const int64_t first = first_row(ROWS_PER_BLOCK);
    if (first >= rows) return;
    const RowAt at_row = row_at(threadIdx.x / LANES, rows - first, row_mask, first);
    Distilled<LANES, VPL, NK> o;
    distill_row<false, T, LANES, VPL, VEC, NK>(logits, first, at_row, E, ld, inv_tau, t_idx, t_logit, t_lse, K, q0, mine, o);
    float terms = 0.0f, twice = 0.0f;
#pragma unroll
    for (int r = 0; r < NK; ++r) {
        if (o.at[r] >= 0) {
            // q (e^d - 1 - d) where e^d does not carry it off, and p alone where q has vanished
            terms += o.q[r] == 0.0f ? o.p[r] : o.d[r] < 1.0f ? o.q[r] * exp_above(o.d[r]) : o.p[r] - o.q[r] - o.q[r] * o.d[r];
            if (o.again[r]) twice += o.p[r];
        }
    }
    terms = row_sum<LANES>(terms);
    if (__ballot(twice != 0.0f) != 0ull) twice = row_sum<LANES>(twice);
    // sum q + q_r - (sum of p over the entries and outside): p of an expert listed twice is in its terms twice
    float sum = terms - twice;
    if (t_lse && o.rest_q > 0.0f) {
        const float over = inverse(o.rest_q);
        sum += o.rest_q * above_log(o.gap * over, o.rest_p * over);      // p_r / q_r - 1 and p_r / q_r
    } else {
        sum += o.rest_p + (o.mass - 1.0f);
    }
    if (at_row.there && q0 == 0) loss[first + threadIdx.x / LANES] = at_row.live && o.soft.total != 0.0f && o.listed ? tau * tau * sum : 0.0f;
    lds_order();
}

template <typename T, int LANES, int VPL, bool VEC, int NK>
__global__ __launch_bounds__(256) void route_distill_backward_kernel(const T *__restrict__ logits, int64_t rows, int E, int64_t ld, float tau, float inv_tau,
                                                                     const uint8_t *__restrict__ row_mask, const int32_t *__restrict__ t_idx,
                                                                     const float *__restrict__ t_logit, const float *__restrict__ t_lse, int K,
                                                                     const float *__restrict__ d_loss, int add, T *__restrict__ d_logits,
                                                                     int64_t ld_d)
{
    constexpr int ROWS_PER_BLOCK = 256 / LANES;
    __shared__ __align__(16) float lds[ROWS_PER_BLOCK * LANES * VPL];
    const int q0 = threadIdx.x % LANES;
    float *mine = lds + threadIdx.x / LANES * (LANES * VPL);
    const int64_t first = first_row(ROWS_PER_BLOCK);
    if (first >= rows) return;
    const RowAt at_row = row_at(threadIdx.x / LANES, rows - first, row_mask, first);
    Distilled<LANES, VPL, NK> o;
    distill_row<true, T, LANES, VPL, VEC, NK>(logits, first, at_row, E, ld, inv_tau, t_idx, t_logit, t_lse, K, q0, mine, o);
    const bool counts = at_row.live && o.soft.total != 0.0f;
    const float along = d_loss[first + at_row.slot];
    lds_order();
    // sum q - (Q + q_r) p: where Q + q_r is not 1, the rest of p goes along
    const float off = o.rest_q > 0.0f ? 0.0f : 1.0f - o.mass;
#pragma unroll
    for (int r = 0; r < NK; ++r) o.less[r] = o.again[r] ? o.less[r] : fmaf(o.p[r], off, o.less[r]);
    lds_put<LANES, NK>(mine, q0, K, o.at, o.again, o.less);
    float listed[VPL];
    lds_values<LANES, VPL, VEC>(mine, q0, listed);
    lds_order();
    const float unit = tau * along;
    const float scale = inverse(o.soft.total);
    // Q + q_r - q_r / p_r is (p_r - q_r) / p_r where sum q + q_r is 1
    const float outside = (o.rest_q > 0.0f ? o.gap / o.rest_p : o.mass) * scale;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        const float g = listed[j] == -INFINITY ? o.e[j] * outside : -listed[j];
        o.y[j] = counts && o.listed ? unit * g : 0.0f;
    }
    if (at_row.there && (counts || !add)) row_store<T, LANES, VPL, VEC>(d_logits + (first + threadIdx.x / LANES) * ld_d, E, q0, add != 0, o.y);
}

// The temperatures that fp32 carries.  d = log p - log q is off by a few 2^-24 times 1 + |logit - t_logit| / tau + |t_lse|.  A large tau makes d itself small, of order 1 / tau, so that
// the gradient loses tau 2^-24 of itself; a small one makes that error 2^-24 / tau of q.  Largest errors of 2000 rows of 64 experts, teacher within 0.5 of the student's
// logits, as a share of a row's gradient: tau 32 7e-5, 256 4e-4, 10^4 2e-2, 10^6 more than all of it; as a share of tau d_loss: 2^-6 1e-5, 2^-8 5e-5, 10^-4 1e-3, 10^-6 0.06.
constexpr float kLeastTau = 0x1p-8f, kMostTau = 0x1p8f;

static int check_distill(int64_t rows, int32_t E, float temperature, const int32_t *t_idx, const float *t_logit, int32_t K)
{
    if (K < 1 || K > E || !(temperature >= kLeastTau) || !(temperature <= kMostTau)) return RAILSCHED_ERR_INVALID_ARG;
    if (K > kMaxListed) return RAILSCHED_ERR_UNSUPPORTED;
    if (rows > 0 && (!t_idx || !t_logit)) return RAILSCHED_ERR_NULL_PTR;
    return RAILSCHED_OK;
}

}  // namespace rs

extern "C" int railsched_route_distill(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, float temperature,
                                       const uint8_t *row_mask, const int32_t *t_idx, const float *t_logit, const float *t_lse, int32_t K,
                                       float *loss, void *stream)
{
    using namespace rs;
    if (int rc = check_router(logits, dtype, rows, E, ld, temperature)) return rc;
    if (int rc = check_distill(rows, E, temperature, t_idx, t_logit, K)) return rc;
    if (rows == 0) return RAILSCHED_OK;
    if (!loss) return RAILSCHED_ERR_NULL_PTR;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return by_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        return by_shape<false, T>(E, [&](auto s) {
            using S = decltype(s);
            return by_entries<S>(K, [&](auto n) {
            hipLaunchKernelGGL((route_distill_kernel<T, S::LANES, S::VPL, S::VEC, decltype(n)::value>), row_grid(rows, 256 / S::LANES), dim3(256), 0, st,
                                   static_cast<const T *>(logits), rows, E, ld, temperature, 1.0f / temperature, row_mask, t_idx, t_logit, t_lse, K, loss);
                return launch_status();
            });
        });
    });
}

extern "C" int railsched_route_distill_backward(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, float temperature,
                                                const uint8_t *row_mask, const int32_t *t_idx, const float *t_logit, const float *t_lse,
                                                int32_t K, const float *d_loss, int32_t accumulate, void *d_logits, int64_t ld_d,
                                                void *stream)
{
    using namespace rs;
    if (int rc = check_router(logits, dtype, rows, E, ld, temperature)) return rc;
    if (int rc = check_gradient(logits, d_logits, rows, E, ld_d, accumulate)) return rc;
    if (int rc = check_distill(rows, E, temperature, t_idx, t_logit, K)) return rc;
    if (rows == 0) return RAILSCHED_OK;
    if (!d_loss) return RAILSCHED_ERR_NULL_PTR;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return by_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        return by_shape<true, T>(E, [&](auto s) {
            using S = decltype(s);
            return by_entries<S>(K, [&](auto n) {
            hipLaunchKernelGGL((route_distill_backward_kernel<T, S::LANES, S::VPL, S::VEC, decltype(n)::value>), row_grid(rows, 256 / S::LANES), dim3(256), 0, st,
                                   static_cast<const T *>(logits), rows, E, ld, temperature, 1.0f / temperature, row_mask, t_idx, t_logit, t_lse, K, d_loss, accumulate,
                                   static_cast<T *>(d_logits), ld_d);
                return launch_status();
            });
        });
    });
}
