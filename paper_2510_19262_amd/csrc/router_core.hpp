// Device-side pieces of the operators on a router's logits (log probabilities, balance loss, distillation): rows of
// E <= 1024 logits held in registers by LANES consecutive lanes, VPL values each, their softmax, and a row in LDS
// through which values listed by expert (picks, a teacher's entries) reach the lanes that hold the experts.  Not one of the .h files, which the
// kernels of the five stages share and the figures measured for them go by: none of those kernels includes it.
#pragma once

#include "topk_core.h"

#include <type_traits>

namespace rs {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16_t;
typedef _Float16 f16_t;

constexpr int kMaxListed = 64;     // alternatives of a row, entries of a teacher's list

// ---- four consecutive values: 16 bytes of fp32, 8 of the short types, which global memory gives and takes at any address that a value can have
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
template <typename T>
__device__ __forceinline__ void load4(const T *p, float (&v)[4])
{
    if constexpr (sizeof(T) == 4) {
        const f32x4 x = __builtin_nontemporal_load(reinterpret_cast<const f32x4_any *>(p));
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    } else {
        const u16x4 x = __builtin_bit_cast(u16x4, __builtin_nontemporal_load(reinterpret_cast<const u32x2_any *>(p)));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)__builtin_bit_cast(T, (uint16_t)x[i]);
    }
}
template <bool STREAMING, typename T>
__device__ __forceinline__ void store4(T *p, const float (&v)[4])
{
    if constexpr (sizeof(T) == 4) {
        f32x4_any x;
        x.x = v[0]; x.y = v[1]; x.z = v[2]; x.w = v[3];
        if constexpr (STREAMING) __builtin_nontemporal_store(x, reinterpret_cast<f32x4_any *>(p));
        else *reinterpret_cast<f32x4_any *>(p) = x;
    } else {
        u16x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(uint16_t, (T)v[i]);      // to nearest, ties to even
        if constexpr (STREAMING) __builtin_nontemporal_store(__builtin_bit_cast(u32x2_any, x), reinterpret_cast<u32x2_any *>(p));
        else *reinterpret_cast<u32x2_any *>(p) = __builtin_bit_cast(u32x2_any, x);
    }
}

// ---- sums and maxima over the LANES lanes of a row, in all of them.  Inside 16 lanes the partner's value is an operand of the addition itself.
template <int OFF>
__device__ __forceinline__ float partner(float v)
{
    if constexpr (OFF <= 8) return __int_as_float(from_partner<OFF>(__float_as_int(v)));
    else return xlane<OFF>(v);
}
template <int LANES, typename F>
__device__ __forceinline__ float row_reduce(float v, F op)
{
    if constexpr (LANES >= 2) v = op(v, partner<1>(v));
    if constexpr (LANES >= 4) v = op(v, partner<2>(v));
    if constexpr (LANES >= 8) v = op(v, partner<4>(v));
    if constexpr (LANES >= 16) v = op(v, partner<8>(v));
    if constexpr (LANES >= 32) v = op(v, partner<16>(v));
    if constexpr (LANES >= 64) v = op(v, partner<32>(v));
    return v;
}
template <int LANES>
__device__ __forceinline__ float row_max(float v) { return row_reduce<LANES>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int LANES>
__device__ __forceinline__ float row_sum(float v) { return row_reduce<LANES>(v, [](float a, float b) { return a + b; }); }

// whether any lane of this lane's row says so
template <int LANES>
__device__ __forceinline__ bool row_any(bool v)
{
    const unsigned long long all = __ballot(v);
    if constexpr (LANES == 64) return all != 0ull;
    else return ((all >> (threadIdx.x & 63u & ~(unsigned)(LANES - 1))) & ((1ull << LANES) - 1ull)) != 0ull;
}

// ---- the first of a workgroup's `each` rows.  A grid covers all rows, in two dimensions where one would have more work-items than 32 bits count; a loop over
// the rows instead would keep every loop-invariant condition in scalar registers, and spill them.
__device__ __forceinline__ int64_t first_row(int each) { return ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * each; }
inline dim3 row_grid(int64_t rows, int each)
{
    const int64_t blocks = (rows + each - 1) / each, wide = 1 << 22;
    return blocks <= wide ? dim3((unsigned)blocks) : dim3((unsigned)wide, (unsigned)((blocks + wide - 1) / wide));
}

// ---- which row the lanes are at.  A workgroup has the rows first, first + 1, ... in hand, one to LANES lanes, of which `left` exist.  Lanes without a row, and
// lanes whose row is masked, follow the workgroup's first row instead: their loads need no branch (a load under a condition is waited for before
// the next one is made), read what is read anyway, and what comes of them is not used.
struct RowAt {
    int slot;       // the row followed, from the first one
    bool there;     // a row of its own
    bool live;      // that is not masked
};
__device__ __forceinline__ RowAt row_at(int slot, int64_t left, const uint8_t *__restrict__ row_mask, int64_t first)
{
    RowAt r;
    r.there = slot < left;
    r.slot = r.there ? slot : 0;
    r.live = r.there;
    if (row_mask) {
        r.live = r.there && row_mask[first + r.slot] != 0;
        r.slot = r.live ? r.slot : 0;
    }
    return r;
}
// row `slot` of rows `ld` apart (both below 2^32)
template <typename T>
__device__ __forceinline__ T *row_of(T *first, int slot, int64_t ld) { return first + (uint64_t)(uint32_t)slot * (uint32_t)ld; }

// This lane's places of a row as they are in memory: fetched, and made fp32 values when they are needed (anything done to a loaded value waits for it).
template <typename T, int VPL, bool VEC>
struct RowRaw {
    typedef typename std::conditional<sizeof(T) == 4, f32x4, u32x2>::type four;
    typedef typename std::conditional<sizeof(T) == 4, f32x4_any, u32x2_any>::type four_any;
    typename std::conditional<VEC, four, T>::type v[VEC ? VPL / 4 : VPL];
};
// VEC (E >= 4): places of four consecutive experts, interleaved over the lanes, as slot_index() numbers them.  Where E is no multiple of four, the row's last four values stand for
// the part of a four that it ends with, and are moved to their places when they are taken.  Streaming, but for rows some of whose logits are
// fetched again (AGAIN): those are to stay in the L2 until then.  Gradient of the distillation of 2^20 x 256: 386 us streaming, 370 so; of the balance
// loss, which fetches nothing again: 340, 356.
template <bool AGAIN, typename T, int LANES, int VPL, bool VEC>
__device__ __forceinline__ void row_fetch(const T *__restrict__ row, int E, int q, RowRaw<T, VPL, VEC> &raw)
{
    if constexpr (VEC) {
#pragma unroll
        for (int c = 0; c < VPL / 4; ++c) {
            const int e0 = 4 * (q + LANES * c);
            const auto *from = reinterpret_cast<const typename RowRaw<T, VPL, VEC>::four_any *>(row + (e0 < E - 4 ? e0 : E - 4));
            raw.v[c] = AGAIN ? *from : __builtin_nontemporal_load(from);
        }
    } else {
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int e = q + LANES * j;
            raw.v[j] = row[e < E ? e : 0];
        }
    }
}
template <typename T, typename R>
__device__ __forceinline__ void four_values(const R &raw, float (&v)[4])
{
    if constexpr (sizeof(T) == 4) {
        v[0] = raw.x; v[1] = raw.y; v[2] = raw.z; v[3] = raw.w;
    } else {
        const u16x4 h = __builtin_bit_cast(u16x4, raw);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)__builtin_bit_cast(T, (uint16_t)h[i]);
    }
}
// the values; places behind the row are -infinity.  PARTS: whether the row may end with a part of a four
template <typename T, int LANES, int VPL, bool VEC, bool PARTS = true>
__device__ __forceinline__ void row_take(const RowRaw<T, VPL, VEC> &raw, int E, int q, float (&x)[VPL])
{
    if constexpr (VEC) {
        float v[4];
#pragma unroll
        for (int c = 0; c < VPL / 4; ++c) {
            four_values<T>(raw.v[c], v);
            const int e0 = 4 * (q + LANES * c);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * c + i] = e0 < E ? v[i] : -INFINITY;
        }
        if (const int r = E & 3; PARTS && r != 0) {
#pragma unroll
            for (int c = 0; c < VPL / 4; ++c) {
                if ((E >> 2) / LANES != c) continue;      // of these, a lane has the row's last r < 4 values
                four_values<T>(raw.v[c], v);
                const bool last = q == (E >> 2) % LANES;
                x[4 * c] = last ? (r == 1 ? v[3] : r == 2 ? v[2] : v[1]) : x[4 * c];
                x[4 * c + 1] = last ? (r == 1 ? -INFINITY : r == 2 ? v[3] : v[2]) : x[4 * c + 1];
                x[4 * c + 2] = last ? (r == 3 ? v[3] : -INFINITY) : x[4 * c + 2];
                x[4 * c + 3] = last ? -INFINITY : x[4 * c + 3];
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < VPL; ++j) x[j] = q + LANES * j < E ? (float)raw.v[j] : -INFINITY;
    }
}
template <bool AGAIN, typename T, int LANES, int VPL, bool VEC, bool PARTS = true>
__device__ __forceinline__ void row_values(const T *__restrict__ row, int E, int q, float (&x)[VPL])
{
    RowRaw<T, VPL, VEC> raw;
    row_fetch<AGAIN, T, LANES, VPL, VEC>(row, E, q, raw);
    row_take<T, LANES, VPL, VEC, PARTS>(raw, E, q, x);
}

// The gradient of a row: written, or added to what is there.  Streaming where its fours are all there is; a row that ends with a part of a four has lines written
// by two stores, which then meet in the L2 (gradient of 2^20 x 61: 114 us, 243 streaming).
template <typename T, int LANES, int VPL, bool VEC, bool PARTS = true>
__device__ __forceinline__ void row_store(T *__restrict__ row, int E, int q, bool add, const float (&x)[VPL])
{
    if constexpr (VEC) {
        auto four = [&](int c, int e0, auto streaming) {
            float v[4];
            if (add) load4(row + e0, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = add ? v[i] + x[4 * c + i] : x[4 * c + i];
            store4<decltype(streaming)::value>(row + e0, v);
        };
        if (!PARTS || (E & 3) == 0) {
#pragma unroll
            for (int c = 0; c < VPL / 4; ++c) {
                const int e0 = 4 * (q + LANES * c);
                if (e0 < E) four(c, e0, std::true_type());
            }
            return;
        }
#pragma unroll
        for (int c = 0; c < VPL / 4; ++c) {
            const int e0 = 4 * (q + LANES * c);
            if (e0 + 4 <= E) four(c, e0, std::false_type());
            if ((E >> 2) / LANES == c && q == (E >> 2) % LANES) {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (e0 + i < E) row[e0 + i] = (T)(add ? (float)row[e0 + i] + x[4 * c + i] : x[4 * c + i]);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int e = q + LANES * j;
            if (e < E) row[e] = (T)(add ? (float)row[e] + x[j] : x[j]);
        }
    }
}

// Everything about a row is done in powers of two: with c = log2(e) / tau, y = c (logit - largest) and the hardware's 2^y.  y is 0 for the largest logit,
// exactly, and no finite logits overflow; 2^y is off by about 2 |y| 2^-24 of itself: at most about 2^-24 of the row's largest.
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
__device__ __forceinline__ float pow2(float y) { return __builtin_amdgcn_exp2f(y); }
__device__ __forceinline__ float log2_of(float v) { return __builtin_amdgcn_logf(v); }       // of normal numbers, to one step
__device__ __forceinline__ float inverse(float v) { return __builtin_amdgcn_rcpf(v); }        // likewise: a tenth of a division's instructions

// Softmax of a row: x holds the logits on entry and y on return, e the powers.
struct RowSoft {
    float largest;  // logit (0 in a row without one)
    float total;    // sum of e: at least 1, or 0 in a row that does not count (every logit -infinity), or NaN
    __device__ __forceinline__ float y(float logit, float c) const { return c * (logit - largest); }
};
template <int LANES, int VPL>
__device__ __forceinline__ RowSoft row_softmax(float (&x)[VPL], float (&e)[VPL], float c)
{
    RowSoft r;
    float m = x[0];
#pragma unroll
    for (int j = 1; j < VPL; ++j) m = fmaxf(m, x[j]);
    m = row_max<LANES>(m);
    r.largest = m == -INFINITY ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        x[j] = r.y(x[j], c);
        e[j] = pow2(x[j]);
        s += e[j];
    }
    r.total = row_sum<LANES>(s);
    return r;
}

// The same without the powers: the logits stay as they are, and dot is the sum of 2^y y.
template <int LANES, int VPL>
__device__ __forceinline__ RowSoft row_sums(const float (&x)[VPL], float c, float &dot)
{
    RowSoft r;
    float m = x[0];
#pragma unroll
    for (int j = 1; j < VPL; ++j) m = fmaxf(m, x[j]);
    m = row_max<LANES>(m);
    r.largest = m == -INFINITY ? 0.0f : m;
    float s = 0.0f, d = 0.0f;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        const float y = r.y(x[j], c), e = pow2(y);
        s += e;
        d = fmaf(e, fmaxf(y, -1e30f), d);
    }
    r.total = row_sum<LANES>(s);
    dot = row_sum<LANES>(d);
    return r;
}

// sum of e y over the row (e 0 where y is -infinity: the product is 0 there)
template <int LANES, int VPL>
__device__ __forceinline__ float row_dot(const float (&y)[VPL], const float (&e)[VPL])
{
    float a = 0.0f;
#pragma unroll
    for (int j = 0; j < VPL; ++j) a += e[j] * fmaxf(y[j], -1e30f);
    return row_sum<LANES>(a);
}

// ---- a row of LANES * VPL floats in LDS for every row of the wavefront.  Only lanes of one wavefront meet in it, and a wavefront's LDS
// accesses are carried out in order: a fence that keeps the compiler from moving them is all that is needed.
__device__ __forceinline__ void lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
template <int LANES, int VPL, bool VEC>
__device__ __forceinline__ void lds_fill(float *row, int q, float value)
{
#pragma unroll
    for (int c = 0; c < VPL / 4; ++c) {                  // every place belongs to one lane, whatever the order
        f32x4 v;
        v.x = v.y = v.z = v.w = value;
        *reinterpret_cast<f32x4 *>(row + 4 * (q + LANES * c)) = v;
    }
}
template <int LANES, int VPL, bool VEC>
__device__ __forceinline__ void lds_values(const float *row, int q, float (&x)[VPL])
{
    if constexpr (VEC) {
#pragma unroll
        for (int c = 0; c < VPL / 4; ++c) {
            const f32x4 v = *reinterpret_cast<const f32x4 *>(row + 4 * (q + LANES * c));
            x[4 * c + 0] = v.x; x[4 * c + 1] = v.y; x[4 * c + 2] = v.z; x[4 * c + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < VPL; ++j) x[j] = row[q + LANES * j];
    }
}

// Marks the places at[r] (-1: none) of this lane's entries q, q + LANES, ... of `count` in the row, whose places hold nothing above 0; on return again[r] says that a
// later entry of the same place holds it (of several entries with one place exactly the last is not `again`).  The marked places hold values above 0.
template <int LANES, int N>
__device__ __forceinline__ void lds_mark(float *row, int q, int count, const int (&at)[N], bool (&again)[N])
{
    auto mark = [&](int r) { return __float_as_int((float)(q + LANES * r + 1)); };       // positive floats are in order as integers too
#pragma unroll
    for (int r = 0; r < N; ++r)
        if (LANES * r < count && at[r] >= 0) atomicMax(reinterpret_cast<int *>(row + at[r]), mark(r));
    lds_order();
#pragma unroll
    for (int r = 0; r < N; ++r) again[r] = LANES * r < count && at[r] >= 0 && __float_as_int(row[at[r]]) != mark(r);
    lds_order();
}

// Puts value[r] at the marked places; entries of one place are added up in the order of the entries, so that equal inputs give equal bits.
template <int LANES, int N>
__device__ __forceinline__ void lds_put(float *row, int q, int count, const int (&at)[N], const bool (&again)[N], const float (&value)[N])
{
    bool any = false;
#pragma unroll
    for (int r = 0; r < N; ++r) any |= again[r];
    if (__ballot(any) == 0ull) {
#pragma unroll
        for (int r = 0; r < N; ++r)
            if (LANES * r < count && at[r] >= 0) row[at[r]] = value[r];
    } else {                                             // an expert listed twice: one entry after the other
#pragma unroll
        for (int r = 0; r < N; ++r)
            if (LANES * r < count && at[r] >= 0) row[at[r]] = 0.0f;
        lds_order();
#pragma unroll
        for (int r = 0; r < N; ++r)
            if (LANES * r < count)
                for (int i = 0; i < LANES; ++i) {
                    if (q == i && at[r] >= 0) row[at[r]] += value[r];
                    lds_order();
                }
    }
    lds_order();
}

// ---- host side
inline int check_router(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, float temperature)
{
    if (dtype < RAILSCHED_F32 || dtype > RAILSCHED_F16 || rows < 0 || E < 1 || ld < E) return RAILSCHED_ERR_INVALID_ARG;
    if (!(temperature >= 0x1p-60f) || !(temperature <= 0x1p60f)) return RAILSCHED_ERR_INVALID_ARG;
    if (E > kMaxExperts || rows > 0x7FFFFFFFll || ld > (int64_t(1) << 31)) return RAILSCHED_ERR_UNSUPPORTED;
    if (rows > 0 && !logits) return RAILSCHED_ERR_NULL_PTR;
    return RAILSCHED_OK;
}
inline int check_gradient(const void *logits, const void *d_logits, int64_t rows, int32_t E, int64_t ld_d, int32_t accumulate)
{
    if (ld_d < E || (accumulate != 0 && accumulate != 1)) return RAILSCHED_ERR_INVALID_ARG;
    if (ld_d > (int64_t(1) << 31)) return RAILSCHED_ERR_UNSUPPORTED;
    if (rows > 0 && !d_logits) return RAILSCHED_ERR_NULL_PTR;
    if (rows > 0 && d_logits == logits) return RAILSCHED_ERR_INVALID_ARG;
    return RAILSCHED_OK;
}
// The shape a row of E logits is held in: LANES lanes, VPL values each, in places of four or one by one.
template <int L, int V, bool F>
struct Shape {
    static constexpr int LANES = L, VPL = V;
    static constexpr bool VEC = F;
};
// f(Shape) for rows of E logits.  Every lane less is a step less in the row's sums and more rows to a wavefront; more than 16 values a lane cost occupancy.
// A kernel that only reads its rows (not WHOLE) takes the fewest lanes that pay: 8 values a lane at least, 16 or 32 of the short types, whose four are
// half as many bytes.  2^22 x 32: 123 us with 4 lanes, 172 with 8; 2^20 x 64 bf16: 44 with 4, 48 with 8, but fp32 68 and 61; 2^20 x 256 bf16: 118 with 8 lanes,
// 128 with 16, fp32 205 and 198.  One that writes them too, or keeps sums of its places (WHOLE), is faster with more: gradient of 2^22 x 32: 222 us
// with 8 lanes, 247 with 4; 2^20 x 64: 95 with 8, 116 with 4.  Read and written one by one: rows of less than four, and where WHOLE rows of 9 to 31
// that end with a part of a four.  Balance gradient of 2^26 logits, one by one and in fours: bf16 in rows of 9 83 and 114 us, of 17 89 and 118, of 31 60 and 87; fp32 of 9 133 and 136, of 11 127
// and 141, of 17 134 and 140, but of 14 138 and 115, of 27 136 and 128, of 30 134 and 112; the other gradients and types differ less, the same way.  Longer rows: of 45 bf16 133 and 88.
template <bool WHOLE, typename T, typename F>
inline int by_shape(int E, F f)
{
    constexpr bool brief = !WHOLE && sizeof(T) == 2;
    if (E < 4) return f(Shape<1, 4, false>());
    if constexpr (WHOLE) {
        if (E > 8 && E <= 16 && E % 4 != 0) return f(Shape<4, 4, false>());
        if (E > 16 && E <= 32 && E % 4 != 0) return f(Shape<8, 4, false>());
    }
    if (E <= 8) return f(Shape<WHOLE ? 2 : 1, WHOLE ? 4 : 8, true>());
    if (E <= 16) return f(Shape<WHOLE ? 4 : 2, WHOLE ? 4 : 8, true>());
    if (E <= 32) return f(Shape<WHOLE ? 8 : 4, WHOLE ? 4 : 8, true>());
    if (E <= 64) return f(Shape<brief ? 4 : 8, brief ? 16 : 8, true>());
    if (E <= 128) return f(Shape<8, 16, true>());
    if (E <= 256) return f(Shape<brief ? 8 : 16, brief ? 32 : 16, true>());
    if (E <= 512) return f(Shape<brief ? 16 : 32, brief ? 32 : 16, true>());
    return f(Shape<64, 16, true>());
}
// f(how many of `count` <= kMaxListed entries of a list a lane holds, at most): 1 or 2 where they fit, or as many as the longest list takes (of E entries at most)
template <typename S, typename F>
inline int by_entries(int count, F f)
{
    constexpr int most = S::VPL < kMaxListed / S::LANES ? S::VPL : kMaxListed / S::LANES;
    if (most == 1 || count <= S::LANES) return f(std::integral_constant<int, 1>());
    if (most == 2 || count <= 2 * S::LANES) return f(std::integral_constant<int, 2>());
    return f(std::integral_constant<int, most>());
}

// f(T()) for the type that dtype names
template <typename F>
inline int by_dtype(int32_t dtype, F f)
{
    if (dtype == RAILSCHED_BF16) return f(bf16_t());
    if (dtype == RAILSCHED_F16) return f(f16_t());
    return f(float());
}

}  // namespace rs
