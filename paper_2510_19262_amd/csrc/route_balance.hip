// Balance loss of groups of rows with the counts of picks per expert, and its gradient.
//
// A workgroup adds up the probabilities of a part of a group's rows (fp32, a lane its own experts), counts its picks (LDS) and writes one record; a second kernel
// adds the records of a group up in their order (fp64) and forms the loss.  No floating-point atomics: equal inputs give equal bits.  Equal groups are dealt out, `per`
// workgroups to a group, round after round, so that what is in flight lies together; with one workgroup to a group the outputs leave at once.  Rows of ragged groups
// are cut into slices, a workgroup each, whose parts are of one group or several; slices and groups are both in row order, so the part of group g in slice s can take
// the record s + g: no two parts share it.
//
// Bound by the reads of logits and picks (2^25 x 8 with 2 picks: 1.34 GB in 209 us, 6.4 TB/s; one group of 2^20 x 256: 187 us), where the rows are few by a chain of dependent
// reads (offsets, rows, records: 13 and 6 us for 300 sequences of 65537 x 61).  The gradient reads and writes every logit: 2^20 x 256 in 341 us, 6.3 TB/s.
#include "router_core.hpp"

namespace rs {

// rows of group g, kept within [0, rows]
struct Groups {
    const int64_t *off;     // NULL: equal parts of `each` rows
    int64_t each, rows;
    int n;
    __device__ __forceinline__ int64_t within(int64_t b) const { return b < 0 ? 0 : b < rows ? b : rows; }
    __device__ __forceinline__ int64_t begin(int g) const { return within(off ? off[g] : g * each); }
    // the last group that begins at r or before, the first one if none does: 64 probes a step by the lanes of a wavefront
    __device__ __forceinline__ int holding(int64_t r) const
    {
        if (!off) return (int)(r / each);
        const int lane = threadIdx.x & 63;
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int step = (hi - lo + 63) / 64;
            const int at = lo + lane * step;
            const unsigned long long ok = __ballot(at < hi && off[at < hi ? at : lo] <= r);
            if (ok == 0ull) return lo;
            lo += (63 - __clzll((long long)ok)) * step;
            hi = lo + step < hi ? lo + step : hi;
        }
        return lo;
    }
};

// The groups from `first` on, one after the other: their offsets are fetched 63 groups at a time, a lane each.
struct GroupWalk {
    int g, base;
    int64_t held;           // this lane's offset: of group base + lane
    __device__ __forceinline__ void fetch(const Groups &groups)
    {
        base = g;
        const int at = g + (int)(threadIdx.x & 63);
        held = groups.begin(at <= groups.n ? at : groups.n);
    }
    __device__ __forceinline__ GroupWalk(const Groups &groups, int first) : g(first) { fetch(groups); }
    __device__ __forceinline__ void next(const Groups &groups)
    {
        if (++g - base == 63 && g < groups.n) fetch(groups);
    }
    __device__ __forceinline__ int64_t lane(int i) const
    {
        const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(uint32_t)(uint64_t)held, i);
        const unsigned hi = (unsigned)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)held >> 32), i);
        return (int64_t)(((uint64_t)hi << 32) | lo);
    }
    __device__ __forceinline__ int64_t begin() const { return lane(g - base); }
    __device__ __forceinline__ int64_t end() const { return lane(g - base + 1); }
};

// The workspace: a record for every part (E sums, E counts, the rows that count), the tickets of the groups, and the products of their column tiles.
struct Records {
    float *data;
    unsigned *tickets;
    double *dots;
    int64_t words;
    int per;                // records of a group, one after the other; 0: of slices
    __device__ __forceinline__ float *at(int64_t r, int64_t group) const { return data + (r + (per ? group * per : group)) * words; }
};

constexpr int kMaxGroups = 1 << 23;                     // a workgroup of 256 threads each: half the work-items that a grid counts
constexpr int kTile = 32;                               // columns of a tile where a grid of them joins the records

// v added up over the lanes that are a multiple of LANES away from this one, in all of them
template <int LANES>
__device__ __forceinline__ float rows_sum(float v)
{
    if constexpr (LANES <= 1) v += xlane<1>(v);
    if constexpr (LANES <= 2) v += xlane<2>(v);
    if constexpr (LANES <= 4) v += __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), 0x101F));     // lane ^ 4
    if constexpr (LANES <= 8) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xF, 0xF, false));   // row_ror:8, lane ^ 8
    if constexpr (LANES <= 16) v += xlane<16>(v);
    if constexpr (LANES <= 32) v += xlane<32>(v);
    return v;
}

// sum over the workgroup of 64 * WAVES threads, in thread 0; the order is fixed
template <int WAVES>
__device__ __forceinline__ double block_sum(double v, double *part)
{
#pragma unroll
    for (int w = 32; w >= 1; w /= 2) v += __shfl_down(v, w);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += part[w];
    }
    return s;
}
__device__ __forceinline__ float balance_loss(float coef, int E, int k, int64_t n, double dot)
{
    return n ? (float)((double)coef * E / ((double)k * n * n) * dot) : 0.0f;
}

// EQUAL: groups of `each` rows, dealt out to `per` workgroups; otherwise slices of slice_rows.
template <typename T, int LANES, int VPL, bool VEC, int THREADS, bool EQUAL>
__global__ __launch_bounds__(THREADS) void route_balance_kernel(const T *__restrict__ logits, int E, int64_t ld, const uint8_t *__restrict__ row_mask,
                                                                const int32_t *__restrict__ topk_idx, int k, Groups groups, int64_t slice_rows,
                                                                float coef, Records records, int64_t *__restrict__ counts,
                                                                int64_t *__restrict__ tokens, float *__restrict__ prob_sum, float *__restrict__ loss)
{
    constexpr int ROWS_PER_BLOCK = THREADS / LANES, WAVES = THREADS / 64;
    __shared__ float sums[WAVES][LANES * VPL];
    __shared__ unsigned picks[LANES * VPL];
    __shared__ unsigned counted;
    __shared__ double part[WAVES];
    const int q = threadIdx.x % LANES, slot = threadIdx.x / LANES, wave = threadIdx.x >> 6;
    for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < groups.n; i += (int64_t)gridDim.x * THREADS) records.tickets[i] = 0;

    // the rows lo, lo + 1, ... (as many as the workgroup has in hand), then those `step` further on, up to hi: a part of group g, whose r-th record this is
    auto add_up = [&](int g, int64_t lo, int64_t hi, int64_t step, int64_t r) {
        for (int i = threadIdx.x; i < E; i += THREADS) picks[i] = 0;
        if (threadIdx.x == 0) counted = 0;
        __syncthreads();
        float acc[VPL];
#pragma unroll
        for (int j = 0; j < VPL; ++j) acc[j] = 0.0f;
        unsigned here = 0;
        // the rows in hand, with a lane's first pick; the next ones are on their way while these are worked on (2^20 x 256 bf16: 116 us, 159 without)
        RowAt at_next;
        RowRaw<T, VPL, VEC> raw;
        int pick_next;
        auto fetch = [&](int64_t w) {
            at_next = row_at(slot, hi - w, row_mask, w);
            pick_next = topk_idx[w * k + at_next.slot * k + (q < k ? q : 0)];
            row_fetch<false, T, LANES, VPL, VEC>(row_of(logits + w * ld, at_next.slot, ld), E, q, raw);
        };
        // each group starts at another of its rounds: groups a power of two apart would have all their workgroups at the same memory channels (32 groups of 2^20 x 8: 210 us, 228
        // from the first round on)
        const int64_t turns = lo < hi ? (hi - lo + step - 1) / step : 0;
        int64_t turn = g * turns / groups.n;
        if (turns) fetch(lo + turn * step);
        for (int64_t done = 0; done < turns; ++done) {
            const int64_t w0 = lo + turn * step;
            if (++turn == turns) turn = 0;
            const RowAt at_row = at_next;
            const int pick = pick_next;
            float t[VPL], e[VPL];
            row_take<T, LANES, VPL, VEC>(raw, E, q, t);
            if (done + 1 < turns) fetch(lo + turn * step);
            const RowSoft soft = row_softmax<LANES, VPL>(t, e, kLog2e);
            const bool use = at_row.live && soft.total != 0.0f;
            const float scale = inverse(soft.total);
#pragma unroll
            for (int j = 0; j < VPL; ++j) acc[j] += use ? e[j] * scale : 0.0f;
            if (use) {
                here += q == 0;
                if (q < k && pick >= 0 && pick < E) atomicAdd(&picks[pick], 1u);
                for (int j = q + LANES; j < k; j += LANES) {
                    const int at = topk_idx[w0 * k + at_row.slot * k + j];
                    if (at >= 0 && at < E) atomicAdd(&picks[at], 1u);
                }
            }
        }
        if (here) atomicAdd(&counted, here);
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const float s = rows_sum<LANES>(acc[j]);
            if ((threadIdx.x & 63) < LANES) sums[wave][slot_index<LANES, VPL, VEC>(q, j)] = s;
        }
        __syncthreads();
        auto wave_sums = [&](int i) {
            float s = sums[0][i];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += sums[w][i];
            return s;
        };
        if (EQUAL && records.per == 1) {
            double dot = 0.0;
            for (int i = threadIdx.x; i < E; i += THREADS) {
                const float s = wave_sums(i);
                prob_sum[(int64_t)g * E + i] = s;
                counts[(int64_t)g * E + i] = picks[i];
                dot += (double)s * picks[i];
            }
            dot = block_sum<WAVES>(dot, part);
            if (threadIdx.x == 0) {
                tokens[g] = counted;
                loss[g] = balance_loss(coef, E, k, counted, dot);
            }
        } else {
            float *rec = records.at(r, g);
            for (int i = threadIdx.x; i < E; i += THREADS) {
                rec[i] = wave_sums(i);
                reinterpret_cast<unsigned *>(rec)[E + i] = picks[i];
            }
            if (threadIdx.x == 0) reinterpret_cast<unsigned *>(rec)[2 * E] = counted;
        }
        __syncthreads();
    };

    if constexpr (EQUAL) {
        const int g = (int)(blockIdx.x / (unsigned)records.per), r = (int)(blockIdx.x % (unsigned)records.per);
        add_up(g, g * groups.each + (int64_t)r * ROWS_PER_BLOCK, (g + 1) * groups.each, (int64_t)records.per * ROWS_PER_BLOCK, r);
    } else {
        const int64_t r0 = blockIdx.x * slice_rows;
        const int64_t r1 = r0 + slice_rows < groups.rows ? r0 + slice_rows : groups.rows;
        for (GroupWalk walk(groups, groups.holding(r0)); walk.g < groups.n; walk.next(groups)) {
            const int64_t gb = walk.begin(), ge = walk.end();
            if (gb >= r1) break;
            const int64_t lo = gb > r0 ? gb : r0, hi = ge < r1 ? ge : r1;
            if (lo < hi) add_up(walk.g, lo, hi, ROWS_PER_BLOCK, blockIdx.x);
        }
    }
}

// Adds the records of a group up: a workgroup takes TILE columns at a time (all of them, or one tile in a grid of tiles), its threads rows of records.  TILE holds the
// columns where the records are few: every tile is a round trip to memory (164 groups of 13 records of 891 experts: 28 us in tiles of 32 for a call's 89).
// The last tile of a group to arrive forms the loss from the tiles' products, in the order of the tiles.
template <int THREADS, int TILE>
__global__ __launch_bounds__(THREADS) void route_balance_join_kernel(Records records, int E, int k, Groups groups, int64_t slice_rows, float coef,
                                                                     int64_t *__restrict__ counts, int64_t *__restrict__ tokens,
                                                                     float *__restrict__ prob_sum, float *__restrict__ loss)
{
    constexpr int LINES = THREADS / TILE;
    __shared__ double sums[LINES][TILE];
    __shared__ int64_t picks[LINES][TILE];
    __shared__ double part[THREADS / 64];
    const int g = blockIdx.x, tiles = gridDim.y;
    const int col = threadIdx.x % TILE, line = threadIdx.x / TILE;
    const int64_t gb = groups.begin(g), ge = groups.begin(g + 1);
    const int64_t s0 = records.per ? 0 : gb / slice_rows;
    const int64_t s1 = records.per ? records.per : gb < ge ? (ge - 1) / slice_rows + 1 : s0;
    double dot = 0.0, n = 0.0;
    for (int i0 = blockIdx.y * TILE; i0 < E; i0 += tiles * TILE) {
        const int i = i0 + col;
        double s = 0.0;
        int64_t c = 0;
        if (i < E) {
#pragma unroll 8
            for (int64_t r = s0 + line; r < s1; r += LINES) {
                const float *rec = records.at(r, g);
                s += rec[i];
                c += reinterpret_cast<const unsigned *>(rec)[E + i];
            }
        }
        sums[line][col] = s;
        picks[line][col] = c;
        __syncthreads();
        if (line == 0 && i < E) {
#pragma unroll
            for (int l = 1; l < LINES; ++l) {
                s += sums[l][col];
                c += picks[l][col];
            }
            prob_sum[(int64_t)g * E + i] = (float)s;
            counts[(int64_t)g * E + i] = c;
            dot += s * (double)c;
        }
        __syncthreads();
    }
    for (int64_t r = s0 + threadIdx.x; r < s1; r += THREADS) n += reinterpret_cast<const unsigned *>(records.at(r, g))[2 * E];
    dot = block_sum<THREADS / 64>(dot, part);
    __syncthreads();
    n = block_sum<THREADS / 64>(n, part);
    if (threadIdx.x != 0) return;
    if (tiles > 1) {
        double *dots = records.dots + (int64_t)g * tiles;
        __hip_atomic_store(&dots[blockIdx.y], dot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const unsigned ticket = __hip_atomic_fetch_add(&records.tickets[g], 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        if (ticket != (unsigned)tiles - 1) return;
        dot = 0.0;
        for (int t = 0; t < tiles; ++t) dot += __hip_atomic_load(&dots[t], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    tokens[g] = (int64_t)n;
    loss[g] = balance_loss(coef, E, k, (int64_t)n, dot);
}

// d_logits[e] = p_e (a_e - sum_f a_f p_f), a_e = d_loss coef E c_e / (k n^2).  The gradient does not change with a constant added to a: the mean
// count is taken off first (fp64), so that nothing is lost where the counts are nearly equal.
// PARTS costs this loop over rows 4% where there are none (2^20 x 256: 342 us, 357): 60 scalar registers are spilled with it and 16 values to a lane, 2 without.
template <typename T, int LANES, int VPL, bool VEC, bool PARTS>
__global__ __launch_bounds__(256) void route_balance_backward_kernel(const T *__restrict__ logits, int E, int64_t ld,
                                                                     const uint8_t *__restrict__ row_mask, int k, Groups groups,
                                                                     int slice_rows, float coef, const int64_t *__restrict__ counts,
                                                                     const int64_t *__restrict__ tokens, const float *__restrict__ d_loss,
                                                                     int add, int clear, T *__restrict__ d_logits, int64_t ld_d)
{
    constexpr int ROWS_PER_BLOCK = 256 / LANES;
    __shared__ double part[4], total;
    __shared__ float weight[LANES * VPL];
    const int q = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int64_t r0 = first_row(slice_rows);
    if (r0 >= groups.rows) return;
    const int64_t r1 = r0 + slice_rows < groups.rows ? r0 + slice_rows : groups.rows;
    if (clear) {                                         // the rows before the first group and behind the last one; all, where there is no group
        const int64_t begin = groups.begin(0), end = groups.begin(groups.n);
        float none[VPL];
#pragma unroll
        for (int j = 0; j < VPL; ++j) none[j] = 0.0f;
        for (int64_t w = r0 + slot; w < r1; w += ROWS_PER_BLOCK)
            if (w < begin || w >= end) row_store<T, LANES, VPL, VEC, PARTS>(d_logits + w * ld_d, E, q, false, none);
    }
    for (GroupWalk walk(groups, groups.holding(r0)); walk.g < groups.n; walk.next(groups)) {
        const int g = walk.g;
        const int64_t gb = walk.begin(), ge = walk.end();
        if (gb >= r1) break;
        const int64_t lo = gb > r0 ? gb : r0, hi = ge < r1 ? ge : r1;
        if (lo >= hi) continue;
        const int64_t *__restrict__ c = counts + (int64_t)g * E;
        // the first rows in hand are on their way while the weights are formed
        RowAt at_row = row_at(slot, hi - lo, row_mask, lo);
        float t[VPL];
        row_values<false, T, LANES, VPL, VEC, PARTS>(row_of(logits + lo * ld, at_row.slot, ld), E, q, t);
        double sum = 0.0;
        for (int i = threadIdx.x; i < E; i += 256) sum += (double)c[i];
        sum = block_sum<4>(sum, part);
        if (threadIdx.x == 0) total = sum;
        __syncthreads();
        const double mean = total / E, n = (double)tokens[g];
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
            float e[VPL];
            const RowSoft soft = row_softmax<LANES, VPL>(t, e, kLog2e);
            const bool counts_here = at_row.live && soft.total != 0.0f;
            const float scale = inverse(soft.total);
            float ap = 0.0f;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                e[j] *= scale;
                ap += a[j] * e[j];
            }
            ap = row_sum<LANES>(ap);
#pragma unroll
            for (int j = 0; j < VPL; ++j) t[j] = counts_here ? e[j] * (a[j] - ap) : 0.0f;
            if (at_row.there && (counts_here || !add)) row_store<T, LANES, VPL, VEC, PARTS>(d_logits + (w0 + slot) * ld_d, E, q, add != 0, t);
            if (w0 + ROWS_PER_BLOCK < hi) {
                at_row = row_at(slot, hi - (w0 + ROWS_PER_BLOCK), row_mask, w0 + ROWS_PER_BLOCK);
                row_values<false, T, LANES, VPL, VEC, PARTS>(row_of(logits + (w0 + ROWS_PER_BLOCK) * ld, at_row.slot, ld), E, q, t);
            }
        }
        __syncthreads();
    }
}

// How the rows are shared out, in whole rounds of the rows that a workgroup has in hand.  About as many workgroups as are resident at a time, as many more are another round for
// all: of 256 threads where the groups are short, 8 on a CU with 4 values to a lane, 6 with 8, 5 with 16; of 512 threads, 3 or 2, where a group would have more than 8 records
// of the smaller ones, so that its records stay few (289392 x 128 in 24 groups: 34 us with 504 workgroups, 44 with 528 of 1024 threads; 2^20 x 64 in 200 ragged
// groups: 54 and 65; 200000 x 1000 in 150: 141, 155 of 256 threads).  The registers hold one wavefront less in two places: ragged groups of rows read in fours, 4 values to a lane, have 7
// workgroups on a CU, so that 256 and more of them leave a second round of an eighth; and ragged groups of 16 values to a lane spill 6 to 13 scalar registers.
// Equal groups have whole workgroups, as many as fit or one each: with one each they are anything up to what is resident, or more (4096 x 256 a group: 512 groups
// 319 us, 700 459, 1280 840, all 6.4 to 6.7 TB/s, but 1300 943, 5.8).  Equal groups of at most 16384 logits have a workgroup of 256 threads each: one launch.
struct Cut {
    int threads, per;       // per: workgroups to a group; 0: slices
    int64_t slice_rows, blocks, records;
};
static Cut balance_cut(int64_t rows, int32_t groups, int E, bool equal)
{
    Cut c = {};
    int few = 1, vpl = 1;
    by_shape<true, float>(E, [&](auto s) { vpl = decltype(s)::VPL; return few = 256 / decltype(s)::LANES; });
    for (c.threads = 256;; c.threads = 512) {
        const int64_t in_hand = few * (c.threads / 256), wanted = c.threads == 256 ? (vpl >= 16 ? 1280 : vpl >= 8 ? 1536 : 2048) : (vpl >= 16 ? 512 : 768);
        if (equal) {
            const int64_t each = rows / groups, rounds = (each + in_hand - 1) / in_hand, share = wanted > groups ? wanted / groups : 1;
            c.per = each * E <= 16384 ? 1 : (int)(rounds < share ? rounds : share);
            c.blocks = c.records = (int64_t)groups * c.per;
        } else {
            const int64_t rounds = (rows + wanted * in_hand - 1) / (wanted * in_hand);
            c.slice_rows = (rounds > 1 ? rounds : 1) * in_hand;
            c.blocks = (rows + c.slice_rows - 1) / c.slice_rows;
            c.records = c.blocks + groups;
        }
        if (c.threads == 512 || c.blocks <= 8 * (int64_t)groups) return c;
    }
}
// Rows of a workgroup of the gradient: 16 KiB of logits, 32 KiB of rows of more than 256 bytes; whole rounds of the rows in hand; fewer where the GPU would not be full.  Much
// more is slower by up to a third (2^20 x 256: 340 us with 32 KiB, 417 with 512; 2^21 x 64: 178 with 16, 235 with 256), less pays for the weights too often (2^23 x 8: 135 us
// with 4 KiB, the least, a round of the rows in hand, 90 with 16; 2^20 x 256: 352 with 4).
static int gradient_slice_rows(int64_t rows, int row_bytes, int in_hand)
{
    int64_t r = (row_bytes <= 256 ? 16384 : 32768) / row_bytes;
    if (r > rows / 2048) r = rows / 2048;
    r -= r % in_hand;
    return r > in_hand ? (int)r : in_hand;
}
static int balance_tiles(int E) { return (E + kTile - 1) / kTile; }

// enough for equal groups and for ragged ones
static size_t records_bytes(int64_t rows, int32_t groups, int32_t E)
{
    const int64_t ragged = balance_cut(rows, groups, E, false).records;
    const int64_t equal = groups > 0 && rows % groups == 0 ? balance_cut(rows, groups, E, true).records : 0;
    return align_up((size_t)(ragged > equal ? ragged : equal) * (2 * (size_t)E + 1) * sizeof(float), 256);
}
static size_t tickets_bytes(int32_t groups) { return align_up((size_t)groups * sizeof(unsigned), 256); }

static int check_groups(int64_t rows, const int64_t *group_off, int32_t groups)
{
    if (groups > kMaxGroups) return RAILSCHED_ERR_UNSUPPORTED;
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
    if (rows < 0 || rows > 0x7FFFFFFFll || groups < 0 || groups > kMaxGroups || E < 1 || E > kMaxExperts) return 0;
    return records_bytes(rows, groups, E) + tickets_bytes(groups) + align_up((size_t)groups * balance_tiles(E) * sizeof(double), 256);
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
    const Cut cut = balance_cut(rows, groups, E, !group_off);
    Records records;
    records.data = static_cast<float *>(ws);
    records.words = 2 * (int64_t)E + 1;
    records.per = rows > 0 ? cut.per : 0;
    records.tickets = reinterpret_cast<unsigned *>(static_cast<char *>(ws) + records_bytes(rows, groups, E));
    records.dots = reinterpret_cast<double *>(reinterpret_cast<char *>(records.tickets) + tickets_bytes(groups));
    if (rows > 0) {
        const int rc = by_dtype(dtype, [&](auto t) {
            using T = decltype(t);
            return by_shape<true, T>(E, [&](auto s) {
                using S = decltype(s);
                auto go = [&](auto threads, auto equal) {
                    hipLaunchKernelGGL((route_balance_kernel<T, S::LANES, S::VPL, S::VEC, decltype(threads)::value, decltype(equal)::value>),
                                       dim3((unsigned)cut.blocks), dim3(decltype(threads)::value), 0, st, static_cast<const T *>(logits), E, ld, row_mask,
                                       topk_idx, k, gr, cut.slice_rows, coef, records, counts, tokens, prob_sum, loss);
                    return launch_status();
                };
                constexpr std::integral_constant<int, 256> small;
                constexpr std::integral_constant<int, 512> large;
                if (cut.per) return cut.threads == 256 ? go(small, std::true_type()) : go(large, std::true_type());
                return cut.threads == 256 ? go(small, std::false_type()) : go(large, std::false_type());
            });
        });
        if (rc || cut.per == 1) return rc;
    }
    // a workgroup for every tile of columns where a group has many records; otherwise one for the group, whose tile is all of them, or 256 columns in turn where workgroups
    // of 1024 threads would be 2^32 work-items, which is one more than a launch can have
    const int64_t slice_rows = cut.slice_rows > 0 ? cut.slice_rows : 1;
    auto join = [&](auto threads, auto tile, unsigned tiles) {
        hipLaunchKernelGGL((route_balance_join_kernel<decltype(threads)::value, decltype(tile)::value>), dim3((unsigned)groups, tiles), dim3(decltype(threads)::value),
                           0, st, records, E, k, gr, slice_rows, coef, counts, tokens, prob_sum, loss);
        return launch_status();
    };
    constexpr std::integral_constant<int, 64> narrow;
    constexpr std::integral_constant<int, 256> small;
    constexpr std::integral_constant<int, 1024> large;
    if (cut.records / groups > 16) return join(large, std::integral_constant<int, kTile>(), (unsigned)balance_tiles(E));
    if (E <= kTile) return join(small, std::integral_constant<int, kTile>(), 1);
    if (E <= 64) return join(small, narrow, 1);
    if (E <= 256 || groups >= 1 << 22) return join(small, small, 1);
    return join(large, large, 1);
}

extern "C" int railsched_route_balance_backward(const void *logits, int32_t dtype, int64_t rows, int32_t E, int64_t ld, const uint8_t *row_mask,
                                                int32_t k, const int64_t *group_off, int32_t groups, float coef, const int64_t *counts,
                                                const int64_t *tokens, const float *d_loss, int32_t accumulate, void *d_logits,
                                                int64_t ld_d, void *stream)
{
    using namespace rs;
    if (int rc = check_router(logits, dtype, rows, E, ld, 1.0f)) return rc;
    if (int rc = check_gradient(logits, d_logits, rows, E, ld_d, accumulate == 2 ? 0 : accumulate)) return rc;
    if (k < 1 || k > E) return RAILSCHED_ERR_INVALID_ARG;
    if (int rc = check_groups(rows, group_off, groups)) return rc;
    const bool clear = accumulate == 2 && group_off;
    if (rows == 0 || (groups == 0 && !clear)) return RAILSCHED_OK;
    if (groups > 0 && (!counts || !tokens || !d_loss)) return RAILSCHED_ERR_NULL_PTR;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const Groups gr = make_groups(rows, group_off, groups);
    return by_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        return by_shape<true, T>(E, [&](auto s) {
            using S = decltype(s);
            const int slice_rows = gradient_slice_rows(rows, (int)sizeof(T) * E, 256 / S::LANES);
            auto go = [&](auto parts) {
                hipLaunchKernelGGL((route_balance_backward_kernel<T, S::LANES, S::VPL, S::VEC, decltype(parts)::value>), row_grid(rows, slice_rows), dim3(256), 0, st,
                                   static_cast<const T *>(logits), E, ld, row_mask, k, gr, slice_rows, coef, counts, tokens, d_loss, accumulate == 1,
                                   clear, static_cast<T *>(d_logits), ld_d);
                return launch_status();
            };
            return S::VEC && E % 4 != 0 ? go(std::integral_constant<bool, S::VEC>()) : go(std::false_type());
        });
    });
}
