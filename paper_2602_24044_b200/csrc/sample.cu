// The next token of every request from its row of logits: temperature, top-k, min-p, top-p, a given number.
//
// w_i = exp((l_i - m) / tau), m the row's largest; tokens are ordered by l, ties by the lower index; kept are
// the first k, of these the ones with w_i >= min_p, of these the shortest run from the front whose weight
// reaches top_p of theirs; the token is the lowest index at which the kept weights so far exceed u times their
// sum.  A row is read once: the time should be the logits' way from memory.
//
// What is kept hangs on borders (a sum of thousands of weights against p times another), and a token on where
// u falls among as many: weights are good to 1e-11 and sums are held in fp64 or in whole numbers of 64 bits (candidates)
// and 96 (a whole vocabulary's).  A weight below 2^-46 counts as nothing, but for the sums of all that the first
// reading takes: it does not know the largest value yet.
// 2^t is a table of 64 powers and a polynomial of degree 3 in fp64 (7 fp64 instructions a weight, which issue
// at half the rate of fp32's; a polynomial alone would be 12).  The table is there once for each pair of
// banks, so that lanes with different entries do not wait for one another.
//
// A cluster of blocks takes a row, in steps of 2 KB a warp.  Rows with a filter collect candidates in shared memory:
// whatever is not below a threshold that only rises (one that K values so far are not below, or min_p of the largest
// so far); K = top_k, or KEEP_P for top_p alone, where the sum of all weights is taken on the way.  The first block
// picks from what is left at the end.  Rows without a filter only sum, a step's sum by itself: the token's step is looked
// up among the sums and read again.  What does not fit (top_k over KEEP_K, a nucleus of thousands) is found with two
// more readings of the row, which the second-level cache has in part: band_row.  What does not fit there either
// (thousands of ties) takes a reading for each digit of the cut: general_row.
//
// 256 rows of 128000 fp32 (131 MB, 20 us at a copy's rate): greedy 31 us, top_k 50 46, top_k 200 64, min_p 0.1 40,
// temperature alone 45, all kinds together with 30 or so wide nuclei 124.  512 rows of 150001 bf16, temperature
// alone: 94 us, 22 instructions a value.  4 rows of 32000: 8 us (greedy) .. 23 (top_k 200), with a nucleus of
// thousands or a top_k over 256 among them 38 .. 47.
#include <cooperative_groups.h>

#include <cfloat>
#include <cmath>
#include <type_traits>

#include "fused_ptx.cuh"
#include "kv_common.cuh"

namespace lora {

namespace cg = cooperative_groups;

constexpr int SP_THREADS = 256, SP_WARPS = SP_THREADS / 32;
constexpr int SP_CLUSTER = 8;                 // blocks of a row at most
constexpr int SP_LIST = 2048;                 // entries of a list
constexpr int SP_STAGES = 4, SP_BLOCKS = 2;   // steps of a warp in shared memory; blocks on an SM
constexpr int KEEP_K = 256, KEEP_P = 64;      // what a list is kept to at most by rank, and where top_p alone asks for one
constexpr int SP_SUM_BLOCKS = 4;              // blocks of sample_sum_kernel on an SM
constexpr int SP_REST = 8;                    // blocks of a row in the second launch
constexpr int SP_BINS = 2048;                 // of the band path: 64 to a power of two below the largest
constexpr int SP_MAX_V = (1 << 20) - 8;       // a row's steps have their sums in a list
constexpr double SP_LOW = -46.0;              // a weight below 2^-46 counts as nothing
// Sums nearer to each other than this, of themselves, count as equal: the weights' errors leave no more, and among equal
// logits borders do fall together (half of two equal weights is the first of them, not a little more).
constexpr double SP_SAME = 1.0 / (1ll << 34);
constexpr double SP_ONE = 70368744177664.0;   // 2^46: the largest weight as a whole number
constexpr double SP_MAGIC = 105553116266496.0;   // 1.5 * 2^46: sums with it are rounded to 1/64

struct SampleQueue {             // rows for the second launch
    int32_t count, next, done, reserved;
    struct Row {
        int32_t row;
        float max;
        double total;
    } rows[1];
};

struct SampleParams {
    const void *logits;
    int64_t ld;
    int32_t R, V, segs, steps;   // rows, their values; steps of 2 KB in a row, and of one warp
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t *top_k;
    int32_t *token;
    float *logprob;
    SampleQueue *queue;          // or NULL
};

// what a row asks for
struct RowPlan {
    double c;                    // log2(e) / temperature
    double low;                  // smallest exponent that min_p keeps, -inf: all
    float drop;                  // min_p: how far below the largest so far candidates may be
    float u;
    double p;
    int32_t k;                   // 0: all
    int32_t keep;                // entries that a list is cut to; 0: not by rank
    bool greedy, by_p, by_min, list, sums, segments;
};

// A sum of weights of a whole vocabulary, 2^20 of them at most: in units of 2^-43 (so 2^63 is the most there can be) and, what
// is left beside these, of 2^-75.
struct Exact {
    uint64_t units, rest;
    __device__ __forceinline__ double value() const { return fma((double)units, 4294967296.0, (double)rest); }   // in units of 2^-75
    __device__ __forceinline__ Exact operator+(const Exact &o) const { return {units + o.units, rest + o.rest}; }
};

struct SampleShared {
    RowPlan plan;
    double table[64 * 16];       // 2^(i / 64), once for each pair of banks
    uint32_t bins[256];
    uint64_t scan_u[SP_WARPS];
    double scan_d[SP_WARPS];
    int32_t n, failed_here;
    uint32_t threshold, best;    // what candidates are not below, and the block's largest so far, as keys
    uint32_t begin;              // the largest of its first steps: what sums are taken against, so nothing raises it later
    uint32_t warp_threshold[4][SP_WARPS];    // for m = 8, 4, 2, 1
    uint32_t key_min, key_max;
    int32_t pick_bin, pick_above, pick_kept;
    uint64_t pick_count, pick_here;
    Exact pick_weight;
    int32_t found;
    double rest;
    // written by the blocks of the cluster to the first one
    uint32_t top[SP_CLUSTER], cut[SP_CLUSTER];
    int32_t bad[SP_CLUSTER], failed[SP_CLUSTER];
    double sum[SP_CLUSTER], above[SP_CLUSTER];
    int32_t merged;
    // of the first block: what turns the blocks' sums into sums against the largest value
    double scale[SP_CLUSTER];
    // written by the first block to all
    int32_t general, k_bin, p_first, p_last;
    float row_max;
    double total;                // of all weights, NaN where the row was not summed
    // (from here on not for sample_sum_kernel)
    alignas(16) uint64_t list[SP_LIST];     // candidates; sums of steps; weights
    uint64_t merge[SP_LIST];     // (first block) the cluster's candidates; sums of all steps
    union {
        uint4 ring[SP_WARPS][SP_STAGES][4][32];   // steps on their way from memory
        struct {                                  // general path
            uint32_t digit_weight[2][256][3];         // in units of 2^-75
            uint32_t digit_count[2][256];
        };
        struct {                                  // (first block) band path: of the whole row
            double bin_weight[SP_BINS];
            uint32_t bin_count[SP_BINS];
        };
        double step_sums[SP_LIST];                // (first block) band path: the sums of all steps
    };
};

// ---- values, keys -----------------------------------------------------------------------------
__device__ __forceinline__ uint32_t key_of(float l) {          // larger value, larger key; -0 and 0 alike
    const uint32_t u = __float_as_uint(__fadd_rn(l, 0.0f));
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ uint64_t entry_of(float l, int32_t i) { return (uint64_t)key_of(l) << 32 | (uint32_t)~i; }
__device__ __forceinline__ int32_t index_of(uint64_t entry) { return (int32_t)~(uint32_t)entry; }
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// 2^(x c - b) with magic = SP_MAGIC - b (b a multiple of 1/64): the nearest 1/64 from a rounded sum, the rest by
// the exponential series to the third power.  Its fourth term is a4 r^4 with |r| <= h = 1/128; the square's
// coefficient has 2 (sqrt 2 - 1) a4 h^2 more, which leaves 6.1e-12 of it at most (not 3.6e-11).
__device__ __forceinline__ double power2(double x, double c, double magic, const double *table) {
    const double t = fma(x, c, magic);
    const int32_t k = __double2loint(t);
    const double r = fma(x, c, -(t - magic));
    const double p = fma(r, fma(r, fma(r, 0.05550410866482158, 0.24022699328228442), 0.6931471805599453), 1.0);
    const double e = table[(k & 63) * 16 + (threadIdx.x & 15)];
    return p * __hiloint2double(__double2hiint(e) + ((k & ~63) << 14), __double2loint(e));
}
// the weight of a value against the row's largest
__device__ __forceinline__ double exponent_of(float l, float m, double c) {
    return l == m ? 0.0 : ((double)l - (double)m) * c;
}
__device__ __forceinline__ double weight_of(double t, const double *table) {
    return t >= SP_LOW ? power2(t, 1.0, SP_MAGIC, table) : 0.0;        // (not a number: nothing)
}
__device__ __forceinline__ uint64_t whole(double w) { return (uint64_t)(w * SP_ONE); }

// Adds a weight to a sum of three words in shared memory, whose carries each go with the addition that made them.  (An
// addition of 64 bits there is a loop in which lanes with one sum wait for one another: with two of them a row of 128000
// equal logits took 4450 us for 311, one at a temperature of 100 1100 for 207.)
__device__ __forceinline__ void add_weight(uint32_t *sum, double w) {
    const double units = w * 8796093022208.0;                          // 2^43
    uint64_t u = (uint64_t)units;
    const uint32_t r = (uint32_t)((units - (double)u) * 4294967296.0);
    if (r && atomicAdd(&sum[0], r) + r < r) ++u;
    const uint32_t low = (uint32_t)u;
    uint32_t high = (uint32_t)(u >> 32);
    if (low && atomicAdd(&sum[1], low) + low < low) ++high;
    if (high) atomicAdd(&sum[2], high);
}

__device__ __forceinline__ double nan_value() { return __longlong_as_double(0x7ff8000000000000ll); }

// What the sums of a block (or, in the band path, a row) are taken against: a power of two 2^base next to the weight of
// its largest value `top` so far; values below `low` are taken for it, so that exponents do not leave the numbers.  `c` is
// the row's, but no more than makes neighbouring fp32 numbers around `top` 2^7 apart: values that differ are as good as
// nothing beside the larger one either way, and |top c| stays below 2^31, where `low`, rounded to fp32, is within 2^7.1 of
// the 800 that it is meant to lie below the base.  (With the base at 0 it is as good as exact, and lies 1000 below: the
// first steps may hold no value at all, and what comes then may lie below the base, up to the 900 that sums are turned by.)
struct SumBase {
    double c, base, magic;
    float low;
    __device__ __forceinline__ SumBase() : c(0.0), base(0.0), magic(SP_MAGIC), low(-FLT_MAX) {}
    __device__ __forceinline__ SumBase(float top, double row_c) {
        c = row_c;
        base = rint((double)top * c);
        if (fabs(base) < 1e12) {                                       // a spacing is 2^(e - 150), e the biased exponent
            const int e = max((int)(__float_as_uint(top) >> 23 & 255u), 1);
            c = fmin(c, __hiloint2double((1023 + 157 - e) << 20, 0));
            base = rint((double)top * c);
        } else {
            base = 0.0;
        }
        magic = SP_MAGIC - base;
        low = (float)fmax((base - (base == 0.0 ? 1000.0 : 800.0)) / c, -(double)FLT_MAX);
    }
    __device__ __forceinline__ double weight(float l, const double *table) const {
        return power2((double)fmaxf(l, low), c, magic, table);
    }
    // the exponent of a value against the base: what sums are turned by, if it is not far from it
    __device__ __forceinline__ double above(float l) const { return fma((double)l, c, -base); }
};

struct SampleRow { const char *base; int32_t off, end; };       // see Step::load

// where sample_sum_kernel's steps are in its shared memory, behind the sums
__host__ __device__ inline size_t sum_ring(int32_t segs) {
    return offsetof(SampleShared, list) + ((size_t)segs * 8 + 15) / 16 * 16;
}


// ---- a step: 64 bytes a lane ------------------------------------------------------------------
template <bool BF16>
struct Step {
    static constexpr int VEC = BF16 ? 8 : 4, N = 4 * VEC, SEG = 32 * N;     // values of a vector, a lane, a warp
    static constexpr uint32_t NOTHING = BF16 ? 0xff80ff80u : 0xff800000u;   // -inf
    uint32_t w[16];

    // Places count from the 16-byte boundary at or before the row's first value, which is place `off`: what a vector
    // holds besides the row is masked out (its 16 bytes lie in one piece of memory with a value of the row).
    __device__ __forceinline__ void load(const SampleRow &row, int32_t seg) {
        const char *from = row.base + (int64_t)seg * 2048 + (threadIdx.x & 31) * 16;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int32_t at = seg * SEG + (v * 32 + (int)(threadIdx.x & 31)) * VEC;
            uint4 q = make_uint4(NOTHING, NOTHING, NOTHING, NOTHING);
            if (at < row.end) q = __ldg(reinterpret_cast<const uint4 *>(from + v * 512));
            w[4 * v] = q.x; w[4 * v + 1] = q.y; w[4 * v + 2] = q.z; w[4 * v + 3] = q.w;
        }
        if (seg * SEG < row.off || (seg + 1) * SEG > row.end) mask(row, seg);
    }
    // the same by way of shared memory: a lane's own 64 bytes, asked for ahead
    static __device__ __forceinline__ void ask(const SampleRow &row, int32_t seg, uint4 (*to)[32]) {
        const int lane = threadIdx.x & 31;
        const char *from = row.base + (int64_t)seg * 2048 + lane * 16;
        const uint32_t at = (uint32_t)__cvta_generic_to_shared(&to[0][lane]);
        if ((seg + 1) * SEG <= row.end) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + v * 512), "l"(from + v * 512) : "memory");
        } else {
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (seg * SEG + (v * 32 + lane) * VEC < row.end)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + v * 512), "l"(from + v * 512) : "memory");
        }
    }
    __device__ __forceinline__ void take(const SampleRow &row, int32_t seg, const uint4 (*from)[32]) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const uint4 q = from[v][lane];
            w[4 * v] = q.x; w[4 * v + 1] = q.y; w[4 * v + 2] = q.z; w[4 * v + 3] = q.w;
        }
        if (seg * SEG < row.off || (seg + 1) * SEG > row.end) mask(row, seg);
    }
    __device__ __forceinline__ void mask(const SampleRow &row, int32_t seg) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int32_t at = seg * SEG + (v * 32 + (int)(threadIdx.x & 31)) * VEC;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int32_t lo = at + j * (VEC / 4), hi = lo + VEC / 4 - 1;
                const bool low = lo >= row.off && lo < row.end, high = hi >= row.off && hi < row.end;
                uint32_t &x = w[4 * v + j];
                x = BF16 ? (low ? x & 0xffffu : 0xff80u) | (high ? x & 0xffff0000u : 0xff800000u) : (low ? x : NOTHING);
            }
        }
    }
    // the largest of each vector's values (NaN where there is one)
    __device__ __forceinline__ void tops(float (&top)[4]) const {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const uint32_t *x = w + 4 * v;
            if (BF16) {
                uint32_t a, b;
                asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(x[0]), "r"(x[1]));
                asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(x[2]), "r"(x[3]));
                asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
                top[v] = max_or_nan(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
            } else {
                float a;
                asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(a) : "f"(value(4 * v)), "f"(value(4 * v + 1)), "f"(value(4 * v + 2)));
                top[v] = max_or_nan(a, value(4 * v + 3));
            }
        }
    }
    __device__ __forceinline__ float value(int e) const {
        if (BF16) return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
        return __uint_as_float(w[e]);
    }
    static __device__ __forceinline__ int32_t index(const SampleRow &row, int32_t seg, int e) {
        return seg * SEG - row.off + (e / VEC * 32 + (int)(threadIdx.x & 31)) * VEC + e % VEC;
    }
};

// A warp's steps of a row: every C * SP_WARPS-th of the row's.  The next ones are on their way while f looks at one.
template <bool BF16>
__device__ __forceinline__ void ask_step(SampleShared &s, const SampleParams &P, const SampleRow &row, int C, int rank, int it) {
    const int warp = threadIdx.x >> 5;
    if (it < P.steps) Step<BF16>::ask(row, (it * C + rank) * SP_WARPS + warp, s.ring[warp][it % SP_STAGES]);
    asm volatile("cp.async.commit_group;" ::: "memory");
}
template <bool BF16>
__device__ __forceinline__ void ask_first_steps(SampleShared &s, const SampleParams &P, const SampleRow &row, int C, int rank) {
#pragma unroll
    for (int it = 0; it < SP_STAGES - 1; ++it) ask_step<BF16>(s, P, row, C, rank, it);
}
template <bool BF16, typename F>
__device__ __forceinline__ void read_steps(SampleShared &s, const SampleParams &P, const SampleRow &row, int C, int rank, F f) {
    const int warp = threadIdx.x >> 5;
    for (int it = 0; it < P.steps; ++it) {
        const int32_t seg = (it * C + rank) * SP_WARPS + warp;
        ask_step<BF16>(s, P, row, C, rank, it + SP_STAGES - 1);     // (where the step before this one was)
        asm volatile("cp.async.wait_group %0;" ::"n"(SP_STAGES - 1) : "memory");
        Step<BF16> x;
        x.take(row, seg, s.ring[warp][it % SP_STAGES]);
        f(x, seg, it);
    }
}

// A cluster of one block needs no more than the block's barrier.
__device__ __forceinline__ void cluster_sync(cg::cluster_group &cluster, int C) {
    if (C == 1) __syncthreads(); else cluster.sync();
}

// ---- block-wide sums --------------------------------------------------------------------------
// What lies before this thread, and (total) all of it.  Every thread of the block calls it.
template <typename I>
__device__ __forceinline__ I block_before(I v, I *warp_sum, I &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    I incl = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const I o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    __syncthreads();
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    I before = incl - v;
    if (std::is_floating_point<I>::value) {                   // not by a difference
        before = __shfl_up_sync(0xffffffffu, incl, 1);
        if (lane == 0) before = 0;
    }
    total = 0;
    I ahead = 0;
#pragma unroll
    for (int i = 0; i < SP_WARPS; ++i) {
        if (i == warp) ahead = total;
        total += warp_sum[i];
    }
    return ahead + before;
}

// E entries a thread in descending or ascending order (a bitonic network): partners in one thread, by shuffles, and
// only those of other warps through shared memory.  All threads of the block call it.
template <bool DOWN, int E>
__device__ __forceinline__ void sort_blocked(uint64_t *a) {
    const int tid = threadIdx.x;
    uint64_t e[E];
#pragma unroll
    for (int x = 0; x < E; ++x) e[x] = a[tid * E + x];
#pragma unroll 1
    for (int k = 2; k <= SP_THREADS * E; k <<= 1) {
#pragma unroll 1
        for (int d = k / (2 * E); d > 0; d >>= 1) {
            // the larger entry stays in the lower thread of a descending run
            const bool larger = (((tid & d) == 0) == (((tid * E) & k) == 0)) == DOWN;
            if (d >= 32) {
                __syncthreads();
#pragma unroll
                for (int x = 0; x < E; ++x) a[tid * E + x] = e[x];
                __syncthreads();
#pragma unroll
                for (int x = 0; x < E; ++x) {
                    const uint64_t o = a[(tid ^ d) * E + x];
                    e[x] = (e[x] > o) == larger ? e[x] : o;
                }
            } else {
#pragma unroll
                for (int x = 0; x < E; ++x) {
                    const uint64_t o = __shfl_xor_sync(0xffffffffu, e[x], d);
                    e[x] = (e[x] > o) == larger ? e[x] : o;
                }
            }
        }
#pragma unroll
        for (int j = E / 2; j > 0; j >>= 1) {
            if (j < k) {
#pragma unroll
                for (int x = 0; x < E; ++x) {
                    if (x & j) continue;
                    const bool first = (((tid * E + x) & k) == 0) == DOWN;       // the larger one first
                    const uint64_t p = e[x], q = e[x | j];
                    const bool swap = (p < q) == first;
                    e[x] = swap ? q : p;
                    e[x | j] = swap ? p : q;
                }
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < E; ++x) a[tid * E + x] = e[x];
    __syncthreads();
}
// The entries a[0 .. n), n <= SP_LIST, filled up to the size that is sorted, which is returned.
template <bool DOWN>
__device__ __noinline__ int sort_entries(uint64_t *a, int n) {
    const int size = n <= 256 ? 256 : n <= 512 ? 512 : n <= 1024 ? 1024 : 2048;
    for (int i = n + (int)threadIdx.x; i < size; i += SP_THREADS) a[i] = DOWN ? 0 : ~0ull;
    __syncthreads();
    if (size == 256) sort_blocked<DOWN, 1>(a);
    else if (size == 512) sort_blocked<DOWN, 2>(a);
    else if (size == 1024) sort_blocked<DOWN, 4>(a);
    else sort_blocked<DOWN, 8>(a);
    return size;
}

// ---- the list ---------------------------------------------------------------------------------
__device__ __forceinline__ void put(SampleShared &s, uint64_t entry, int most = SP_LIST) {
    const int at = atomicAdd(&s.n, 1);
    if (at < most) s.list[at] = entry;
}

// Leaves the entries whose keys are not below `cut`; returns how many there are.
__device__ __noinline__ int leave_from(SampleShared &s, uint64_t *a, int n, uint32_t cut) {
    const int tid = threadIdx.x;
    uint64_t mine[SP_LIST / SP_THREADS];
#pragma unroll
    for (int j = 0; j < SP_LIST / SP_THREADS; ++j) mine[j] = tid + j * SP_THREADS < n ? a[tid + j * SP_THREADS] : 0;
    __syncthreads();
    if (tid == 0) s.found = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < SP_LIST / SP_THREADS; ++j)
        if (mine[j] && (uint32_t)(mine[j] >> 32) >= cut) a[atomicAdd(&s.found, 1)] = mine[j];
    __syncthreads();
    const int left = s.found;
    __syncthreads();
    return left;
}

// Leaves at least `keep` of the n entries of `a`, the best ones, and as a rule no more than `most`; returns their
// number and the smallest key among them (n < keep: all of them, and 0).  All threads of the block call it.
// The K-th is looked for in 256 equal parts of the values' range, then of the part it is in, and so on: any rule
// that never puts a larger value behind a smaller one is right, so roundings, infinities and ties only make the
// parts uneven.
__device__ __noinline__ int cut_list(SampleShared &s, uint64_t *a, int n, int keep, int most, uint32_t &cut) {
    cut = 0;
    if (n < keep) return n;
    const int tid = threadIdx.x, lane = tid & 31;
    uint32_t lo = 0, hi = 0xffffffffu;
    int above = 0, kept = n;
    uint32_t *bins = s.bins;
    for (int round = 0; round < 8; ++round) {
        __syncthreads();
        if (tid == 0) { s.key_min = 0xffffffffu; s.key_max = 0; }
        bins[tid] = 0;
        __syncthreads();
        uint32_t mn = 0xffffffffu, mx = 0;
        for (int i = tid; i < n; i += SP_THREADS) {
            const uint32_t k = (uint32_t)(a[i] >> 32);
            if (k >= lo && k <= hi) { mn = min(mn, k); mx = max(mx, k); }
        }
        mn = __reduce_min_sync(0xffffffffu, mn);
        mx = __reduce_max_sync(0xffffffffu, mx);
        if (lane == 0) { atomicMin(&s.key_min, mn); atomicMax(&s.key_max, mx); }
        __syncthreads();
        const float top = 0.5f * fminf(value_of(s.key_max), FLT_MAX), bottom = 0.5f * fmaxf(value_of(s.key_min), -FLT_MAX);
        const float scale = 256.0f / (top - bottom);
        auto bin = [&](uint32_t k) {
            return min(255, max(0, (int)((top - 0.5f * fminf(value_of(k), FLT_MAX)) * scale)));
        };
        for (int i = tid; i < n; i += SP_THREADS) {
            const uint32_t k = (uint32_t)(a[i] >> 32);
            if (k >= lo && k <= hi) atomicAdd(&bins[bin(k)], 1u);
        }
        __syncthreads();
        if (tid < 32) {
            uint32_t c[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += c[i] = bins[lane * 8 + i];
            uint32_t incl = sum;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t o = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += o;
            }
            int before = above + (int)(incl - sum);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (before < keep && before + (int)c[i] >= keep) {
                    s.pick_bin = lane * 8 + i;
                    s.pick_above = before;
                    s.pick_kept = before + (int)c[i];
                }
                before += (int)c[i];
            }
            if (lane == 0) { s.key_min = 0xffffffffu; s.key_max = 0; }
        }
        __syncthreads();
        const int b = s.pick_bin;
        mn = 0xffffffffu, mx = 0;
        for (int i = tid; i < n; i += SP_THREADS) {
            const uint32_t k = (uint32_t)(a[i] >> 32);
            if (k >= lo && k <= hi && bin(k) == b) { mn = min(mn, k); mx = max(mx, k); }
        }
        mn = __reduce_min_sync(0xffffffffu, mn);
        mx = __reduce_max_sync(0xffffffffu, mx);
        if (lane == 0) { atomicMin(&s.key_min, mn); atomicMax(&s.key_max, mx); }
        __syncthreads();
        lo = cut = s.key_min;
        hi = s.key_max;
        above = s.pick_above;
        kept = s.pick_kept;
        if (kept <= most || lo == hi) break;
    }
    return leave_from(s, a, n, cut);
}

// A threshold that `keep` values of the block's at least are not below: a lane holds the largest so far of either
// half of its steps, a warp takes the (keep / m)-th of its 64 for m = 8, 4, 2, 1, and the m-th largest of the warps'
// counts, whichever m gives most.  (The lowest of the eight alone, m = 8, was none where a warp had no values: 256
// greedy rows took 39 us for 11 with 4096 of bf16, a block's eight warps having four steps, and 335 for 38 with
// 128000 of fp32 and the first 1024 masked.)  It rises with the steps: as many values again pass it in steps 2 .. 3
// as in 1, in 4 .. 7 as in 2 .. 3, ..
__device__ __forceinline__ void warp_threshold(SampleShared &s, const RowPlan &R, float top0, float top1) {
    const int lane = threadIdx.x & 31;
    const uint32_t k0 = top0 == top0 ? key_of(top0) : 0u, k1 = top1 == top1 ? key_of(top1) : 0u;
    // the 64 in descending order, two neighbours a lane
    uint32_t a = (lane & 1) ? min(k0, k1) : max(k0, k1), b = (lane & 1) ? max(k0, k1) : min(k0, k1);
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1) {
#pragma unroll
        for (int j = k >> 1; j; j >>= 1) {
            const uint32_t oa = __shfl_xor_sync(0xffffffffu, a, j), ob = __shfl_xor_sync(0xffffffffu, b, j);
            const bool larger = ((lane & k) == 0) == ((lane & j) == 0);
            a = larger ? max(a, oa) : min(a, oa);
            b = larger ? max(b, ob) : min(b, ob);
        }
        const bool first = (lane & k) == 0;
        const uint32_t x = max(a, b), y = min(a, b);
        a = first ? x : y;
        b = first ? y : x;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int m = SP_WARPS >> j, want = (R.keep + m - 1) / m - 1;
        const uint32_t mine = __shfl_sync(0xffffffffu, (want & 1) ? b : a, (want >> 1) & 31);
        if (lane == 0) s.warp_threshold[j][threadIdx.x >> 5] = want < 64 ? mine : 0u;
    }
}
__device__ __forceinline__ uint32_t block_threshold(const SampleShared &s) {      // (by whole warps)
    const int lane = threadIdx.x & 31, m = SP_WARPS >> (lane >> 3);
    const uint32_t mine = (&((volatile const SampleShared &)s).warp_threshold[0][0])[lane];
    int from = 1;                          // (where nothing is kept by rank all of them are 0)
#pragma unroll
    for (int i = 1; i < SP_WARPS; ++i) from += __shfl_xor_sync(0xffffffffu, mine, i) >= mine ? 1 : 0;
    return max(__reduce_max_sync(0xffffffffu, from >= m ? mine : 0u), *(volatile const uint32_t *)&s.threshold);
}

// The values of a step that are not below t: a lane takes its places at once.
template <bool BF16>
__device__ __forceinline__ void put_step(SampleShared &s, const SampleRow &row, const Step<BF16> &x, const float (&vec)[4],
                                         int32_t seg, float t) {
    using S = Step<BF16>;
    uint32_t in = 0;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        if (vec[v] >= t) {
#pragma unroll
            for (int e = v * S::VEC; e < (v + 1) * S::VEC; ++e) in |= x.value(e) >= t ? 1u << e : 0u;
        }
    }
    int at = atomicAdd(&s.n, __popc(in));
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        if (in >> (v * S::VEC) & ((1u << S::VEC) - 1u)) {
#pragma unroll
            for (int e = v * S::VEC; e < (v + 1) * S::VEC; ++e)
                if (in >> e & 1u) {
                    if (at < SP_LIST) s.list[at] = entry_of(x.value(e), S::index(row, seg, e));
                    ++at;
                }
        }
    }
}

// A list that fills up: what the threshold as it is now leaves of it, or (by rank) the best ones.  s.n is its length
// afterwards; s.failed_here where it is still nearly full, or where entries had no place.
__device__ __noinline__ void shorten(SampleShared &s, const RowPlan &R) {
    const bool lost = s.n > SP_LIST;
    uint32_t cut = block_threshold(s);
    int n = leave_from(s, s.list, min(s.n, SP_LIST), cut);
    if (R.keep && n > SP_LIST / 2) n = cut_list(s, s.list, n, R.keep, SP_LIST / 4, cut);
    if (threadIdx.x == 0) {
        s.n = n;
        s.threshold = max(s.threshold, cut);
        if (lost || n > SP_LIST * 3 / 4) s.failed_here = 1;
    }
    __syncthreads();
}

// ---- finding the token ------------------------------------------------------------------------
__device__ __forceinline__ void answer(const SampleParams &P, int64_t r, int32_t token, double logprob) {
    P.token[r] = token;
    if (P.logprob) P.logprob[r] = (float)logprob;
}

// The first block, from the cluster's candidates.  False where they do not hold the whole of what is kept.
//
// Up to half a block of candidates, everything is counted: how many candidates are in front of one and what they weigh
// says whether it is kept, what the kept ones of lower index weigh whether u falls on it.  Two or four neighbouring
// threads count for one candidate.
__device__ bool count_candidates(SampleShared &s, const SampleParams &P, const RowPlan &R, int64_t row, float m, double all,
                                 int n) {
    const int tid = threadIdx.x, log_g = n <= 64 ? 2 : 1, g = 1 << log_g, part = tid & (g - 1), me = tid >> log_g;
    ulonglong2 *const pair = reinterpret_cast<ulonglong2 *>(s.list);         // n <= SP_THREADS / 2
    const uint64_t mine = me < n ? s.merge[me] : 0;
    uint64_t w = 0;
    if (me < n) {
        const double t = exponent_of(value_of((uint32_t)(mine >> 32)), m, R.c);
        if (t >= R.low) w = whole(weight_of(t, s.table));
    }
    if (part == 0) pair[me] = make_ulonglong2(mine, w);
    __syncthreads();
    int rank = 0;
    uint64_t before = 0;
    const int rounds = (n + 8 * g - 1) / (8 * g);          // (there are SP_THREADS / g entries, those from n on nothing)
    for (int j = 0; j < rounds; ++j) {
        ulonglong2 o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = pair[(j * 8 + i) * g + part];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (o[i].x > mine) {
                ++rank;
                before += o[i].y;
            }
    }
    for (int d = 1; d < g; d <<= 1) {
        rank += __shfl_xor_sync(0xffffffffu, rank, d);
        before += __shfl_xor_sync(0xffffffffu, before, d);
    }
    // (what is in front of one of the first k is so too, and has a weight that min_p leaves if this one has)
    if (R.k && rank >= R.k) w = 0;
    uint64_t total;
    block_before<uint64_t>(part ? 0 : w, s.scan_u, total);
    if (R.p < 1.0) {
        const double need = R.p * (R.sums ? all : (double)total);
        if (!((double)before < need) && rank > 0) w = 0;
        block_before<uint64_t>(part ? 0 : w, s.scan_u, total);
    }
    const uint32_t index = (uint32_t)index_of(mine);
    if (part == 0) pair[me] = make_ulonglong2(index, w);
    __syncthreads();
    before = 0;
    for (int j = 0; j < rounds; ++j) {
        ulonglong2 o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = pair[(j * 8 + i) * g + part];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((uint32_t)o[i].x < index) before += o[i].y;
    }
    for (int d = 1; d < g; d <<= 1) before += __shfl_xor_sync(0xffffffffu, before, d);
    uint64_t target = (uint64_t)((double)R.u * (double)total);
    if (target >= total) target = total - 1;
    if (part == 0 && w && before <= target && target < before + w)
        answer(P, row, (int32_t)index, log((double)w / (double)total));
    return true;
}

__device__ __noinline__ bool pick_from_list(SampleShared &s, const SampleParams &P, const RowPlan &R, int64_t row, float m,
                                            double all, int n) {
    const int tid = threadIdx.x;
    if (R.k == 1) {
        uint64_t best = 0;
        for (int i = tid; i < n; i += SP_THREADS) best = max(best, s.merge[i]);
        if (tid == 0) s.pick_here = 0;
        __syncthreads();
        if (best) atomicMax(reinterpret_cast<unsigned long long *>(&s.pick_here), (unsigned long long)best);
        __syncthreads();
        if (tid == 0) answer(P, row, index_of(s.pick_here), 0.0);
        return true;
    }
    uint32_t cut = 0;
    if (R.sums) {
        // below the highest of the blocks' thresholds the candidates have gaps (among the first k of all they have none)
        for (int i = 0; i < (int)cg::this_cluster().num_blocks(); ++i) cut = max(cut, s.cut[i]);
        n = leave_from(s, s.merge, n, cut);
        // do they reach top_p of all?
        uint64_t sum = 0, reach;
        for (int i = tid; i < n; i += SP_THREADS)
            sum += whole(weight_of(exponent_of(value_of((uint32_t)(s.merge[i] >> 32)), m, R.c), s.table));
        block_before<uint64_t>(sum, s.scan_u, reach);
        if ((double)reach < R.p * all) return false;
    }
    const int few = R.keep <= SP_THREADS / 3 ? SP_THREADS / 2 : SP_THREADS;
    if (n > few && R.k && R.keep) n = cut_list(s, s.merge, n, R.keep, few, cut);
    if (n <= SP_THREADS / 2) return count_candidates(s, P, R, row, m, all, n);
    // more of them: sorted
    int size = sort_entries<true>(s.merge, n);
    const int per = (size + SP_THREADS - 1) / SP_THREADS, first = tid * per;
    constexpr int MOST = SP_LIST / SP_THREADS;
    uint64_t w[MOST], sum = 0;
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
        const int i = first + j;
        w[j] = 0;
        if (j < per && i < n && (R.k == 0 || i < R.k)) {
            const double t = exponent_of(value_of((uint32_t)(s.merge[i] >> 32)), m, R.c);
            if (t >= R.low) w[j] = whole(weight_of(t, s.table));
        }
        sum += w[j];
    }
    uint64_t total;
    uint64_t before = block_before<uint64_t>(sum, s.scan_u, total);
    if (R.p < 1.0) {
        const double need = R.p * (R.sums ? all : (double)total);
        sum = 0;
        uint64_t at = before;
#pragma unroll
        for (int j = 0; j < MOST; ++j) {
            const uint64_t mine = w[j];
            if (!((double)at < need) && first + j > 0) w[j] = 0;
            at += mine;
            sum += w[j];
        }
        block_before<uint64_t>(sum, s.scan_u, total);
    }
    // what is kept, by index: its place in the order goes along
    uint32_t index[MOST];
    int mine = 0;
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
        if (j < per && w[j]) {
            index[j] = (uint32_t)index_of(s.merge[first + j]);
            ++mine;
        }
    }
    uint64_t all_kept;
    int at = (int)block_before<uint64_t>((uint64_t)mine, s.scan_u, all_kept);
    const int kept = (int)all_kept;
#pragma unroll
    for (int j = 0; j < MOST; ++j)
        if (j < per && w[j]) {
            s.merge[at] = (uint64_t)index[j] << 32 | (uint32_t)at;
            s.list[at++] = w[j];
        }
    __syncthreads();
    size = sort_entries<false>(s.merge, kept);
    uint64_t target = (uint64_t)((double)R.u * (double)total);
    if (target >= total) target = total - 1;
    const int per2 = (size + SP_THREADS - 1) / SP_THREADS, first2 = tid * per2;
    sum = 0;
    for (int j = 0; j < per2; ++j)
        if (first2 + j < kept) sum += s.list[(uint32_t)s.merge[first2 + j]];
    uint64_t whole_sum;
    before = block_before<uint64_t>(sum, s.scan_u, whole_sum);
    if (before <= target && target < before + sum)
        for (int j = 0; j < per2; ++j) {
            if (first2 + j >= kept) break;
            const uint64_t e = s.merge[first2 + j], we = s.list[(uint32_t)e];
            if (target < before + we) {
                answer(P, row, (int32_t)(e >> 32), log((double)we / (double)total));
                break;
            }
            before += we;
        }
    return true;
}

// The first block, from the sums of the row's steps; w(value, index) is the weight of a value again.
template <bool BF16, typename W>
__device__ __noinline__ void pick_from_sums(SampleShared &s, const SampleParams &P, const RowPlan &R, int64_t row, const SampleRow &logits,
                               const double *sums, W w) {
    constexpr int SEG = Step<BF16>::SEG, PER = SP_LIST / SP_THREADS, MINE = SEG / SP_THREADS;
    const int tid = threadIdx.x;
    const int per = (P.segs + SP_THREADS - 1) / SP_THREADS;
    double mine[PER], sum = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        mine[j] = j < per && tid * per + j < P.segs ? sums[tid * per + j] : 0.0;
        sum += mine[j];
    }
    double total;
    double before = block_before<double>(sum, s.scan_d, total);
    const double target = (double)R.u * total * (1.0 + SP_SAME);
    if (tid == 0) { s.found = P.segs; s.rest = 0.0; }
    __syncthreads();
    bool here = false;
    int seg = P.segs;
    double rest = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (!here && mine[j] > 0.0 && target < before + mine[j]) {
            here = true;
            seg = tid * per + j;
            rest = target - before;
        }
        before += mine[j];
    }
    if (here) atomicMin(&s.found, seg);
    __syncthreads();
    if (here && s.found == seg) s.rest = rest;
    __syncthreads();
    seg = s.found;
    rest = s.rest;
    // The step at which the sums pass the target; should it hold nothing to draw (the target on a border), the
    // next that does, and behind the last one the last that does.
    int step = seg < P.segs ? 1 : -1;
    if (step < 0) seg = P.segs - 1;
    for (bool begun = false; seg >= 0;) {
        const int32_t at = seg * SEG + tid * MINE - logits.off;
        double x[MINE], own = 0.0;
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            x[j] = 0.0;
            if (at + j >= 0 && at + j < P.V) {
                const char *from = logits.base + (int64_t)(at + j + logits.off) * (BF16 ? 2 : 4);
                const float l = BF16 ? __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t *>(from)) << 16)
                                     : __ldg(reinterpret_cast<const float *>(from));
                x[j] = w(l, at + j);
            }
            own += x[j];
        }
        double here_total;
        const double ahead = block_before<double>(own, s.scan_d, here_total);
        if (tid == 0) s.found = step > 0 ? 0x7fffffff : -1;
        __syncthreads();
        if (here_total > 0.0) {
            // the lowest index that passes the rest; where none does by a rounding, or behind the end: the last one
            const double limit = step < 0 ? INFINITY : begun ? 0.0 : rest;
            double run = ahead;
            int32_t first = -1, last = -1;
#pragma unroll
            for (int j = 0; j < MINE; ++j) {
                run += x[j];
                if (x[j] > 0.0) {
                    if (first < 0 && run > limit) first = at + j;
                    last = at + j;
                }
            }
            if (step > 0 && first >= 0) atomicMin(&s.found, first);
            __syncthreads();
            if (step < 0 || s.found == 0x7fffffff) {
                __syncthreads();
                if (tid == 0) s.found = -1;
                __syncthreads();
                if (last >= 0) atomicMax(&s.found, last);
                __syncthreads();
            }
            const int32_t token = s.found;
#pragma unroll
            for (int j = 0; j < MINE; ++j)
                if (token == at + j) answer(P, row, token, log(x[j] / total));
            return;
        }
        begun = true;
        seg += step;
        if (seg >= P.segs) { seg = P.segs - 1; step = -1; }
        __syncthreads();
    }
}

// ---- the band path ----------------------------------------------------------------------------
// Where the candidates were not enough: how many values and how much weight lie in each 1/64 of a power of two
// below the largest says in which of these the first k end, and (weights to 2^-17, a little room at both sides)
// top_p of them.  The row is read once for that and once more for the values of those bands themselves, with the
// exact weight before them: sorted, they give the cut.  False (the same in the whole cluster) where a band is too
// wide for a list, or where the exact sums do not confirm it: so it is where over 65535 values of a block fall into one
// band, whose sum of weights (2^16 each) has 32 bits.
template <bool BF16>
__device__ __noinline__ bool band_row(SampleShared &s, cg::cluster_group &cluster, const SampleParams &P, const RowPlan &R,
                                      int64_t row, const SampleRow &logits) {
    using S = Step<BF16>;
    constexpr int PER = SP_BINS / SP_THREADS, MOST_SUMS = 512, MOST_BAND = SP_LIST - MOST_SUMS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const float m = s.row_max, c_bins = (float)(R.c * (64.0 / (SP_BINS - 1)));
    if (!(R.c > 1e-30) || !(fabsf(m) <= FLT_MAX) || P.steps * SP_WARPS > MOST_SUMS || !(R.k || R.by_p || R.by_min)) return false;
    // A value's place below the largest, as a part of all bins, and the nearest bin, each 1/64 of a power of two; the last
    // one is all the rest, masked tokens too.  (2^23 and a small number is the nearest whole one in the low bits: no
    // conversions, which issue at an eighth of the rate.  The place is clamped at both ends: in the second launch the largest
    // comes from the caller's memory, and a value above it would have no bin.)
    auto place = [&](float l) { return __saturatef((m - l) * c_bins); };
    auto near_bin = [&](float f) { return fmaf(f, (float)(SP_BINS - 1), 8388608.0f); };
    auto bin_of = [&](float l) { return __float_as_int(near_bin(place(l))) - 0x4b000000; };
    // (weights of a quarter of (1 - p) S / V, S that of all, make up less of it than top_p leaves out, all together: the
    // cut is in front of them.  An atomic addition in shared memory takes a cycle a lane, which is what this reading takes.)
    const bool known = s.total == s.total;
    const float last = R.by_min ? fminf((float)(-R.low * (64.0 / (SP_BINS - 1))), 1e30f)
                       : known && R.by_p ? 64.0f / (SP_BINS - 1) * log2f((float)(4.0 * P.V / ((1.0 - R.p) * s.total))) : INFINITY;
    const bool by_k = R.k != 0, by_p = R.by_p;
    uint32_t *const counts = reinterpret_cast<uint32_t *>(s.list), *const weights = counts + SP_BINS;
    ask_first_steps<BF16>(s, P, logits, C, rank);
    for (int i = tid; i < 2 * SP_BINS; i += SP_THREADS) counts[i] = 0;
    __syncthreads();
    read_steps<BF16>(s, P, logits, C, rank, [&](const S &x, int32_t, int) {
#pragma unroll
        for (int e = 0; e < S::N; ++e) {
            const float f = place(x.value(e)), whole_f = near_bin(f);
            const int b = __float_as_int(whole_f) - 0x4b000000;
            if (by_k) atomicAdd(&counts[b], 1u);
            // 2^(-r / 64) of the rest |r| <= 1/2, to its square
            const float r = fmaf(f, (float)(SP_BINS - 1), 8388608.0f - whole_f);
            if (by_p && f <= last)
                atomicAdd(&weights[b], __float_as_uint(fmaf(r, fmaf(r, 3.843576f, -709.7827f), 65536.0f) + 8388608.0f) - 0x4b000000u);
        }
    });
    cluster_sync(cluster, C);
    SampleShared &first = *cluster.map_shared_rank(&s, 0);
    for (int b = rank * (SP_BINS / C) + tid; b < (rank + 1) * (SP_BINS / C); b += SP_THREADS) {
        uint32_t count = 0;
        uint64_t weight = 0;
        for (int r = 0; r < C; ++r) {
            const uint32_t *from = cluster.map_shared_rank(counts, r);
            count += from[b];
            weight += from[SP_BINS + b];
        }
        first.bin_count[b] = count;
        first.bin_weight[b] = (double)weight * power2(-b / 64.0, 1.0, SP_MAGIC, s.table);
    }
    cluster_sync(cluster, C);
    uint64_t before_k = 0;                     // (first block) values in front of the band in which the first k end
    if (rank == 0) {
        double weight[PER], weighed = 0.0;
        uint64_t counted = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            counted += s.bin_count[tid * PER + j];
            weight[j] = s.bin_weight[tid * PER + j];
            weighed += weight[j];
        }
        uint64_t all_counted;
        double all_weighed;
        uint64_t at = block_before<uint64_t>(counted, s.scan_u, all_counted);
        const double ahead = block_before<double>(weighed, s.scan_d, all_weighed);
        if (tid == 0) {
            s.k_bin = s.p_first = s.p_last = SP_BINS;
            s.rest = known ? 65536.0 * s.total : all_weighed;
            s.pick_count = 0;
            s.merged = 0;
        }
        __syncthreads();
        double run = ahead;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const uint64_t count = s.bin_count[tid * PER + j];
            if (by_k && at < (uint64_t)R.k && at + count >= (uint64_t)R.k) {
                s.k_bin = tid * PER + j;
                s.pick_count = at;
                s.rest = run + weight[j] * ((double)(R.k - (int64_t)at) / (double)count);
            }
            at += count;
            run += weight[j];
        }
        __syncthreads();
        before_k = s.pick_count;
        if (by_p) {
            const double near = R.p * s.rest;
            run = ahead;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                run += weight[j];
                if (weight[j] > 0.0 && run >= near * (1.0 - 2e-5)) atomicMin(&s.p_first, tid * PER + j);
                if (weight[j] > 0.0 && run >= near * (1.0 + 2e-5)) atomicMin(&s.p_last, tid * PER + j);
            }
        }
        __syncthreads();
        const int k_bin = s.k_bin, p_first = by_p ? min(s.p_first, k_bin) : k_bin, p_last = by_p ? min(s.p_last, k_bin) : k_bin;
        const bool none = (by_k && k_bin >= SP_BINS - 1) || (by_p && p_last >= SP_BINS - 1);
        __syncthreads();
        if (tid < C) {
            SampleShared &to = *cluster.map_shared_rank(&s, tid);
            to.k_bin = k_bin;
            to.p_first = p_first;
            to.p_last = p_last;
            to.general = none;
        }
    }
    cluster_sync(cluster, C);
    if (s.general) return false;
    const int k_bin = s.k_bin, p_first = s.p_first, p_last = s.p_last;
    ask_first_steps<BF16>(s, P, logits, C, rank);
    if (tid == 0) s.n = 0;
    __syncthreads();
    double *const sums = reinterpret_cast<double *>(s.list) + MOST_BAND;
    // weights as in the first reading: against the power of two next to the largest, turned into weights against it at
    // the end (what min_p leaves is decided by the exact exponent)
    const SumBase B(m, R.c);
    const double turn = exp2(-B.above(m));
    const bool far = !(fabs(B.above(m)) < 1.0), by_min = R.by_min;
    double between = 0.0;                      // where the weight of all is not known: what is behind top_p's band and in front of that of the first k
    read_steps<BF16>(s, P, logits, C, rank, [&](const S &x, int32_t seg, int it) {
        double sum = 0.0, rest = 0.0;
        uint32_t in_band = 0;
#pragma unroll
        for (int e = 0; e < S::N; ++e) {
            const float l = x.value(e);
            const int b = bin_of(l);
            double w = B.weight(l, s.table);
            if (by_min && !(exponent_of(l, m, R.c) >= R.low)) w = 0.0;
            sum += b < p_first ? w : 0.0;
            if (!known) rest += b > p_last && b < k_bin ? w : 0.0;
            if (b >= p_first && (b <= p_last || b == k_bin)) in_band |= 1u << e;
        }
        between += rest;
        if (in_band) {
#pragma unroll
            for (int e = 0; e < S::N; ++e)
                if (in_band >> e & 1u) put(s, entry_of(x.value(e), S::index(logits, seg, e)), MOST_BAND);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) sums[it * SP_WARPS + warp] = sum * turn;
    });
    between *= turn;
    double block_between;
    block_before<double>(between, s.scan_d, block_between);
    const int n = s.n;
    cluster_sync(cluster, C);                            // (the ring's memory is the candidates' again)
    if (tid == 0) {
        s.found = n ? atomicAdd(&first.merged, n) : 0;
        first.sum[rank] = block_between;
        first.failed[rank] = far || n > MOST_BAND || s.found + n > SP_LIST;
    }
    __syncthreads();
    for (int i = tid; i < min(n, MOST_BAND) && s.found + i < SP_LIST; i += SP_THREADS) first.merge[s.found + i] = s.list[i];
    cluster_sync(cluster, C);
    if (rank == 0) {
        bool failed = false;
        double behind = 0.0;
        for (int i = 0; i < C; ++i) {
            failed = failed || s.failed[i];
            behind += s.sum[i];
        }
        double *const all = s.step_sums;
        double front = 0.0;
        for (int g = tid; g < P.segs; g += SP_THREADS) {
            const int r = g / SP_WARPS % C;
            front += all[g] = cluster.map_shared_rank(sums, r)[g / (SP_WARPS * C) * SP_WARPS + g % SP_WARPS];
        }
        double in_front;
        block_before<double>(front, s.scan_d, in_front);
        if (!failed) {
            const int found = s.merged;
            const int size = sort_entries<true>(s.merge, found);
            // entries of the bands: those of top_p's first.  How many are in front of the k-th's band?
            int ahead = 0;
            for (int i = tid; i < found; i += SP_THREADS) ahead += bin_of(value_of((uint32_t)(s.merge[i] >> 32))) < k_bin;
            uint64_t in_p;
            block_before<uint64_t>((uint64_t)ahead, s.scan_u, in_p);
            constexpr int MOST = SP_LIST / SP_THREADS;
            const int per = (size + SP_THREADS - 1) / SP_THREADS, at = tid * per;
            double w[MOST], mine = 0.0, of_p = 0.0;
#pragma unroll
            for (int j = 0; j < MOST; ++j) {
                w[j] = 0.0;
                const int i = at + j;
                if (j < per && i < found) {
                    const float l = value_of((uint32_t)(s.merge[i] >> 32));
                    const int b = bin_of(l);
                    const double t = exponent_of(l, m, R.c);
                    const bool counts_in = b < k_bin || (uint64_t)i - in_p + before_k < (uint64_t)R.k;
                    if (counts_in && t >= R.low) w[j] = weight_of(t, s.table);
                    if (b <= p_last) of_p += w[j];
                }
                mine += w[j];
            }
            double band, p_band;
            const double ahead_of_me = block_before<double>(mine, s.scan_d, band);
            block_before<double>(of_p, s.scan_d, p_band);
            const double need = by_p ? R.p * (known ? s.total : in_front + band + behind) : INFINITY;
            if (by_p) failed = !((in_front < need || p_first == 0) && in_front + p_band >= need);
            if (tid == 0) s.pick_here = ~0ull;
            __syncthreads();
            double run = in_front + ahead_of_me;
#pragma unroll
            for (int j = 0; j < MOST; ++j) {
                const int i = at + j;
                if (j < per && i < found && w[j] > 0.0 && (run < need || (i == 0 && p_first == 0))) {
                    atomicMin(reinterpret_cast<unsigned long long *>(&s.pick_here), (unsigned long long)s.merge[i]);
                    atomicAdd(&all[(index_of(s.merge[i]) + logits.off) / S::SEG], w[j]);
                }
                run += w[j];
            }
            __syncthreads();
            // none of the bands: all in front of them
            const uint64_t cut = s.pick_here != ~0ull ? s.pick_here : found ? s.merge[0] + 1 : 0;
            if (!failed)
                pick_from_sums<BF16>(s, P, R, row, logits, all, [&](float l, int32_t i) {
                    if (!(l > -INFINITY) || entry_of(l, i) < cut) return 0.0;
                    const double t = exponent_of(l, m, R.c);
                    return t >= R.low ? weight_of(t, s.table) : 0.0;
                });
        }
        __syncthreads();
        if (tid < C) cluster.map_shared_rank(&s, tid)->general = failed;
    }
    cluster_sync(cluster, C);
    return !s.general;
}

// ---- the general path -------------------------------------------------------------------------
// What is kept so far: parts of the range before `part`, and of that one the entries from `from` on.
struct SampleCut {
    int32_t part;
    uint64_t from;
    // both are beginnings of one order: what is in both is the shorter of them
    __device__ __forceinline__ SampleCut within(const SampleCut &o) const {
        return part < o.part ? *this : part > o.part ? o : SampleCut{part, max(from, o.from)};
    }
};

struct GeneralRow {
    float m, c32;
    RowPlan R;
    __device__ __forceinline__ int32_t part_of(float l) const {       // quarters of a power of two below the largest
        return l == m ? 0 : min(255, max(0, (int)((m - l) * c32 * 4.0f)));
    }
    __device__ __forceinline__ bool inside(float l, int32_t i, const SampleCut &cut) const {
        if (!(l > -INFINITY)) return false;
        if (cut.part < 256) {
            const int32_t p = part_of(l);
            if (p > cut.part || (p == cut.part && entry_of(l, i) < cut.from)) return false;
        }
        return R.low == -INFINITY || exponent_of(l, m, R.c) >= R.low;
    }
};

// Finds how far the first k (weight: the first ones with p of all weight) of what `cut` keeps reach, a digit of
// eight bits at a time: the part of the range, the key's bytes, the index's.  Every block of the cluster calls it.
template <bool BF16>
__device__ SampleCut general_cut(SampleShared &s, cg::cluster_group &cluster, const SampleParams &P, const GeneralRow &G,
                                 const SampleRow &logits, SampleCut cut, bool weight, int &turn) {
    using S = Step<BF16>;
    const int tid = threadIdx.x, warp = tid >> 5;
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    SampleCut to = {256, 0};
    uint64_t base_count = 0;
    Exact base_weight = {0, 0};
    double need = weight ? 0.0 : (double)G.R.k;
    for (int level = 0; level < 8; ++level) {
        // (a digit's sums are read by the whole cluster while the next one's are taken: two sets in turn)
        uint32_t *const digit_count = s.digit_count[turn];
        uint32_t (*const digit_weight)[3] = s.digit_weight[turn];
        turn ^= 1;
        const int shift = level <= 4 ? 64 - 8 * level : 56 - 8 * level;
        if (level == 5) to.from |= 0xff000000u;          // an index has 24 bits, and stands there as its complement
        digit_count[tid] = 0;
        digit_weight[tid][0] = digit_weight[tid][1] = digit_weight[tid][2] = 0;
        __syncthreads();
        for (int it = 0; it < P.steps; ++it) {
            const int32_t seg = (it * C + rank) * SP_WARPS + warp;
            if (seg >= P.segs) break;
            S x;
            x.load(logits, seg);
#pragma unroll 4
            for (int e = 0; e < S::N; ++e) {
                const float l = x.value(e);
                const int32_t i = S::index(logits, seg, e);
                if (!G.inside(l, i, cut)) continue;
                const int32_t part = G.part_of(l);
                int digit = part;
                if (level > 0) {
                    const uint64_t entry = entry_of(l, i);
                    if (part != to.part) continue;
                    if (level > 1 && (entry >> (shift + 8)) != (to.from >> (shift + 8))) continue;
                    digit = 255 - (int)(entry >> shift & 255u);
                }
                atomicAdd(&digit_count[digit], 1u);
                if (weight) add_weight(digit_weight[digit], weight_of(exponent_of(l, G.m, G.R.c), s.table));
            }
        }
        cluster_sync(cluster, C);
        uint64_t count = 0;
        Exact sum = {0, 0};
        for (int r = 0; r < C; ++r) {
            count += *cluster.map_shared_rank(digit_count + tid, r);
            const uint32_t *w = cluster.map_shared_rank(&digit_weight[tid][0], r);
            sum = sum + Exact{(uint64_t)w[2] << 32 | w[1], w[0]};
        }
        uint64_t counts, units, rests;
        const uint64_t count_before = block_before<uint64_t>(count, s.scan_u, counts);
        Exact sum_before = base_weight;
        if (weight) {
            const uint64_t units_before = block_before<uint64_t>(sum.units, s.scan_u, units);
            sum_before = sum_before + Exact{units_before, block_before<uint64_t>(sum.rest, s.scan_u, rests)};
            if (level == 0) need = G.R.p * Exact{units, rests}.value();
        }
        const double reached = weight ? (sum_before + sum).value() : (double)(base_count + count_before + count);
        const double before = weight ? sum_before.value() : (double)(base_count + count_before);
        if (tid == 0) s.found = 256;
        __syncthreads();
        if (count && (before < need || (count_before == 0 && base_count == 0)) && reached >= need) atomicMin(&s.found, tid);
        __syncthreads();
        const int digit = s.found;
        if (digit == 256) break;                             // all of it
        if (tid == digit) {
            s.pick_count = base_count + count_before;
            s.pick_weight = sum_before;
            s.pick_here = count;
        }
        __syncthreads();
        if (level == 0) to.part = digit; else to.from |= (uint64_t)(255 - digit) << shift;
        base_count = s.pick_count;
        base_weight = s.pick_weight;
        const uint64_t here = s.pick_here;
        __syncthreads();
        if (here == 1 || (!weight && (double)(base_count + here) == need)) break;     // all that are left belong to it
    }
    return to.within(cut);               // (where it ends early, what `cut` left out is still behind it)
}

template <bool BF16>
__device__ __noinline__ void general_row(SampleShared &s, cg::cluster_group &cluster, const SampleParams &P, const RowPlan &R, int64_t row,
                            const SampleRow &logits) {
    using S = Step<BF16>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const GeneralRow G = {s.row_max, (float)R.c, R};
    SampleCut cut = {256, 0};
    int turn = 0;
    if (R.k) {
        RowPlan all = R;                     // the first k of all, then min_p, then top_p
        all.low = -INFINITY;
        const GeneralRow A = {G.m, G.c32, all};
        cut = general_cut<BF16>(s, cluster, P, A, logits, cut, false, turn);
    }
    if (R.p < 1.0) cut = general_cut<BF16>(s, cluster, P, G, logits, cut, true, turn);
    auto w = [&](float l, int32_t i) { return G.inside(l, i, cut) ? weight_of(exponent_of(l, G.m, R.c), s.table) : 0.0; };
    double *sums = reinterpret_cast<double *>(s.list);
    for (int it = 0; it < P.steps; ++it) {
        const int32_t seg = (it * C + rank) * SP_WARPS + warp;
        double sum = 0.0;
        if (seg < P.segs) {
            S x;
            x.load(logits, seg);
#pragma unroll 4
            for (int e = 0; e < S::N; ++e) sum += w(x.value(e), S::index(logits, seg, e));
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) sums[it * SP_WARPS + warp] = sum;
    }
    cluster_sync(cluster, C);
    if (rank == 0) {
        double *all = reinterpret_cast<double *>(s.merge);
        for (int g = threadIdx.x; g < P.segs; g += SP_THREADS) {
            const int r = g / SP_WARPS % C;
            all[g] = cluster.map_shared_rank(sums, r)[g / (SP_WARPS * C) * SP_WARPS + g % SP_WARPS];
        }
        __syncthreads();
        pick_from_sums<BF16>(s, P, R, row, logits, all, w);
    }
    cluster_sync(cluster, C);
}

static_assert(SP_BLOCKS * (sizeof(SampleShared) + 1024) <= 233472, "the blocks on an SM share 228 KB");

// ---- the kernel -------------------------------------------------------------------------------
__device__ __forceinline__ RowPlan plan_row(const SampleParams &P, int64_t row) {
    RowPlan R;
    const float tau = __ldg(P.temperature + row);
    R.greedy = !(tau > 0.0f);
    R.c = 1.4426950408889634 / (R.greedy ? 1.0 : (double)tau);
    const int32_t k = R.greedy ? 1 : P.top_k ? __ldg(P.top_k + row) : 0;
    R.k = k > 0 && k < P.V ? k : R.greedy ? 1 : 0;
    const float p = R.greedy || !P.top_p ? 1.0f : __ldg(P.top_p + row), mp = R.greedy || !P.min_p ? 0.0f : __ldg(P.min_p + row);
    R.by_p = p < 1.0f;
    R.p = R.by_p ? (double)fmaxf(p, 0.0f) * (1.0 - SP_SAME) : 1.0;
    R.by_min = mp > 0.0f;
    R.low = R.by_min ? log2((double)fminf(mp, 1.0f)) : -INFINITY;
    R.u = fminf(fmaxf(__ldg(P.uniform + row), 0.0f), 1.0f);
    // (far temperatures, at which masked tokens do not vanish by themselves, take the general path)
    const bool far = !(R.c > 1e-30);
    const bool by_rank = R.k && R.k <= KEEP_K;
    R.list = !far && (by_rank || R.by_min || (R.by_p && !R.k));
    R.keep = by_rank ? R.k : R.list && !R.by_min ? KEEP_P : 0;
    // (with a little room for the roundings of this bound)
    R.drop = (float)(-R.low / R.c) * 1.00001f;
    R.sums = !far && !R.k && !R.by_min;
    R.segments = R.sums && !R.by_p;
    return R;
}

__device__ __forceinline__ void fill_table(SampleShared &s) {
    if (threadIdx.x >= 64) return;
    const double e = exp2(threadIdx.x / 64.0);
    for (int i = 0; i < 16; ++i) s.table[threadIdx.x * 16 + i] = e;
}

template <bool BF16>
__device__ __forceinline__ SampleRow row_at(const SampleParams &P, int64_t row) {
    const char *from = reinterpret_cast<const char *>(P.logits) + row * P.ld * (BF16 ? 2 : 4);
    const int skip = (int)((uintptr_t)from & 15);
    SampleRow r;
    r.base = from - skip;
    r.off = skip / (BF16 ? 2 : 4);
    r.end = r.off + P.V;
    return r;
}

template <bool BF16>
__global__ void __launch_bounds__(SP_THREADS, SP_BLOCKS) sample_kernel(const __grid_constant__ SampleParams P) {
    using S = Step<BF16>;
    extern __shared__ __align__(16) unsigned char sample_smem[];
    SampleShared &s = *reinterpret_cast<SampleShared *>(sample_smem);
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    fill_table(s);
    // The clusters take the rows in turn; the next row's first steps are asked for before the end of this one's work.
    const int64_t rows_apart = gridDim.x / C;
    SampleRow next = row_at<BF16>(P, blockIdx.x / C);
    ask_first_steps<BF16>(s, P, next, C, rank);
    for (int64_t row = blockIdx.x / C; row < P.R; row += rows_apart) {
    const SampleRow logits = next;
    if (tid == 64) s.plan = plan_row(P, row);
    if (tid == 0) {
        s.n = s.failed_here = s.merged = 0;
        s.threshold = key_of(-FLT_MAX);
        s.best = s.begin = 0;
    }
    if (tid < 4 * SP_WARPS) (&s.warp_threshold[0][0])[tid] = 0;
    __syncthreads();
    const RowPlan &R = s.plan;
    const bool sums = R.sums, by_min = R.by_min;
    bool list = R.list;
    float top = -INFINITY, top1 = -INFINITY, t = -FLT_MAX;
    double sum = 0.0;
    SumBase B;
    double *const segs = reinterpret_cast<double *>(s.list);
    // What sums are taken against: the largest of the first steps, as a power of two.
    auto set_base = [&](float step_top) {
        const uint32_t k = __reduce_max_sync(0xffffffffu, step_top > -INFINITY ? key_of(step_top) : 0u);
        if (lane == 0) atomicMax(&s.begin, k);
        __syncthreads();
        B = SumBase(s.begin ? value_of(s.begin) : 0.0f, R.c);
    };
    if (R.segments)
        read_steps<BF16>(s, P, logits, C, rank, [&](const S &x, int32_t, int it) {
            float vec[4];
            x.tops(vec);
            const float step_top = max_or_nan(max_or_nan(vec[0], vec[1]), max_or_nan(vec[2], vec[3]));
            top = max_or_nan(top, step_top);
            if (it == 0) set_base(step_top);
            double w = 0.0;
#pragma unroll
            for (int e = 0; e < S::N; ++e) w += B.weight(x.value(e), s.table);
#pragma unroll
            for (int d = 16; d; d >>= 1) w += __shfl_xor_sync(0xffffffffu, w, d);
            if (lane == 0) segs[it * SP_WARPS + warp] = w;
        });
    else
        read_steps<BF16>(s, P, logits, C, rank, [&](const S &x, int32_t seg, int it) {
            float vec[4];
            x.tops(vec);
            const float half = max_or_nan(vec[2], vec[3]);
            float step_top = max_or_nan(vec[0], vec[1]);
            top = max_or_nan(top, step_top);
            top1 = max_or_nan(top1, half);
            step_top = max_or_nan(step_top, half);
            if (sums) {
                if (it == 0) set_base(step_top);
#pragma unroll
                for (int e = 0; e < S::N; ++e) sum += B.weight(x.value(e), s.table);
            }
            if (!list) return;
            if (by_min) {
                const uint32_t k = __reduce_max_sync(0xffffffffu, step_top > -INFINITY ? key_of(step_top) : 0u);
                if (lane == 0 && k > s.best && atomicMax(&s.best, k) < k) {
                    const float m = value_of(k), least = (m - R.drop) - fabsf(m) * 1e-5f;
                    if (least > -FLT_MAX) atomicMax(&s.threshold, key_of(least));
                }
                __syncwarp();
            }
            const int n = it + 1;
            if ((n & (n - 1)) == 0) {           // behind 1, 2, 4, 8, .. steps
                if (R.keep) warp_threshold(s, R, top, top1);
                if (__syncthreads_or(s.n > SP_LIST / 2)) {
                    shorten(s, R);
                    list = !s.failed_here;
                }
                t = value_of(block_threshold(s));
            }
            if (by_min) t = fmaxf(t, value_of(*(volatile uint32_t *)&s.threshold));
            if (list && step_top >= t) put_step<BF16>(s, logits, x, vec, seg, t);
        });
    if (row + rows_apart < P.R) {
        next = row_at<BF16>(P, row + rows_apart);
        ask_first_steps<BF16>(s, P, next, C, rank);
    }
    // to the first block: the largest value, the sum, the candidates
    const bool nan = top != top || top1 != top1;
    const uint32_t block_top = __reduce_max_sync(0xffffffffu, nan ? 0u : key_of(fmaxf(top, top1)));
    if (lane == 0) atomicMax(&s.best, block_top);
    const bool any_nan = __syncthreads_or(nan);
    double block_sum = 0.0;
    if (R.sums && !R.segments) block_before<double>(sum, s.scan_d, block_sum);
    int n = 0;
    if (list) {
        if (R.keep) warp_threshold(s, R, top, top1);
        __syncthreads();
        const bool all_there = s.n <= SP_LIST;
        n = all_there ? leave_from(s, s.list, s.n, block_threshold(s)) : 0;
        if (!all_there) list = false;
        // the cluster's candidates have to fit
        if (R.keep && C > 1 && n * C > SP_LIST) {
            uint32_t cut;
            n = cut_list(s, s.list, n, R.keep, max(R.keep, SP_LIST / C), cut);
            if (tid == 0) s.threshold = max(s.threshold, cut);
        }
    }
    const uint32_t threshold = block_threshold(s);
    cluster_sync(cluster, C);                  // (the first block's counts of this row are at zero)
    SampleShared &first = *cluster.map_shared_rank(&s, 0);
    if (tid == 0) {
        s.found = n ? atomicAdd(&first.merged, n) : 0;
        first.top[rank] = s.best;
        first.bad[rank] = any_nan;
        first.cut[rank] = threshold;
        first.failed[rank] = list != R.list || s.found + n > SP_LIST;
        first.sum[rank] = block_sum;
        first.above[rank] = B.above(value_of(s.best));
    }
    __syncthreads();
    for (int i = tid; i < n && s.found + i < SP_LIST; i += SP_THREADS) first.merge[s.found + i] = s.list[i];
    cluster_sync(cluster, C);
    if (rank == 0) {
        uint32_t best = 0;
        bool bad = false, failed = !R.list && !R.sums;
        for (int i = 0; i < C; ++i) {
            best = max(best, s.top[i]);
            bad = bad || s.bad[i];
            failed = failed || s.failed[i];
        }
        const float m = value_of(best);
        bad = bad || !(m > -INFINITY);
        bool general = false;
        double total = NAN;
        if (bad) {
            if (tid == 0) answer(P, row, -1, nan_value());
        } else {
            if (R.sums) {
                bool in_range = true;
                for (int i = 0; i < C; ++i) {
                    const float l = value_of(s.top[i]);
                    if (l > -INFINITY) in_range = in_range && fabs(s.above[i]) < 900.0;
                    if (tid == i) s.scale[i] = l > -INFINITY ? exp2(exponent_of(l, m, R.c) - s.above[i]) : 0.0;
                }
                __syncthreads();
                failed = failed || !in_range;
                if (in_range) {
                    total = 0.0;
                    for (int i = 0; i < C; ++i) total += s.scale[i] > 0.0 ? s.sum[i] * s.scale[i] : 0.0;
                }
            }
            if (!failed && R.segments) {
                double *const sums = reinterpret_cast<double *>(s.merge);
                for (int g = tid; g < P.segs; g += SP_THREADS) {
                    const int r = g / SP_WARPS % C;
                    const double v = cluster.map_shared_rank(segs, r)[g / (SP_WARPS * C) * SP_WARPS + g % SP_WARPS];
                    sums[g] = s.scale[r] > 0.0 ? v * s.scale[r] : 0.0;
                }
                __syncthreads();
                pick_from_sums<BF16>(s, P, R, row, logits, sums,
                                     [&](float l, int32_t) { return weight_of(exponent_of(l, m, R.c), s.table); });
            } else if (!failed) {
                general = !pick_from_list(s, P, R, row, m, total * SP_ONE, s.merged);
            }
            general = general || failed;
        }
        if (tid < C) {
            SampleShared &to = *cluster.map_shared_rank(&s, tid);
            to.general = general;
            to.row_max = m;
            to.total = total;
        }
    }
    cluster_sync(cluster, C);
    if (s.general && P.queue) {
        if (rank == 0 && tid == 0) {
            const uint32_t at = (uint32_t)atomicAdd(&P.queue->count, 1);
            if (at < (uint32_t)P.R) P.queue->rows[at] = {(int32_t)row, s.row_max, s.total};
        }
    } else if (s.general) {
        // the next row's steps make room, and are asked for again
        asm volatile("cp.async.wait_all;" ::: "memory");
        cluster_sync(cluster, C);
        if (!band_row<BF16>(s, cluster, P, R, row, logits)) general_row<BF16>(s, cluster, P, R, row, logits);
        cluster_sync(cluster, C);
        if (row + rows_apart < P.R) ask_first_steps<BF16>(s, P, next, C, rank);
    }
    }
}

// The rows that the first launch left over, SP_REST blocks each: few as a rule, so that their time is one row's.
template <bool BF16>
__global__ void __launch_bounds__(SP_THREADS, SP_BLOCKS) sample_rest_kernel(const __grid_constant__ SampleParams P) {
    extern __shared__ __align__(16) unsigned char sample_smem[];
    SampleShared &s = *reinterpret_cast<SampleShared *>(sample_smem);
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), tid = threadIdx.x;
    cg::cluster_group::barrier_arrive();
    fill_table(s);
    griddep_wait();
    const uint32_t rows = min((uint32_t) * (volatile int32_t *)&P.queue->count, (uint32_t)P.R);
    cg::cluster_group::barrier_wait();                 // every block of the cluster runs: its shared memory may be written
    // the next row is whichever cluster's comes first: not all of them need to be there at a time
    for (;;) {
        if (rank == 0 && tid == 0) {
            const int i = atomicAdd(&P.queue->next, 1);
            for (int c = 0; c < C; ++c) cluster.map_shared_rank(&s, c)->found = i;
        }
        cluster_sync(cluster, C);
        const uint32_t i = (uint32_t)s.found;
        if (i >= rows) break;
        const SampleQueue::Row &r = P.queue->rows[i];
        const int32_t row = r.row;
        cluster_sync(cluster, C);
        if (row < 0 || row >= P.R) continue;           // (the caller's memory)
        if (tid == 64) s.plan = plan_row(P, row);
        if (tid == 0) {
            s.row_max = r.max;
            s.total = r.total;
        }
        cluster_sync(cluster, C);
        const SampleRow logits = row_at<BF16>(P, row);
        if (!band_row<BF16>(s, cluster, P, s.plan, row, logits)) general_row<BF16>(s, cluster, P, s.plan, row, logits);
        cluster_sync(cluster, C);
    }
    if (rank == 0 && tid == 0 && atomicAdd(&P.queue->done, 1) == (int)gridDim.x / C - 1) {     // every cluster has read it
        P.queue->count = P.queue->next = P.queue->done = 0;
    }
}

// Rows without filters, more of them than blocks of sample_kernel are there at a time: a block a row with no more shared
// memory than the sums of its steps and two steps a warp, so that four are on an SM.  They end apart, and one's end (a
// search, a step read again) is hidden behind the others' sums.  us, this kernel against sample_kernel: 512 rows of
// 150001 bf16, greedy 43, 53, temperature alone 93, 91 (the sums' instructions); 1000 of 32000 fp32 32, 54 and 56, 60;
// 2000 of 1000 fp32 18, 54 and 35, 53.
template <bool BF16>
__global__ void __launch_bounds__(SP_THREADS, SP_SUM_BLOCKS) sample_sum_kernel(const __grid_constant__ SampleParams P) {
    using S = Step<BF16>;
    extern __shared__ __align__(16) unsigned char sample_smem[];
    SampleShared &s = *reinterpret_cast<SampleShared *>(sample_smem);      // (up to its list)
    double *const sums = reinterpret_cast<double *>(s.list);
    uint4 (*const ring)[4][32] = reinterpret_cast<uint4 (*)[4][32]>(sample_smem + sum_ring(P.segs));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    auto ask = [&](const SampleRow &row, int it) {
        if (it < P.steps) S::ask(row, it * SP_WARPS + warp, ring[warp * 2 + (it & 1)]);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    fill_table(s);
    SampleRow next = row_at<BF16>(P, blockIdx.x);
    ask(next, 0);
    for (int64_t row = blockIdx.x; row < P.R; row += gridDim.x) {
        const SampleRow logits = next;
        __syncthreads();
        if (tid == 64) s.plan = plan_row(P, row);
        if (tid == 0) {
            s.best = s.begin = 0;
            s.pick_here = 0;
        }
        __syncthreads();
        const RowPlan &R = s.plan;
        const double c = R.c;
        const bool add = R.sums, greedy = R.k == 1;
        float top = -INFINITY;
        SumBase B;
        uint64_t best = 0;
        for (int it = 0; it < P.steps; ++it) {
            const int32_t seg = it * SP_WARPS + warp;
            ask(logits, it + 1);                     // (where the step before this one was)
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            S x;
            x.take(logits, seg, ring[warp * 2 + (it & 1)]);
            float vec[4];
            x.tops(vec);
            const float step_top = max_or_nan(max_or_nan(vec[0], vec[1]), max_or_nan(vec[2], vec[3]));
            if (greedy && step_top > top) {          // (a lane's values come in the order of their indices)
#pragma unroll
                for (int e = S::N - 1; e >= 0; --e)
                    if (x.value(e) == step_top) best = entry_of(step_top, S::index(logits, seg, e));
            }
            top = max_or_nan(top, step_top);
            if (!add) continue;
            if (it == 0) {
                const uint32_t k = __reduce_max_sync(0xffffffffu, step_top > -INFINITY ? key_of(step_top) : 0u);
                if (lane == 0) atomicMax(&s.begin, k);
                __syncthreads();
                B = SumBase(s.begin ? value_of(s.begin) : 0.0f, c);
            }
            double w = 0.0;
#pragma unroll
            for (int e = 0; e < S::N; ++e) w += B.weight(x.value(e), s.table);
#pragma unroll
            for (int d = 16; d; d >>= 1) w += __shfl_xor_sync(0xffffffffu, w, d);
            if (lane == 0 && seg < P.segs) sums[seg] = w;
        }
        if (row + gridDim.x < P.R) {
            next = row_at<BF16>(P, row + gridDim.x);
            ask(next, 0);
        }
        const bool nan = top != top;
        const uint32_t block_top = __reduce_max_sync(0xffffffffu, nan ? 0u : key_of(top));
        if (lane == 0) atomicMax(&s.best, block_top);
        if (best) atomicMax(reinterpret_cast<unsigned long long *>(&s.pick_here), (unsigned long long)best);
        const bool bad = __syncthreads_or(nan) || !(value_of(s.best) > -INFINITY);
        const float m = value_of(s.best);
        if (bad || greedy) {
            if (tid == 0) answer(P, row, bad ? -1 : index_of(s.pick_here), bad ? nan_value() : 0.0);
        } else if (!add || !(fabs(B.above(m)) < 900.0)) {
            if (tid == 0) {
                const uint32_t at = (uint32_t)atomicAdd(&P.queue->count, 1);
                if (at < (uint32_t)P.R) P.queue->rows[at] = {(int32_t)row, m, nan_value()};
            }
        } else {
            const double scale = exp2(-B.above(m));
            for (int g = tid; g < P.segs; g += SP_THREADS) sums[g] *= scale;
            __syncthreads();
            pick_from_sums<BF16>(s, P, R, row, logits, sums,
                                 [&](float l, int32_t) { return weight_of(exponent_of(l, m, c), s.table); });
        }
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
template <bool BF16>
static lora_status_t launch_sample(SampleParams P, int32_t R, int32_t device, cudaStream_t stream) {
    static std::atomic<bool> allowed[DEVICE_TABLE];
    if (device >= DEVICE_TABLE || !allowed[device].load(std::memory_order_relaxed)) {
        LORA_CUDA_TRY(allow_all_smem(sample_kernel<BF16>, device));
        LORA_CUDA_TRY(allow_all_smem(sample_rest_kernel<BF16>, device));
        LORA_CUDA_TRY(allow_all_smem(sample_sum_kernel<BF16>, device));
        if (device < DEVICE_TABLE) allowed[device].store(true, std::memory_order_relaxed);
    }
    constexpr int SEG = Step<BF16>::SEG;
    // (rows that do not begin on 16-byte boundaries have a part of a vector more)
    const bool even = ((uintptr_t)P.logits | (uint64_t)(P.ld * (BF16 ? 2 : 4))) % 16 == 0;
    P.segs = (P.V + (even ? 0 : Step<BF16>::VEC - 1) + SEG - 1) / SEG;
    // Blocks of a row: as many as the GPU holds for all rows at a time (SP_BLOCKS on an SM), while each of their
    // warps has a step.
    int C = 1;
    while (C < SP_CLUSTER && (((int64_t)R * 2 * C <= SP_BLOCKS * 148 && P.segs > C * SP_WARPS) ||
                              P.segs > SP_LIST * C)) C *= 2;
    P.steps = (P.segs + C * SP_WARPS - 1) / (C * SP_WARPS);
    const int32_t clusters = R < SP_BLOCKS * 148 / C ? R : SP_BLOCKS * 148 / C;
    // What no list holds would take one row's time with few blocks: it goes to a second launch where there is memory
    // to note it, more blocks would help, and the parameters can ask for it.
    const bool filters = P.top_k || P.top_p || P.min_p, sums = P.queue && !filters && R > SP_BLOCKS * 148;
    if (!sums && (C >= SP_REST || P.segs <= C * SP_WARPS || !filters)) P.queue = nullptr;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(clusters * C));
    cfg.blockDim = dim3(SP_THREADS);
    cfg.dynamicSmemBytes = sizeof(SampleShared);
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)C;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (sums) {
        P.steps = (P.segs + SP_WARPS - 1) / SP_WARPS;
        cfg.gridDim = dim3((unsigned)(R < SP_SUM_BLOCKS * 148 ? R : SP_SUM_BLOCKS * 148));
        cfg.dynamicSmemBytes = sum_ring(P.segs) + SP_WARPS * 2 * 2048;
        cfg.numAttrs = 0;
        LORA_CUDA_TRY(cudaLaunchKernelEx(&cfg, sample_sum_kernel<BF16>, P));
    } else {
        LORA_CUDA_TRY(cudaLaunchKernelEx(&cfg, sample_kernel<BF16>, P));
    }
    lora_status_t s = count_launch();
    if (s != LORA_OK || !P.queue) return s;
    const int32_t most = SP_BLOCKS * 148 / SP_REST;
    P.steps = (P.segs + SP_REST * SP_WARPS - 1) / (SP_REST * SP_WARPS);
    cfg.dynamicSmemBytes = sizeof(SampleShared);
    cfg.gridDim = dim3((unsigned)((R < most ? R : most) * SP_REST));
    at[0].val.clusterDim.x = SP_REST;
    cfg.numAttrs = 2;
    LORA_CUDA_TRY(cudaLaunchKernelEx(&cfg, sample_rest_kernel<BF16>, P));
    return count_launch();
}

}  // namespace lora

using namespace lora;

extern "C" lora_status_t lora_sample_workspace_bytes(int32_t R, size_t *bytes) {
    if (!bytes) return LORA_ERR_INVALID_ARG;
    if (R < 0 || R > (1 << 24)) return LORA_ERR_SHAPE;
    *bytes = offsetof(SampleQueue, rows) + (size_t)R * sizeof(SampleQueue::Row);
    return LORA_OK;
}

extern "C" lora_status_t lora_sample(const lora_sample_args_t *args, int32_t R, void *stream) {
    if (!args) return LORA_ERR_INVALID_ARG;
    const bool bf16 = args->logits_type == LORA_LOGITS_BF16;
    if (!bf16 && args->logits_type != LORA_LOGITS_FP32) return LORA_ERR_INVALID_ARG;
    if (R < 0 || R > (1 << 24) || args->vocab < 1 || args->vocab > SP_MAX_V) return LORA_ERR_SHAPE;
    if (R == 0) return LORA_OK;
    if (!args->logits || !args->temperature || !args->uniform || !args->token) return LORA_ERR_INVALID_ARG;
    if (args->ld < args->vocab) return LORA_ERR_SHAPE;
    const int64_t unit = bf16 ? 2 : 4;
    // no output lies on anything else, nor does the workspace (which is written too)
    const int64_t row_words = 4 * (int64_t)R, logits_bytes = ((R - 1) * args->ld + args->vocab) * unit;
    auto touch = [](const void *a, int64_t na, const void *b, int64_t nb) { return rows_overlap(a, na, na, b, nb, nb, 1); };
    const void *words[7] = {args->token, args->logprob, args->temperature, args->top_k, args->top_p, args->min_p, args->uniform};
    if ((uintptr_t)args->logits % unit) return LORA_ERR_INVALID_ARG;
    for (int i = 0; i < 7; ++i) {
        if (!words[i]) continue;
        if ((uintptr_t)words[i] & 3) return LORA_ERR_INVALID_ARG;
        for (int o = 0; o < 2 && o < i; ++o)
            if (words[o] && touch(words[o], row_words, words[i], row_words)) return LORA_ERR_INVALID_ARG;
        if (i < 2 && touch(words[i], row_words, args->logits, logits_bytes)) return LORA_ERR_INVALID_ARG;
    }
    size_t need = 0;
    lora_sample_workspace_bytes(R, &need);
    if ((uintptr_t)args->workspace & 15) return LORA_ERR_INVALID_ARG;
    if (args->workspace) {
        if (args->workspace_bytes < need) return LORA_ERR_BUFFER_TOO_SMALL;
        if (touch(args->workspace, (int64_t)need, args->logits, logits_bytes)) return LORA_ERR_INVALID_ARG;
        for (int i = 0; i < 7; ++i)
            if (words[i] && touch(args->workspace, (int64_t)need, words[i], row_words)) return LORA_ERR_INVALID_ARG;
    }
    SampleParams P;
    P.queue = (SampleQueue *)args->workspace;
    P.logits = args->logits;
    P.ld = args->ld;
    P.R = R;
    P.V = args->vocab;
    P.segs = P.steps = 0;
    P.temperature = args->temperature;
    P.top_p = args->top_p;
    P.min_p = args->min_p;
    P.uniform = args->uniform;
    P.top_k = args->top_k;
    P.token = args->token;
    P.logprob = args->logprob;
    DeviceGuard g(args->device);
    if (!g.ok) return cuda_fail(cudaErrorInvalidDevice);
    return bf16 ? launch_sample<true>(P, R, args->device, (cudaStream_t)stream)
                : launch_sample<false>(P, R, args->device, (cudaStream_t)stream);
}
