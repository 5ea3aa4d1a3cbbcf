// Rows into and out of the cache: per-head norm and rotation of queries and keys, the 4-bit write of
// keys and values in the same pass, and the read back.
//
// y = x / sqrt(mean(x^2) + eps) * w, rotated; a key or value row then becomes 4-bit codes with one scale
// and one low value.  A stream: every input is read once and every output written once, with no reuse but
// the angles of a token, which all its heads share.  A head is held by head_dim / 16 lanes of a warp, each
// with two runs of 8 elements (i.. and head_dim/2 + i..: both partners of a rotation pair when the whole
// head is rotated, and two 16-byte loads), so the norm's sum and a row's minimum and maximum are three
// shuffles and nothing goes through shared memory.  Every operation is rounded by itself (the _rn
// intrinsics are never contracted), the sum is a fixed tree: the codes do not depend on the launch.
#include <cstring>

#include "kv_common.cuh"

namespace lora {

// Passes of a warp when there are many rows, and blocks of 256 threads that the registers have to leave room for
// on an SM.  (Ten and twelve passes a token, three a warp, are blocks of 128: with the bound of three blocks, 80
// registers a thread, six of them are on an SM.)
// Norm and rotation of 12936 tokens (10 passes a token) / with the cache and the read back (12 passes), us:
//   no bound on registers:  2 passes 65.9 / 104   3 passes 59.8 / 101   4 passes 64.4 / 103
//   three blocks:           2 passes 59.1 / 102   3 passes 58.3 / 92.2
//   four blocks:            2 passes 57.9 / 106   3 passes 63.9 / 100
constexpr int ROWS_NP = 3, ROWS_BLOCKS = 3;
struct RowParams {
    const __nv_bfloat16 *q, *k, *v, *qw, *kw;
    const float *cos_sin;
    const int32_t *positions, *slots;
    __nv_bfloat16 *q_out, *k_out;
    int64_t ldq, ldk, ldv, ldqo, ldko;
    int32_t T, hq, hk, num_positions, rot_dim;
    float eps;
    KvView kv;          // with slots
    int32_t *status;    // NULL without a cache
    // positions on several axes: [num_axes, ld_pos], and two bits a rotation pair that say which turns it
    int64_t ld_pos;
    int32_t num_axes;
    uint32_t axis[4];
};

// Elements 8 j .. 8 j + 7 and D/2 + 8 j .. of lane j of the head, two to a register pair: the packed
// operations round each half by itself, so they are the scalar ones at half the instructions.
struct Row { uint64_t a[4], b[4]; };

__device__ __forceinline__ void unpack8(const uint4 &u, uint64_t (&f)[4]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = pack2f(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ uint4 pack8(const uint64_t (&f)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        unpack2f(f[i], a, b);
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float lo2(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float hi2(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
// The sum of two products that are rounded by themselves.  The assembler fuses packed products and packed
// sums whatever their rounding modifiers say (one bit in 10^5 rotated values came out different), so this
// sum is taken in halves; elsewhere the products that are added are exact.
__device__ __forceinline__ uint64_t sum_of_products(uint64_t a, uint64_t b, uint64_t c, uint64_t d) {
    const uint64_t p = mul2(a, b), q = mul2(c, d);
    return pack2f(__fadd_rn(lo2(p), lo2(q)), __fadd_rn(hi2(p), hi2(q)));
}
__device__ __forceinline__ uint64_t neg2(uint64_t v) { return v ^ 0x8000000080000000ull; }
__device__ __forceinline__ uint64_t both(float x) { return pack2f(x, x); }
__device__ __forceinline__ float elem(const uint64_t (&f)[4], int i) { return (i & 1) ? hi2(f[i >> 1]) : lo2(f[i >> 1]); }

// 1 / sqrt(mean(x^2) + eps) of the head
template <int D>
__device__ __forceinline__ float inverse_norm(const Row &x, float eps) {
    float s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t q = add2(mul2(x.a[i], x.a[i]), mul2(x.b[i], x.b[i]));
        s[i] = __fadd_rn(lo2(q), hi2(q));
    }
    float sum = __fadd_rn(__fadd_rn(s[0], s[1]), __fadd_rn(s[2], s[3]));
#pragma unroll
    for (int d = 1; d < D / 16; d <<= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xffffffffu, sum, d));
    return __frcp_rn(__fsqrt_rn(__fadd_rn(__fmul_rn(sum, 1.0f / D), eps)));
}

enum { ROT_NONE = 0, ROT_HALF = 1, ROT_PART = 2, ROT_PAIRS = 3 };

// The angles a lane needs.  HALF: pairs (i, i + D/2), both in this lane.  PART: pairs (i, i + rot/2) with
// rot < D, the partner in another lane of the head.  PAIRS: (2 p, 2 p + 1), both in this lane.
template <int ROT>
struct Angles { uint64_t c[4], s[4]; };      // PAIRS: one cosine and one sine a pair, 4 of each run

template <int D, int ROT>
__device__ __forceinline__ void load_angles(Angles<ROT> &A, const float *row, int rot_dim, int j) {
    if (ROT == ROT_HALF) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 c = __ldg(reinterpret_cast<const float4 *>(row + 8 * j + 4 * i));
            const float4 s = __ldg(reinterpret_cast<const float4 *>(row + D / 2 + 8 * j + 4 * i));
            A.c[2 * i] = pack2f(c.x, c.y); A.c[2 * i + 1] = pack2f(c.z, c.w);
            A.s[2 * i] = pack2f(s.x, s.y); A.s[2 * i + 1] = pack2f(s.z, s.w);
        }
    } else if (ROT == ROT_PAIRS) {   // pair 4 j + i of the first run with pair D/4 + 4 j + i of the second
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = 4 * j + i, q = D / 4 + 4 * j + i;
            const bool in_p = 2 * p < rot_dim, in_q = 2 * q < rot_dim;
            A.c[i] = pack2f(in_p ? __ldg(row + p) : 1.0f, in_q ? __ldg(row + q) : 1.0f);
            A.s[i] = pack2f(in_p ? __ldg(row + rot_dim / 2 + p) : 0.0f, in_q ? __ldg(row + rot_dim / 2 + q) : 0.0f);
        }
    }
}

// The same from the rows of several axes: each pair's axis is two bits of `axis`.
__device__ __forceinline__ const float *axis_row(const float *cos_sin, const int32_t (&pos)[4], uint32_t axis, int rot_dim) {
    const int32_t lo = axis & 1 ? pos[1] : pos[0], hi = axis & 1 ? pos[3] : pos[2];
    return cos_sin + (int64_t)(axis & 2 ? hi : lo) * rot_dim;
}
template <int D, int ROT>
__device__ __forceinline__ void load_axes_angles(Angles<ROT> &A, const float *cos_sin, const uint32_t (&axis)[4],
                                                 const int32_t (&pos)[4], int rot_dim, int j) {
    if (ROT == ROT_HALF) {
        const uint32_t mine = axis[j / 2] >> (16 * (j & 1));
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float *row = axis_row(cos_sin, pos, mine >> (2 * i), rot_dim) + 8 * j + i;
            c[i] = __ldg(row);
            s[i] = __ldg(row + D / 2);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            A.c[i] = pack2f(c[2 * i], c[2 * i + 1]);
            A.s[i] = pack2f(s[2 * i], s[2 * i + 1]);
        }
    } else {
        const uint32_t of_p = axis[j / 4] >> (8 * (j & 3)), of_q = axis[D / 64 + j / 4] >> (8 * (j & 3));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = 4 * j + i, q = D / 4 + 4 * j + i;
            const float *rp = axis_row(cos_sin, pos, of_p >> (2 * i), rot_dim) + p;
            const float *rq = axis_row(cos_sin, pos, of_q >> (2 * i), rot_dim) + q;
            const bool in_p = 2 * p < rot_dim, in_q = 2 * q < rot_dim;
            A.c[i] = pack2f(in_p ? __ldg(rp) : 1.0f, in_q ? __ldg(rq) : 1.0f);
            A.s[i] = pack2f(in_p ? __ldg(rp + rot_dim / 2) : 0.0f, in_q ? __ldg(rq + rot_dim / 2) : 0.0f);
        }
    }
}

// Angles in global memory, or (SH) in shared memory.
template <bool SH, typename V>
__device__ __forceinline__ V angle(const V *p) { return SH ? *p : __ldg(p); }

// The rotated run (0: x.a, 1: x.b) of a head whose first rot_dim < D elements are rotated: the partner of
// element e is e +- rot/2.  rot/2 is a multiple of 8, so the eight elements of a run have their partners
// in one run of one lane.
template <int D, bool SH>
__device__ __forceinline__ void rotate_part(const Row &x, int run, const float *row, int rot_dim, int j, uint64_t (&o)[4]) {
    const int half = rot_dim / 2, e = run * (D / 2) + 8 * j;
    const bool first = e < half, in = e < rot_dim;
    const int pe = first ? e + half : in ? e - half : e;
    const int src = (threadIdx.x & 31) - j + (pe / 8) % (D / 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // a lane sends both of its runs: which one the reader wants is the reader's to choose
        const uint64_t pa = __shfl_sync(0xffffffffu, x.a[i], src), pb = __shfl_sync(0xffffffffu, x.b[i], src);
        const uint64_t other = pe >= D / 2 ? pb : pa, mine = run ? x.b[i] : x.a[i];
        o[i] = mine;
        if (in) {
            const int p = (first ? e : e - half) + 2 * i;
            const uint64_t c = pack2f(angle<SH>(row + p), angle<SH>(row + p + 1));
            const uint64_t s = pack2f(angle<SH>(row + half + p), angle<SH>(row + half + p + 1));
            o[i] = sum_of_products(mine, c, other, first ? neg2(s) : s);
        }
    }
}

// (a, b) -> (a c - b s, b c + a s).  a c - b s is taken as a c + b (-s): the same roundings.
template <int D, int ROT, bool SH>
__device__ __forceinline__ void rotate_row(Row &x, const Angles<ROT> &A, const float *row, int rot_dim, int j) {
    if (ROT == ROT_HALF) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t a = x.a[i], b = x.b[i];
            x.a[i] = sum_of_products(a, A.c[i], b, neg2(A.s[i]));
            x.b[i] = sum_of_products(b, A.c[i], a, A.s[i]);
        }
    } else if (ROT == ROT_PAIRS) {   // pairs past rot_dim have cosine 1 and sine 0, but -0 and NaN must pass unchanged
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // the two partners of a pair: swapped halves, the first times -s
#pragma unroll
            for (int run = 0; run < 2; ++run) {
                uint64_t &v = run ? x.b[i] : x.a[i];
                const float c = run ? hi2(A.c[i]) : lo2(A.c[i]), s = run ? hi2(A.s[i]) : lo2(A.s[i]);
                const uint64_t r = sum_of_products(v, both(c), pack2f(hi2(v), lo2(v)), pack2f(-s, s));
                if (run * (D / 2) + 8 * j + 2 * i < rot_dim) v = r;
            }
        }
    } else if (ROT == ROT_PART) {
        uint64_t na[4], nb[4];
        rotate_part<D, SH>(x, 0, row, rot_dim, j, na);
        rotate_part<D, SH>(x, 1, row, rot_dim, j, nb);
#pragma unroll
        for (int i = 0; i < 4; ++i) { x.a[i] = na[i]; x.b[i] = nb[i]; }
    }
}

__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Eight codes as a word: nibble n holds element {0,2,4,6,1,3,5,7}[n], so that (word >> 4 i) & 0x000f000f
// is elements 2 i and 2 i + 1.  A number in 0 .. 15 plus 1.5 2^23 is rounded to the nearest whole one (ties
// to even) and has it in its low bits; the constant's own bits are taken out of the sum at the start.
__device__ __forceinline__ uint32_t codes8(const uint64_t (&x)[4], float low, float inv, bool bad) {
    constexpr uint32_t MAGIC = 0x4b400000u;
    uint32_t w = 0u - (MAGIC + (MAGIC << 4) + (MAGIC << 8) + (MAGIC << 12) + (MAGIC << 16) + (MAGIC << 20) +
                       (MAGIC << 24) + (MAGIC << 28));
    const uint64_t inv2 = both(inv), magic = both(12582912.0f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // (the difference in halves: x may be a packed product, which a packed sum would be fused with)
        const uint64_t c = mul2(pack2f(__fsub_rn(lo2(x[i]), low), __fsub_rn(hi2(x[i]), low)), inv2);
        const uint64_t r = add2(pack2f(fminf(fmaxf(lo2(c), 0.0f), 15.0f), fminf(fmaxf(hi2(c), 0.0f), 15.0f)), magic);
        w += (uint32_t)r << (4 * i);
        w += (uint32_t)(r >> 32) << (4 * i + 16);
    }
    return bad ? 0u : w;
}
// One head's row as 4-bit codes: the words of runs a and b, and (scale, low) as two bf16.
template <int D>
__device__ __forceinline__ void quantise_row(const Row &x, uint32_t &wa, uint32_t &wb, uint32_t &param) {
    float lo = lo2(x.a[0]), hi = lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo = min_nan(lo, min_nan(elem(x.a, i), elem(x.b, i)));
        hi = max_nan(hi, max_nan(elem(x.a, i), elem(x.b, i)));
    }
#pragma unroll
    for (int d = 1; d < D / 16; d <<= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
    const float low = __bfloat162float(__float2bfloat16_rn(lo));
    float scale = __bfloat162float(__float2bfloat16_rn(__fmul_rn(__fsub_rn(hi, low), 1.0f / 15.0f)));
    if (scale < 1.17549435e-38f) scale = 0.0f;
    const bool bad = !(fabsf(scale) < INFINITY) || !(fabsf(low) < INFINITY);
    const float inv = scale == 0.0f ? 0.0f : __frcp_rn(scale);
    wa = codes8(x.a, low, inv, bad);
    wb = codes8(x.b, low, inv, bad);
    param = bad ? 0x7fc07fc0u : __float_as_uint(scale) >> 16 | (__float_as_uint(low) & 0xffff0000u);
}

// A block takes one token; a warp of it NP passes of 32 / (D/16) consecutive heads each of its row of query,
// key and (with a cache) value heads.  All its rows are requested before anything is waited for: position,
// angles and rows one after the other were 2 us a warp with 2 KB on their way (prefill of 12936 tokens:
// 94 us a launch, 187 with the cache; bytes alone 41 and 40).
// AXES: the token's positions on several axes each give some of the pairs their angles.  A lane fetches its pairs'
// angles one by one, each from the row of its axis; where a head is rotated in part, every head would fetch them again,
// and the block puts the token's row together in shared memory once.  (That for all: one barrier a token, 68.8 us
// against 61.5 for the rotation of 12936 tokens.)
template <int D, int ROT, bool CACHE, int NP, bool AXES>
__global__ void __launch_bounds__(256, ROWS_BLOCKS) rows_kernel(const RowParams P) {
    __shared__ __align__(16) float angle_row[AXES && ROT == ROT_PART ? D : 4];
    constexpr int LPH = D / 16, HPP = 32 / LPH;     // lanes of a head, heads of a pass
    const int lane = threadIdx.x & 31, j = lane % LPH, g = lane / LPH;
    const int heads = P.hq + P.hk + (CACHE ? P.hk : 0);
    const int32_t t = blockIdx.x;
    for (int h0 = (threadIdx.x >> 5) * (NP * HPP); h0 < heads; h0 += (blockDim.x >> 5) * (NP * HPP)) {
        uint4 raw[NP][2];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int h = h0 + p * HPP + g;
            if (h < heads) {
                const __nv_bfloat16 *src = h < P.hq          ? P.q + t * P.ldq + h * D
                                           : h < P.hq + P.hk ? P.k + t * P.ldk + (h - P.hq) * D
                                                             : P.v + t * P.ldv + (h - P.hq - P.hk) * D;
                raw[p][0] = *reinterpret_cast<const uint4 *>(src + 8 * j);
                raw[p][1] = *reinterpret_cast<const uint4 *>(src + D / 2 + 8 * j);
            } else {
                raw[p][0] = raw[p][1] = make_uint4(0u, 0u, 0u, 0u);
            }
        }
        int32_t slot = -1;
        if (CACHE) slot = __ldg(P.slots + t);
        const float *row = nullptr;
        Angles<ROT> A;
        bool turn = false;
        if (ROT != ROT_NONE) {
            int32_t pos[4] = {0, 0, 0, 0};
            if (AXES) {
                turn = true;
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    if (a < P.num_axes) pos[a] = __ldg(P.positions + a * P.ld_pos + t);
                    turn = turn && pos[a] >= 0 && pos[a] < P.num_positions;
                }
#pragma unroll
                for (int a = 0; a < 4; ++a) pos[a] = turn ? pos[a] : 0;
                if (ROT == ROT_PART) {
                    if (h0 == (int)(threadIdx.x >> 5) * (NP * HPP)) {      // every warp has a first pass
                        const int half = P.rot_dim / 2;
                        for (int p = threadIdx.x; p < half; p += blockDim.x) {
                            const float *from = axis_row(P.cos_sin, pos, P.axis[p / 16] >> (2 * (p % 16)), P.rot_dim) + p;
                            angle_row[p] = __ldg(from);
                            angle_row[half + p] = __ldg(from + half);
                        }
                        __syncthreads();
                    }
                    row = angle_row;
                } else {
                    load_axes_angles<D, ROT>(A, P.cos_sin, P.axis, pos, P.rot_dim, j);
                }
            } else {
                pos[0] = __ldg(P.positions + t);
                turn = pos[0] >= 0 && pos[0] < P.num_positions;
                row = P.cos_sin + (int64_t)(turn ? pos[0] : 0) * P.rot_dim;
                load_angles<D, ROT>(A, row, P.rot_dim, j);
            }
            if (!turn && P.status && h0 == 0 && lane == 0) atomicAdd(&P.status[STATUS_INVALID_TOKENS], 1);
        }
        if (CACHE) {
            const bool in = slot >= 0 && (slot >> P.kv.page_shift) < P.kv.num_pages;
            if (!in && slot != -1 && h0 == 0 && lane == 0) atomicAdd(&P.kv.status[STATUS_INVALID_TOKENS], 1);
            if (!in) slot = -1;
        }
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int h = h0 + p * HPP + g;
            const bool live = h < heads;
            // 0 query, 1 key, 2 value
            const int kind = h < P.hq ? 0 : h < P.hq + P.hk ? 1 : 2;
            const int hh = kind == 0 ? h : kind == 1 ? h - P.hq : h - P.hq - P.hk;
            if (h0 + p * HPP >= heads) break;
            Row y;
            unpack8(raw[p][0], y.a);
            unpack8(raw[p][1], y.b);
            // lanes of one warp may hold query, key and value heads: every shuffle is executed by all of them, and
            // what no lane needs is skipped by the whole warp
            const __nv_bfloat16 *w = kind == 0 ? P.qw : kind == 1 ? P.kw : nullptr;
            const bool norm = live && w;
            if (__any_sync(0xffffffffu, norm)) {
                const float r = inverse_norm<D>(y, P.eps);
                if (norm) {
                    uint64_t wa[4], wb[4];
                    unpack8(__ldg(reinterpret_cast<const uint4 *>(w + 8 * j)), wa);
                    unpack8(__ldg(reinterpret_cast<const uint4 *>(w + D / 2 + 8 * j)), wb);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        y.a[i] = mul2(mul2(y.a[i], both(r)), wa[i]);
                        y.b[i] = mul2(mul2(y.b[i], both(r)), wb[i]);
                    }
                }
            }
            if (ROT != ROT_NONE && turn && __any_sync(0xffffffffu, kind < 2)) {   // `turn` is the token's, the same in the whole warp
                const Row x = y;
                rotate_row<D, ROT, AXES>(y, A, row, P.rot_dim, j);
                if (kind == 2) y = x;
            }
            if (live && kind == 0) {
                __nv_bfloat16 *dst = P.q_out + t * P.ldqo + hh * D + 8 * j;
                *reinterpret_cast<uint4 *>(dst) = pack8(y.a);
                *reinterpret_cast<uint4 *>(dst + D / 2) = pack8(y.b);
            }
            if (live && kind == 1 && P.k_out) {
                __nv_bfloat16 *dst = P.k_out + t * P.ldko + hh * D + 8 * j;
                *reinterpret_cast<uint4 *>(dst) = pack8(y.a);
                *reinterpret_cast<uint4 *>(dst + D / 2) = pack8(y.b);
            }
            if (CACHE && h0 + p * HPP + HPP > P.hq) {   // some lane holds a key or a value (the same for all lanes)
                uint32_t wa, wb, param;
                quantise_row<D>(y, wa, wb, param);
                if (live && kind > 0 && slot >= 0) {
                    const int off = slot & (P.kv.page_size - 1), r = off % KV_CELL;
                    unsigned char *cell = kv_cell(P.kv, slot >> P.kv.page_shift, hh, off, kv_cell_bytes(D));
                    uint32_t *codes = reinterpret_cast<uint32_t *>(cell + ((kind - 1) * KV_CELL + r) * (D / 2));
                    codes[j] = wa;
                    codes[D / 16 + j] = wb;
                    if (j == 0)
                        *reinterpret_cast<uint32_t *>(cell + kv_cell_params(D) + ((kind - 1) * KV_CELL + r) * 4) = param;
                }
            }
        }
    }
}

// Rows of the cache as bf16: low + scale * code, the product exact in fp32, one rounding of the sum, one
// to bf16.  A lane takes 8 elements of one row: one word of codes, one 16-byte store.
template <int D>
__global__ void __launch_bounds__(256)
read_kernel(const KvView kv, const int32_t *slots, int32_t n, int32_t per_block, __nv_bfloat16 *k_out, int64_t ldk,
            __nv_bfloat16 *v_out, int64_t ldv) {
    constexpr uint32_t W = D / 8;                       // words of a row
    const uint32_t units = 2 * kv.hkv * W;              // of a token: key rows, then value rows
    const int32_t first = (int32_t)min((int64_t)blockIdx.x * per_block, (int64_t)n);
    const uint32_t tokens = min(per_block, n - first);
    for (uint32_t u = threadIdx.x; u < tokens * units; u += 256) {
        const uint32_t i = u / units, rest = u - i * units, w = rest % W, row = rest / W;
        const int which = row >= (uint32_t)kv.hkv, h = row - which * kv.hkv;
        __nv_bfloat16 *dst = which ? v_out : k_out;
        if (!dst) continue;
        dst += (first + i) * (which ? ldv : ldk) + h * D + w * 8;
        const int32_t slot = __ldg(slots + first + i);
        uint64_t f[4];
        if (slot >= 0 && (slot >> kv.page_shift) < kv.num_pages) {
            const int off = slot & (kv.page_size - 1), r = off % KV_CELL;
            const unsigned char *cell = kv_cell(kv, slot >> kv.page_shift, h, off, kv_cell_bytes(D));
            const uint32_t c = *reinterpret_cast<const uint32_t *>(cell + (which * KV_CELL + r) * (D / 2) + w * 4);
            const uint32_t p = *reinterpret_cast<const uint32_t *>(cell + kv_cell_params(D) + (which * KV_CELL + r) * 4);
            const uint64_t scale = both(__uint_as_float(p << 16)), low = both(__uint_as_float(p & 0xffff0000u));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                f[e] = add2(mul2(pack2f((float)((c >> (4 * e)) & 15u), (float)((c >> (4 * e + 16)) & 15u)), scale), low);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = 0;
        }
        *reinterpret_cast<uint4 *>(dst) = pack8(f);
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
static lora_status_t check_rows(const void *p, int64_t ld, int32_t heads, int32_t d) {
    if (!p || ((uintptr_t)p & 15)) return LORA_ERR_INVALID_ARG;
    if (ld < (int64_t)heads * d || ld % 8) return LORA_ERR_SHAPE;
    return LORA_OK;
}

static lora_status_t fill_rows(const lora_qk_args_t *a, int32_t T, bool cache, RowParams *P) {
    if (!a) return LORA_ERR_INVALID_ARG;
    if (T < 0 || a->num_q_heads < 0 || a->num_kv_heads < 0) return LORA_ERR_SHAPE;
    if (a->num_q_heads > 65536 || a->num_kv_heads > 65536) return LORA_ERR_SHAPE;
    const int32_t d = a->head_dim, hq = a->num_q_heads, hk = a->num_kv_heads;
    if (d != 64 && d != 128) return LORA_ERR_SHAPE;
    if (hq + hk == 0) return LORA_ERR_SHAPE;
    if (a->cos_sin) {
        if (a->rot_dim < 16 || a->rot_dim > d || a->rot_dim % 16 || a->num_positions < 1) return LORA_ERR_SHAPE;
        if (!a->positions || ((uintptr_t)a->cos_sin & 15)) return LORA_ERR_INVALID_ARG;
    }
    if (!(a->eps >= 0.0f)) return LORA_ERR_INVALID_ARG;
    if (((uintptr_t)a->q_weight | (uintptr_t)a->k_weight) & 15) return LORA_ERR_INVALID_ARG;
    lora_status_t s = LORA_OK;
    if (T == 0) return s;
    if (hq && (s = check_rows(a->q, a->ldq, hq, d)) != LORA_OK) return s;
    if (hq && (s = check_rows(a->q_out, a->ldqo, hq, d)) != LORA_OK) return s;
    if (hk && (s = check_rows(a->k, a->ldk, hk, d)) != LORA_OK) return s;
    if (hk && (a->k_out || !cache) && (s = check_rows(a->k_out, a->ldko, hk, d)) != LORA_OK) return s;
    if (hk && cache && (s = check_rows(a->v, a->ldv, hk, d)) != LORA_OK) return s;
    // an output may be its own input in place; anything else it may not touch
    const int64_t bq = (int64_t)hq * d * 2, bk = (int64_t)hk * d * 2;
    const void *out[2] = {hq ? a->q_out : nullptr, hk ? a->k_out : nullptr};
    const int64_t wo[2] = {bq, bk}, lo[2] = {a->ldqo * 2, a->ldko * 2};
    const void *in[3] = {hq ? a->q : nullptr, hk ? a->k : nullptr, hk && cache ? a->v : nullptr};
    const int64_t wi[3] = {bq, bk, bk}, li[3] = {a->ldq * 2, a->ldk * 2, a->ldv * 2};
    for (int o = 0; o < 2; ++o)
        for (int i = 0; i < 3; ++i) {
            if (!out[o] || !in[i]) continue;
            if (o == i && out[o] == in[i] && lo[o] == li[i]) continue;
            if (rows_overlap(out[o], wo[o], lo[o], in[i], wi[i], li[i], T)) return LORA_ERR_INVALID_ARG;
        }
    if (out[0] && out[1] && rows_overlap(out[0], wo[0], lo[0], out[1], wo[1], lo[1], T)) return LORA_ERR_INVALID_ARG;
    P->q = (const __nv_bfloat16 *)a->q;
    P->k = (const __nv_bfloat16 *)a->k;
    P->v = (const __nv_bfloat16 *)a->v;
    P->qw = (const __nv_bfloat16 *)a->q_weight;
    P->kw = (const __nv_bfloat16 *)a->k_weight;
    P->cos_sin = a->cos_sin;
    P->positions = a->positions;
    P->slots = nullptr;
    P->q_out = (__nv_bfloat16 *)a->q_out;
    P->k_out = (__nv_bfloat16 *)a->k_out;
    P->ldq = a->ldq; P->ldk = a->ldk; P->ldv = a->ldv; P->ldqo = a->ldqo; P->ldko = a->ldko;
    P->T = T;
    P->hq = hq;
    P->hk = hk;
    P->num_positions = a->num_positions;
    P->rot_dim = a->rot_dim;
    P->eps = a->eps;
    P->status = nullptr;
    memset(&P->kv, 0, sizeof(P->kv));
    P->ld_pos = 0;
    P->num_axes = 0;
    memset(P->axis, 0, sizeof(P->axis));
    return LORA_OK;
}

static lora_status_t fill_axes(const lora_qk_args_t *a, const lora_rope_axes_t *axes, int32_t T, RowParams *P) {
    if (!a->cos_sin || !axes->axis_of_pair) return LORA_ERR_INVALID_ARG;
    if (axes->num_axes < 1 || axes->num_axes > LORA_ROPE_AXES_MAX || axes->ld_positions < T) return LORA_ERR_SHAPE;
    P->ld_pos = axes->ld_positions;
    P->num_axes = axes->num_axes;
    for (int p = 0; p < a->rot_dim / 2; ++p) {
        if (axes->axis_of_pair[p] >= axes->num_axes) return LORA_ERR_SHAPE;
        P->axis[p / 16] |= (uint32_t)axes->axis_of_pair[p] << (2 * (p % 16));
    }
    return LORA_OK;
}

template <int D, bool CACHE, int NP>
static void launch_rows(const RowParams &P, int rot, int threads, cudaStream_t s) {
    if (P.num_axes) {
        if (rot == ROT_HALF) rows_kernel<D, ROT_HALF, CACHE, NP, true><<<P.T, threads, 0, s>>>(P);
        else if (rot == ROT_PART) rows_kernel<D, ROT_PART, CACHE, NP, true><<<P.T, threads, 0, s>>>(P);
        else rows_kernel<D, ROT_PAIRS, CACHE, NP, true><<<P.T, threads, 0, s>>>(P);
    } else if (rot == ROT_NONE) rows_kernel<D, ROT_NONE, CACHE, NP, false><<<P.T, threads, 0, s>>>(P);
    else if (rot == ROT_HALF) rows_kernel<D, ROT_HALF, CACHE, NP, false><<<P.T, threads, 0, s>>>(P);
    else if (rot == ROT_PART) rows_kernel<D, ROT_PART, CACHE, NP, false><<<P.T, threads, 0, s>>>(P);
    else rows_kernel<D, ROT_PAIRS, CACHE, NP, false><<<P.T, threads, 0, s>>>(P);
}
template <int D, bool CACHE>
static lora_status_t launch_rows_for(const RowParams &P, int rot, cudaStream_t s) {
    constexpr int HPP = 512 / D;                        // heads of one pass of a warp
    const int heads = P.hq + P.hk * (CACHE ? 2 : 1), passes = (heads + HPP - 1) / HPP;
    // Several passes a warp once there are enough of them to fill the GPU several times over (their loads are
    // in flight together and share the token's angles); fewer rows are spread over as many warps as possible.
    const bool many = (int64_t)P.T * passes >= 32768 && passes >= ROWS_NP;
    const int warps = (passes + (many ? ROWS_NP : 1) - 1) / (many ? ROWS_NP : 1);
    const int threads = 32 * (warps < 8 ? warps : 8);
    if (many) launch_rows<D, CACHE, ROWS_NP>(P, rot, threads, s);
    else launch_rows<D, CACHE, 1>(P, rot, threads, s);
    return count_launch();
}

static lora_status_t run_rows(const lora_qk_args_t *a, RowParams &P, bool cache, cudaStream_t stream) {
    const int d = a->head_dim;
    const int rot = !a->cos_sin ? ROT_NONE : a->interleaved ? ROT_PAIRS : a->rot_dim == d ? ROT_HALF : ROT_PART;
    if (d == 64) return cache ? launch_rows_for<64, true>(P, rot, stream) : launch_rows_for<64, false>(P, rot, stream);
    return cache ? launch_rows_for<128, true>(P, rot, stream) : launch_rows_for<128, false>(P, rot, stream);
}

}  // namespace lora

using namespace lora;

extern "C" {

static lora_status_t norm_rope(const lora_qk_args_t *args, const lora_rope_axes_t *axes, int32_t T, void *stream) {
    RowParams P;
    lora_status_t s = fill_rows(args, T, false, &P);
    if (s != LORA_OK || T == 0) return s;
    if (axes && (s = fill_axes(args, axes, T, &P)) != LORA_OK) return s;
    DeviceGuard g(args->device);
    if (!g.ok) return cuda_fail(cudaErrorInvalidDevice);
    return run_rows(args, P, false, (cudaStream_t)stream);
}

static lora_status_t append(lora_kv_t *kv, int32_t layer, const lora_qk_args_t *args, const lora_rope_axes_t *axes,
                            const int32_t *slots, int32_t T, void *stream) {
    if (!kv || !args) return LORA_ERR_INVALID_ARG;
    if (layer < 0 || layer >= kv->num_layers) return LORA_ERR_SLOT_RANGE;
    if (args->head_dim != kv->d || args->num_kv_heads != kv->hkv) return LORA_ERR_SHAPE;
    if (args->num_q_heads != kv->hq && args->num_q_heads != 0) return LORA_ERR_SHAPE;
    RowParams P;
    lora_status_t s = fill_rows(args, T, true, &P);
    if (s != LORA_OK || T == 0) return s;
    if (axes && (s = fill_axes(args, axes, T, &P)) != LORA_OK) return s;
    if (!slots) return LORA_ERR_INVALID_ARG;
    P.slots = slots;
    P.kv = kv->view(layer);
    P.status = kv->status_dev;
    DeviceGuard g(kv->device);
    return run_rows(args, P, true, (cudaStream_t)stream);
}

lora_status_t lora_qk_norm_rope(const lora_qk_args_t *args, int32_t T, void *stream) {
    return norm_rope(args, nullptr, T, stream);
}

lora_status_t lora_qk_norm_rope_axes(const lora_qk_args_t *args, const lora_rope_axes_t *axes, int32_t T, void *stream) {
    if (!axes) return LORA_ERR_INVALID_ARG;
    return norm_rope(args, axes, T, stream);
}

lora_status_t lora_kv_append(lora_kv_t *kv, int32_t layer, const lora_qk_args_t *args, const int32_t *slots,
                             int32_t T, void *stream) {
    return append(kv, layer, args, nullptr, slots, T, stream);
}

lora_status_t lora_kv_append_axes(lora_kv_t *kv, int32_t layer, const lora_qk_args_t *args,
                                  const lora_rope_axes_t *axes, const int32_t *slots, int32_t T, void *stream) {
    if (!axes) return LORA_ERR_INVALID_ARG;
    return append(kv, layer, args, axes, slots, T, stream);
}

lora_status_t lora_kv_read(lora_kv_t *kv, int32_t layer, const int32_t *slots, int32_t n, void *k_out, int64_t ldk,
                           void *v_out, int64_t ldv, void *stream) {
    if (!kv) return LORA_ERR_INVALID_ARG;
    if (layer < 0 || layer >= kv->num_layers) return LORA_ERR_SLOT_RANGE;
    if (n < 0) return LORA_ERR_SHAPE;
    if (n == 0) return LORA_OK;
    if (!slots) return LORA_ERR_INVALID_ARG;
    lora_status_t s;
    if (k_out && (s = check_rows(k_out, ldk, kv->hkv, kv->d)) != LORA_OK) return s;
    if (v_out && (s = check_rows(v_out, ldv, kv->hkv, kv->d)) != LORA_OK) return s;
    if (!k_out && !v_out) return LORA_OK;
    // about 2048 sixteen-byte stores a block, a token at least
    const int32_t units = 2 * kv->hkv * (kv->d / 8), per_block = units >= 2048 ? 1 : 2048 / units;
    const unsigned blocks = (unsigned)(((int64_t)n + per_block - 1) / per_block);
    DeviceGuard g(kv->device);
    if (kv->d == 64)
        read_kernel<64><<<blocks, 256, 0, (cudaStream_t)stream>>>(
            kv->view(layer), slots, n, per_block, (__nv_bfloat16 *)k_out, ldk, (__nv_bfloat16 *)v_out, ldv);
    else
        read_kernel<128><<<blocks, 256, 0, (cudaStream_t)stream>>>(
            kv->view(layer), slots, n, per_block, (__nv_bfloat16 *)k_out, ldk, (__nv_bfloat16 *)v_out, ldv);
    return count_launch();
}

}  // extern "C"
