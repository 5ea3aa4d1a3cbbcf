// Attention of single tokens (and of a few tokens at once) over the 4-bit cache, and the joining of
// pieces that both attention kernels leave.
//
//   o = sum_t p_t v_t / sum_t p_t ,  p_t = 2^(x_t - m) ,  x_t = log2(e) scale q . k_t
//   k_t = low_t + s_t c_t :   q . k_t = s_t (q . c_t) + low_t sum(q)
//   sum_t p_t v_t = sum_A (p_t s_t) c_t + sum_B (-p_t s_t) (15 - c_t) - 7.5 (sum_A p_t s_t + sum_B -p_t s_t)
//                   + sum_t p_t (low_t + 7.5 s_t)
// so a code is never multiplied by its scale: the scale enters once per score and once per probability, and
// the low values of the values add one number per row.  A and B are the first and the last eight keys of a cell:
// the tensor cores cut their sums off towards zero at every step, so that a sum of codes that only grows is too
// small by a part of itself that grows with the number of keys (of equal weight, values around zero: outputs 0.8 %
// off at 16383 keys, 8.7 % at 131071, where their own rounding is 0.17 %); with the complements of half of the
// codes all sums stay about as small as the result is, at no cost.  (The sum of p s, over its rounded values, takes
// the middle of the codes out again, and the last one is taken over the rounded p s as well where that is exact
// enough: a rounding of p then counts v_t times.)
//
// What bounds it: every key costs head_dim + 8 bytes, and each of its codes has to be widened for the
// tensor cores whatever the number of query heads is; 1.2 instructions a code (to c - 8 in bf16 and fp16)
// were 983 a chunk and a full integer pipe, 209 us where the bytes need 97.  Hence:
//   - a nibble masked in place IS an fp16 number (a subnormal one, c 2^-24 or c 2^-20): two thirds of an
//     instruction a code, and the powers of two are put on the queries and taken from the outputs.  (The tensor
//     cores align products by the exponents as they stand, so that small ones lose bits beside a subnormal
//     factor: scores are off by 2^-17.4 of max |q| s scale, rms, 2^-14.7 at most, where prompts, whose codes are
//     normal numbers, have 2^-19.2 and 2^-16.3; outputs by up to 2^-13 of the largest p s, 2^-19 as a rule.  Both are
//     below what the 11 bits of p s cost while |q| s scale is below 4.);
//   - a warp works alone: its own ring of chunks (32 keys, two cells) filled by bulk copies, its own
//     maximum and sums; no block barrier anywhere;
//   - the matrix instructions take the keys as their 16 rows and up to eight query rows as their 8
//     columns (S^T = K q^T, o^T = V^T p^T): the codes of a cell go from shared memory through one widening
//     straight into a fragment, the probabilities through one movmatrix;
//   - all (item, head, chunk) triples of the batch form one walk that is cut into equal spans, one per
//     resident warp: no tail, whatever the lengths.  A span that ends inside an (item, head) leaves a
//     piece (maximum, sum, normalised output) in the workspace, at most two per warp.
// p_t s_t is rounded to fp16 (11 bits, where bf16 would add as much error as the output's own rounding has) and
// has to keep its bits far below the largest: a thousand keys that are each 2^-20 of one with a small value
// count.  So nearly the whole range is used: the running maximum is raised when a score passes it by 2^3, the
// common power of two of the value rows' scales seen so far when one passes it by 2^2, and the largest product of
// both is 2^15.  11 bits then reach down to 2^-22 of the largest p times the largest s; smaller products are off
// by 2^-34 of that at most.  (With margins of 2^8 for p and 2^7 for the rows' magnitudes above 1, one key 2^22
// above 8191 others took their weight from them.)
//
// Measured: 256 requests of 256..8192 keys (638 MB) 162 us with the joining, 3.9 TB/s; four requests of
// 60k..131k keys (397 MB) 101 us.  588 instructions a chunk, of which the widening is less than half, at 2.2 a
// cycle and SM (of 4): four warps a scheduler, each mostly waiting for its own last result, and the integer pipe
// (57 % busy) are what is left, not the memory.
#pragma once

#include <cuda_fp16.h>

#include <type_traits>

#include "fused_ptx.cuh"
#include "kv_common.cuh"

namespace lora {

struct AttnParams {
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    float *lse;
    int64_t ldq, ldo;
    const int32_t *tables, *block_table;
    int64_t ld_table;
    KvTables L;
    KvView kv;
    int32_t window, walkers;
    float scale2;        // scale * log2(e)
    float *part;         // [2 * walkers][rows][D] outputs of pieces, normalised
    float2 *part_ml;     // [2 * walkers][rows] their maximum (log2) and sum
};

constexpr int DK_WARPS = 4;             // warps of a block; each is on its own
// Single tokens: a score may pass the running maximum by DK_RAISE (log2), a value row the common exponent by
// DK_RAISE_E; and the power of two that probabilities come with, so that the largest p s is
// 2^15 (half of what fp16 holds: a large score's own rounding may take p past its margin).
constexpr float DK_RAISE = 3.0f;
constexpr int DK_RAISE_E = 2;
constexpr float DK_UNIT = 15.0f - DK_RAISE - DK_RAISE_E;

template <int D>
struct DecCfg {
    static constexpr int CELL = kv_cell_bytes(D);
    static constexpr int STAGE = 2 * CELL;
    static constexpr int STAGES = D == 128 ? 3 : 6;
    static constexpr int WARP_BYTES = STAGES * STAGE + STAGES * 16;   // ring, then a barrier and a flag word each
    static constexpr int SMEM = DK_WARPS * WARP_BYTES;
};

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma16816_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// fp16: 0x6400 | c is 1024 + c; the nibble above it, left in place, is 1024 + 16 c.  Less `off` (1024, or 1032
// for c - 8); a sixteenth of it, and `off` added (-64, or -72).
__device__ __forceinline__ uint32_t widen_f16_lo(uint32_t w, uint32_t off) {
    uint32_t v = (w & 0x000f000fu) | 0x64006400u, r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(off));
    return r;
}
__device__ __forceinline__ uint32_t widen_f16_hi(uint32_t w, uint32_t off) {
    uint32_t v = (w & 0x00f000f0u) | 0x64006400u, r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(v), "r"(0x2c002c00u), "r"(off));
    return r;
}
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Loads from shared memory by address.  They are ordered against waits and barriers (both clobber memory)
// and may move freely otherwise.
__device__ __forceinline__ const void *shared_at(uint32_t addr) {
    return __cvta_shared_to_generic(addr);
}
__device__ __forceinline__ uint32_t lds_u32(uint32_t addr) {
    return *reinterpret_cast<const uint32_t *>(shared_at(addr));
}
__device__ __forceinline__ void lds_v2(uint32_t addr, uint32_t (&v)[2]) {
    const uint2 u = *reinterpret_cast<const uint2 *>(shared_at(addr));
    v[0] = u.x; v[1] = u.y;
}
__device__ __forceinline__ void lds_v4(uint32_t addr, uint32_t (&v)[4]) {
    const uint4 u = *reinterpret_cast<const uint4 *>(shared_at(addr));
    v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
}
// 2^e as a float, e in -126 .. 127
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }

__device__ __forceinline__ KvItem load_item(const KvItem *p) {
    KvItem it;
    const int4 *s = reinterpret_cast<const int4 *>(p);
    int4 *d = reinterpret_cast<int4 *>(&it);
    d[0] = __ldg(s);
    d[1] = __ldg(s + 1);
    d[2] = __ldg(s + 2);
    return it;
}

// A common exponent of rows: what their scales and lows are divided by.  A row whose magnitude is 2^a
// needs e >= a - MARGIN; a new exponent is set to the row's own, or to MOST.
template <int MARGIN, int MOST>
__device__ __forceinline__ int raise_exponent(int e, uint32_t most_bits) {
    const int a = (int)(most_bits >> 23) - 126;      // magnitude < 2^a
    return a > e + MARGIN ? min(a, MOST) : e;
}
// Single tokens: the magnitude of a value row is that of 16 s, or of its low value where that is more (p s alone
// is rounded to fp16; a low value that is far off only has to stay in fp32's range).  Scales are divided by
// 2^(e - 4).
constexpr uint32_t DK_SIXTEEN = 4u << 23;
constexpr int DK_NO_EXPONENT = -122, DK_MOST_EXPONENT = 127;
// Codes as fp16 without any arithmetic: a nibble at bits 0..3 of a half is the subnormal number c 2^-24,
// at bits 4..7 it is c 2^-20, and the tensor cores take subnormal numbers as they are.
constexpr uint32_t NIB_LO = 0x000f000fu, NIB_HI = 0x00f000f0u;

template <int D, int NT>
__global__ void __launch_bounds__(32 * DK_WARPS, NT == 1 ? 4 : 3) decode_attention_kernel(const AttnParams P) {
    using C = DecCfg<D>;
    constexpr int S = C::STAGES, KW = D / 32, MT = D / 16, ROWS = 8 * NT, OVER = KV_DEC_OVER;   // words of K a lane, column tiles
    extern __shared__ __align__(128) unsigned char dk_smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    unsigned char *ring = dk_smem + warp * (S * C::STAGE);
    uint64_t *full = reinterpret_cast<uint64_t *>(dk_smem + DK_WARPS * S * C::STAGE) + warp * S;
    uint32_t *flags = reinterpret_cast<uint32_t *>(dk_smem + DK_WARPS * S * (C::STAGE + 8)) + warp * S;
    if (lane == 0) {
        for (int s = 0; s < S; ++s) mbar_init(&full[s], 1);
        fence_mbar_init();
    }
    __syncwarp();

    const int32_t w = blockIdx.x * DK_WARPS + warp;
    const KvWalk *walk = reinterpret_cast<const KvWalk *>(P.tables + P.L.walk);
    const int64_t total = walk->total, span = walk->span;
    const int64_t s0 = w * span, s1 = min(s0 + span, total);
    if (s0 >= s1) return;
    griddep_launch_dependents();      // the joining blocks may come as soon as there is room: they wait for the end
    const KvItem *items = reinterpret_cast<const KvItem *>(P.tables + P.L.dec_items);
    const int32_t first = __ldg(P.tables + P.L.dec_first + w);
    const int32_t hkv = P.kv.hkv, group = P.kv.group;

    // ---- the requesting side: a cursor over the walk that runs S - 1 chunks ahead -----------------
    int32_t f_item = first;
    KvItem fi = load_item(items + f_item);
    int32_t f_head = (int32_t)((s0 - hkv * fi.start) / (fi.n + OVER));
    int32_t f_place = (int32_t)(s0 - hkv * fi.start - (int64_t)f_head * (fi.n + OVER));     // of the pair's; chunks come behind OVER
    int64_t f_pos = s0;
    // Lane i holds cell pages_at + i of the cursor's request: the address of its first head (or none), and
    // brings that cell itself when its chunk's turn comes.
    const unsigned char *cell_at = nullptr;
    uint32_t pages_there = 0;                // bit i: lane i has one
    int32_t pages_at = 0, pages_item = -1;
    int f_s = 0;                             // the stage of the next request
    auto request = [&]() {
        if (f_place < OVER) {
            f_pos += OVER - f_place;
            f_place = OVER;
        }
        if (f_pos >= s1) return;
        int32_t idx = fi.k_lo / KV_CELL + 2 * (f_place - OVER) - pages_at;
        if (pages_item != f_item || (uint32_t)idx >= 32u) {
            pages_at += idx;
            pages_item = f_item;
            idx = 0;
            const int32_t k = (pages_at + lane) * KV_CELL, end = fi.lim0 + (fi.row0 + fi.nrows - 1) / group;
            int32_t page = -1;
            if (k < end) page = __ldg(P.block_table + fi.req * P.ld_table + (k >> P.kv.page_shift));
            if (page >= P.kv.num_pages) page = -1;
            pages_there = __ballot_sync(0xffffffffu, page >= 0);
            cell_at = kv_cell(P.kv, max(page, 0), 0, k & (P.kv.page_size - 1), C::CELL);
        }
        const uint32_t there = (pages_there >> idx) & 3u;
        if (lane == 0) {
            flags[f_s] = there;
            mbar_expect_tx(&full[f_s], (there == 3u ? 2 : there ? 1 : 0) * C::CELL);
        }
        if ((lane >> 1) == (idx >> 1) && ((pages_there >> lane) & 1u))
            bulk_g2s(ring + f_s * C::STAGE + (lane & 1) * C::CELL, cell_at + f_head * P.kv.head_bytes, C::CELL, &full[f_s]);
        if (++f_s == S) f_s = 0;
        ++f_pos;
        if (++f_place == fi.n + OVER) {
            f_place = 0;
            if (++f_head == hkv) {
                f_head = 0;
                if (f_pos < s1) fi = load_item(items + ++f_item);
            }
        }
    };
    for (int i = 0; i < S - 1; ++i) request();

    // ---- the working side ---------------------------------------------------------------------
    const int pr = (g >> 1) + (g & 1) * 4;    // the cell's row behind matrix row g (g + 8: pr + 8)
    const uint32_t ring_u = smem_u32(ring);
    int32_t it_i = first;
    KvItem it = load_item(items + it_i);
    int32_t head = (int32_t)((s0 - hkv * it.start) / (it.n + OVER));
    int32_t place = (int32_t)(s0 - hkv * it.start - (int64_t)head * (it.n + OVER));
    int64_t pos = s0;
    int stage = 0;
    uint32_t phase = 0;
    while (pos < s1) {
        // one (item, head): its chunks c0 .. c1 - 1, to the end of the item or of the span
        const int32_t c0 = max(place - OVER, 0), c1 = (int32_t)min((int64_t)it.n, place + (s1 - pos) - OVER);
        if (c1 <= c0) break;      // the span ends inside the pair's empty places
        uint32_t qf[NT][4 * KW];
        float qs[NT][2], qx[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int32_t row = n * 8 + g;
            float sum = 0.0f;
            uint32_t most = 0;
            if (row < it.nrows) {
                const int32_t r = it.row0 + row;
                const uint4 *src = reinterpret_cast<const uint4 *>(
                    P.q + (it.tok0 + r / group) * P.ldq + (int64_t)(head * group + r % group) * D + c * (D / 4));
#pragma unroll
                for (int i = 0; i < KW; ++i) {
                    const uint4 u = __ldg(src + i);
                    qf[n][4 * i] = u.x; qf[n][4 * i + 1] = u.y; qf[n][4 * i + 2] = u.z; qf[n][4 * i + 3] = u.w;
                }
#pragma unroll
                for (int i = 0; i < 4 * KW; ++i) {
                    sum += __uint_as_float(qf[n][i] << 16) + __uint_as_float(qf[n][i] & 0xffff0000u);
                    most = max(most, max((qf[n][i] << 16) & 0x7fff0000u, qf[n][i] & 0x7fff0000u));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4 * KW; ++i) qf[n][i] = 0u;
            }
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
            // the row as fp16, divided by a power of two that brings it just below 2^15 (then 8 bits are exact
            // 30 powers of two down); the columns that meet a high nibble 16 times smaller.  A negative scale
            // turns the queries.
            const int a = min(max((int)(most >> 23) - 126, -100), 110);
            const float unit = copysignf(pow2(15 - a), P.scale2);
            sum = copysignf(pow2(-9 - a), P.scale2) * sum;
#pragma unroll
            for (int i = 0; i < 4 * KW; ++i) {
                const float u = (i & 1) ? unit * 0.0625f : unit;
                qf[n][i] = pack_f16(__uint_as_float(qf[n][i] << 16) * u, __uint_as_float(qf[n][i] & 0xffff0000u) * u);
            }
            const float f = fmaxf(fabsf(P.scale2) * pow2(a + 9), 1.17549435e-38f);     // never 0: masked scores stay -inf
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                qs[n][j] = __shfl_sync(0xffffffffu, sum, (2 * c + j) * 4);
                qx[n][j] = __shfl_sync(0xffffffffu, f, (2 * c + j) * 4);
            }
        }
        const int32_t lim_min = it.lim0 + it.row0 / group;
        const int32_t lim_max = it.lim0 + (it.row0 + it.nrows - 1) / group;
        // o: outputs, lo nibbles times 2^-24, high ones times 2^-20; sp: -7.5 times the sum of the
        // rounded p s, signed as they are, which takes the middle of the codes out again.  A score x as it is held is qx x in log2; nm: DK_UNIT - (maximum in
        // log2) (0 while nothing was seen), so that a probability with its unit is 2^(qx x + nm); top: the x that raises the maximum
        float o[NT][MT][4], sp[NT][4], nm[NT][2], top[NT][2], l[NT][2], z[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][t][i] = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) sp[n][i] = 0.0f;
            top[n][0] = top[n][1] = -INFINITY;
            nm[n][0] = nm[n][1] = 0.0f;
            l[n][0] = l[n][1] = z[n][0] = z[n][1] = 0.0f;
        }
        int ve = DK_NO_EXPONENT;
        uint32_t most_ok = (uint32_t)(ve + DK_RAISE_E + 127) << 23;     // value rows up to this leave ve as it is
        for (int32_t chunk = c0; chunk < c1; ++chunk) {
            const int s = stage;
            request();       // refills the stage that was finished in the previous round
            const bool ok = mbar_wait(&full[s], phase);
            if (++stage == S) {
                stage = 0;
                phase ^= 1u;
            }
            if (!__all_sync(0xffffffffu, ok)) {
                // give up: nothing more is stored; copies on their way have to land first
                if (lane == 0) atomicAdd(&P.kv.status[STATUS_TIMEOUTS], 1);
                for (int i = 0; i < S - 1; ++i) {
                    mbar_wait(&full[stage], phase);
                    if (++stage == S) { stage = 0; phase ^= 1u; }
                }
                return;
            }
            const uint32_t base = ring_u + s * C::STAGE, valid = flags[s];
            const int32_t key0 = it.k_lo + chunk * KV_DEC_CHUNK;
            const bool whole = valid == 3u && key0 + KV_DEC_CHUNK <= lim_min && (P.window == 0 || key0 >= lim_max - P.window);

            // (two copies of what follows: one for chunks of which every row sees every key)
            auto work = [&](auto all) {
                constexpr bool WHOLE = decltype(all)::value;
                // scores of both cells: x[n][cell][i]: i 0, 1: row pr, columns 2c, 2c+1; i 2, 3: row pr + 8
                float x[NT][2][4];
                uint32_t vp_[2][2];      // (scale, low) of the value rows, 0 where there is none
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint32_t cell = base + b * C::CELL;
                    float acc[NT][4];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
                    uint32_t ka[KW], kb[KW];
                    const uint32_t at = cell + pr * (D / 2) + c * (D / 8);
                    if constexpr (D == 128) {
                        lds_v4(at, ka);
                        lds_v4(at + 8 * (D / 2), kb);
                    } else {
                        lds_v2(at, ka);
                        lds_v2(at + 8 * (D / 2), kb);
                    }
#pragma unroll
                    for (int i = 0; i < KW; ++i) {
                        const uint32_t ah = ka[i] >> 8, bh = kb[i] >> 8;
                        const uint32_t a0[4] = {ka[i] & NIB_LO, kb[i] & NIB_LO, ka[i] & NIB_HI, kb[i] & NIB_HI};
                        const uint32_t a1[4] = {ah & NIB_LO, bh & NIB_LO, ah & NIB_HI, bh & NIB_HI};
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            mma16816_f16(acc[n], a0, qf[n][4 * i], qf[n][4 * i + 1]);
                            mma16816_f16(acc[n], a1, qf[n][4 * i + 2], qf[n][4 * i + 3]);
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint32_t par = cell + kv_cell_params(D) + (pr + 8 * r) * 4;
                        const uint32_t kp = lds_u32(par), vp = lds_u32(par + KV_CELL * 4);
                        const float ks = __uint_as_float(kp << 16), kl = __uint_as_float(kp & 0xffff0000u);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            x[n][b][2 * r] = fmaf(acc[n][2 * r], ks, qs[n][0] * kl);
                            x[n][b][2 * r + 1] = fmaf(acc[n][2 * r + 1], ks, qs[n][1] * kl);
                        }
                        vp_[b][r] = vp;
                        if (!WHOLE && !(((valid >> b) & 1u) && key0 + b * KV_CELL + pr + 8 * r < lim_max)) vp_[b][r] = 0;
                    }
                }
                // magnitude of the value rows (16 scale and |low|, or a little more), for the common exponent
                uint32_t most;
                {
                    const uint32_t h = max_u16x2(max_u16x2(vp_[0][0] & 0x7fff7fffu, vp_[0][1] & 0x7fff7fffu),
                                                 max_u16x2(vp_[1][0] & 0x7fff7fffu, vp_[1][1] & 0x7fff7fffu));
                    most = max((h << 16) + DK_SIXTEEN, h & 0xffff0000u);
                }
                if (!WHOLE) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int32_t hi = it.lim0 + (it.row0 + min(n * 8 + 2 * c + j, it.nrows - 1)) / group - key0;
                            const int32_t lo = P.window > 0 ? hi - P.window : 0;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int32_t k = (i >> 1) * KV_CELL + pr + 8 * (i & 1);
                                const bool seen = ((valid >> (i >> 1)) & 1u) && k < hi && k >= lo;
                                if (!seen) x[n][i >> 1][2 * (i & 1) + j] = -INFINITY;
                            }
                        }
                }
                // maximum and exponent: raised when a score or a value row passes them by the margin
                bool up = most > most_ok;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float mx = fmaxf(fmaxf(x[n][0][j], x[n][0][2 + j]), fmaxf(x[n][1][j], x[n][1][2 + j]));
                        up |= mx > top[n][j];      // (also the first time)
                    }
                if (__any_sync(0xffffffffu, up)) {
                    // rows that are no numbers do not count (their outputs are none either)
                    if (most >= 0x7f800000u) {
                        most = 0;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t vp = vp_[i >> 1][i & 1], sb = vp << 16, lb = vp & 0x7fff0000u;
                            if (max(sb, lb) < 0x7f800000u) most = max(most, max(sb + DK_SIXTEEN, lb));
                        }
                    }
                    const int ve_new = raise_exponent<DK_RAISE_E, DK_MOST_EXPONENT>(ve, __reduce_max_sync(0xffffffffu, most));
                    const float fe = pow2(max(ve - ve_new, -126));
                    most_ok = (uint32_t)(ve_new + DK_RAISE_E + 127) << 23;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float fj[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float mx = fmaxf(fmaxf(x[n][0][j], x[n][0][2 + j]), fmaxf(x[n][1][j], x[n][1][2 + j]));
                            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                            float f = 1.0f;
                            if (mx > top[n][j]) {
                                const float now = fmaf(-mx, qx[n][j], DK_UNIT);
                                f = top[n][j] == -INFINITY ? 0.0f : exp2_approx(now - nm[n][j]);
                                nm[n][j] = now;
                                top[n][j] = mx + DK_RAISE / qx[n][j];
                            }
                            fj[j] = f * fe;
                            l[n][j] *= f;
                            z[n][j] *= fj[j];
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) sp[n][i] *= fj[i & 1];
#pragma unroll
                        for (int t = 0; t < MT; ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[n][t][i] *= fj[i & 1];
                    }
                    ve = ve_new;
                }
                // probabilities, and the second product
                const float unit = pow2(4 - ve);
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint32_t cell = base + b * C::CELL + KV_CELL * (D / 2);
                    uint32_t pb[NT][2];
                    // A row's value is s (c + low / s).  Where the low values are no more than a few steps off, they
                    // are added with the probability as it was rounded for the codes, so that its rounding counts
                    // with the value itself and not with c - 8, which may be much larger; where one is further off
                    // (or a scale is zero beside a low that is not), with the probability before the rounding.
                    float vs[2], add[2];
                    bool near = true;
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float s = __uint_as_float(vp_[b][r] << 16), low = __uint_as_float(vp_[b][r] & 0xffff0000u);
                        // (r = 1: the keys of B, whose p s is negative)
                        vs[r] = s * (r ? -unit : unit);
                        add[r] = r ? fmaf(-low, rcp_approx(s), -7.5f) : fmaf(low, rcp_approx(s), 7.5f);
                        if (!WHOLE && vp_[b][r] == 0) add[r] = 0.0f;
                        near = near && fabsf(add[r]) <= 16.0f;
                    }
                    const bool far = !__all_sync(0xffffffffu, near);
                    if (far) {
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            add[r] = fmaf(r ? -7.5f : 7.5f, vs[r], __uint_as_float(vp_[b][r] & 0xffff0000u) * unit);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float p0 = exp2_approx(fmaf(x[n][b][2 * r], qx[n][0], nm[n][0]));
                            const float p1 = exp2_approx(fmaf(x[n][b][2 * r + 1], qx[n][1], nm[n][1]));
                            float q0 = p0 * vs[r], q1 = p1 * vs[r];
                            bool h0 = false, h1 = false;
                            if (!WHOLE) {     // a value row's NaN counts only where it is seen
                                h0 = x[n][b][2 * r] == -INFINITY;
                                h1 = x[n][b][2 * r + 1] == -INFINITY;
                                q0 = h0 ? 0.0f : q0;
                                q1 = h1 ? 0.0f : q1;
                            }
                            l[n][0] += p0;
                            l[n][1] += p1;
                            const uint32_t ph = pack_f16(q0, q1);
                            float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&ph));
                            if (far) f = make_float2(p0, p1);
                            if (WHOLE) {
                                z[n][0] = fmaf(f.x, add[r], z[n][0]);
                                z[n][1] = fmaf(f.y, add[r], z[n][1]);
                            } else {
                                z[n][0] += h0 ? 0.0f : f.x * add[r];
                                z[n][1] += h1 ? 0.0f : f.y * add[r];
                            }
                            pb[n][r] = movmatrix_trans(ph);
                        }
                        const uint32_t middle[4] = {0xc780c780u, 0xc780c780u, 0xc780c780u, 0xc780c780u};   // -7.5
                        mma16816_f16(sp[n], middle, pb[n][0], pb[n][1]);
                    }
                    uint32_t v[4][D / 64];     // rows c, c + 4, c + 8, c + 12 of the cell: matrix columns 2c, 2c+1, 2c+8, 2c+9
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint32_t at = cell + (c + 4 * r) * (D / 2) + g * (D / 16);
                        if constexpr (D == 128) lds_v2(at, v[r]);
                        else v[r][0] = lds_u32(at);
                    }
#pragma unroll
                    for (int u = 0; u < D / 64; ++u)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t sel = j | ((4 + j) << 8);     // byte j of both words, one in each half
                            const uint32_t lo = __byte_perm(v[0][u], v[1][u], sel), hi = __byte_perm(v[2][u], v[3][u], sel);
                            const uint32_t a[4] = {lo & NIB_LO, lo & NIB_HI, ~hi & NIB_LO, ~hi & NIB_HI};
#pragma unroll
                            for (int n = 0; n < NT; ++n) mma16816_f16(o[n][u * 4 + j], a, pb[n][0], pb[n][1]);
                        }
                }
            };
            if (whole) work(std::true_type{});
            else work(std::false_type{});
            __syncwarp();     // every lane has read the stage: it may be requested again
        }
        // ---- this (item, head) is over, or the span is -----------------------------------------
        const bool complete = c0 == 0 && c1 == it.n;
        const int64_t slot = 2 * (int64_t)w + (c0 == 0 ? 1 : 0);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float ls = l[n][j], zs = z[n][j];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    ls += __shfl_xor_sync(0xffffffffu, ls, d);
                    zs += __shfl_xor_sync(0xffffffffu, zs, d);
                }
                const int32_t row = n * 8 + 2 * c + j;
                if (row >= it.nrows) continue;
                const float inv = ls == 0.0f ? 0.0f : 1.0f / ls;
                const float off = zs + sp[n][j], ml = -nm[n][j], back = pow2(ve - 4);
                // a lane's columns are g D/8 .. g D/8 + D/8 - 1, in the order of the codes' nibbles
                float f[D / 8];
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const int u = t >> 2, jj = t & 3;
                    f[u * 8 + (jj < 2 ? 4 * jj : 4 * (jj - 2) + 1)] = fmaf(o[n][t][j], 16777216.0f, off) * inv * back;
                    f[u * 8 + (jj < 2 ? 4 * jj + 2 : 4 * (jj - 2) + 3)] = fmaf(o[n][t][2 + j], 1048576.0f, off) * inv * back;
                }
                const int32_t r = it.row0 + row, tok = it.tok0 + r / group, hq = head * group + r % group;
                if (complete) {
                    uint32_t h[D / 16];
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const __nv_bfloat162 b2 = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                        h[i] = *reinterpret_cast<const uint32_t *>(&b2);
                    }
                    uint4 *dst = reinterpret_cast<uint4 *>(P.out + tok * P.ldo + (int64_t)hq * D + g * (D / 8));
#pragma unroll
                    for (int i = 0; i < D / 64; ++i) dst[i] = make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
                    if (P.lse && g == 0)
                        P.lse[(int64_t)tok * P.kv.hq + hq] = inv == 0.0f ? -INFINITY : (ml + log2f(ls)) * 0.69314718f;
                } else {
                    float4 *dst = reinterpret_cast<float4 *>(P.part + (slot * ROWS + row) * D + g * (D / 8));
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) dst[i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
                    if (g == 0) P.part_ml[slot * ROWS + row] = make_float2(top[n][j] == -INFINITY ? -INFINITY : ml, ls);
                }
            }
        pos += c1 + OVER - place;
        if (c1 == it.n) {
            place = 0;
            if (++head == hkv) {
                head = 0;
                if (pos < s1) it = load_item(items + ++it_i);
            }
        }
    }
}

// Joins the pieces of the (item, head) pairs that lie in more than one span, in their order, so that the
// result does not depend on timing.  What bounds it is the chain of dependent loads (walk, item, maxima,
// outputs), so every block reads its item before it waits for the kernel that leaves the pieces, and the
// loads of eight pieces are in flight together.  Two ways to share it out:
//   PAIRS = false  block x looks at the end of walker x's span and takes the pair that begins in the span and
//                  crosses it; a warp per row (rows 8 y .. 8 y + 7): many pairs of few pieces
//   PAIRS = true   block x is a pair, y its row, whose pieces the eight warps share: few pairs of many pieces
//                  (four requests of 100k keys: 75 pieces each)
template <int D, int ROWS, bool PROMPT, bool PAIRS>
__global__ void __launch_bounds__(256) join_kernel(const AttnParams P) {
    constexpr int E = D / 32, U = 8, OVER = PROMPT ? KV_PROMPT_OVER : KV_DEC_OVER;
    __shared__ float acc_s[PAIRS ? 8 : 1][D];
    __shared__ float2 ml_s[PAIRS ? 8 : 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int4 *wk = reinterpret_cast<const int4 *>(reinterpret_cast<const KvWalk *>(P.tables + P.L.walk) + (PROMPT ? 1 : 0));
    const int4 w01 = __ldg(wk), w23 = __ldg(wk + 1);
    const int64_t total = (int64_t)(uint32_t)w01.x | ((int64_t)w01.y << 32), span = (int64_t)(uint32_t)w01.z | ((int64_t)w01.w << 32);
    const KvItem *items = reinterpret_cast<const KvItem *>(P.tables + (PROMPT ? P.L.pr_items : P.L.dec_items));
    KvItem it;
    int32_t head = 0;
    int64_t begin = 0, w = blockIdx.x;
    bool mine = false;       // this block has a pair to join
    if (PAIRS) {
        const int32_t item = blockIdx.x / P.kv.hkv;
        if (item < w23.x) {
            it = load_item(items + item);
            head = blockIdx.x % P.kv.hkv;
            begin = P.kv.hkv * it.start + (int64_t)head * (it.n + OVER) + OVER;
            w = begin / span;
            mine = begin + it.n > (w + 1) * span;
        }
    } else {
        const int64_t cut = (w + 1) * span;
        if (cut < total) {
            it = load_item(items + __ldg(P.tables + (PROMPT ? P.L.pr_first : P.L.dec_first) + w + 1));
            const int64_t off = cut - P.kv.hkv * it.start;
            head = (int32_t)(off / (it.n + OVER));
            begin = P.kv.hkv * it.start + (int64_t)head * (it.n + OVER) + OVER;      // its first chunk
            mine = begin < cut && begin >= w * span && begin + it.n > cut;     // else nothing crosses this end, or another block has it
        }
    }
    // Every block waits, those without work too: what follows on the stream may in its turn wait for no more
    // than this kernel.
    griddep_wait();
    if (!mine) return;
    const int32_t row = PAIRS ? (int32_t)blockIdx.y : (int32_t)blockIdx.y * 8 + warp;
    if (row >= it.nrows) return;
    const int32_t pieces = (int32_t)((begin + it.n - 1) / span - w) + 1;
    // piece i is walker w + i's: its second slot where it begins the pair (i = 0), else its first
    auto slot = [&](int i) { return (2 * (w + i) + (i == 0 ? 1 : 0)) * ROWS + row; };
    // maximum, sum and outputs of eight pieces at a time, all requested before the first is used
    float m = -INFINITY, l = 0.0f, a[E];
#pragma unroll
    for (int e = 0; e < E; ++e) a[e] = 0.0f;
    constexpr int STEP = PAIRS ? 8 : 1;
    for (int i0 = PAIRS ? warp : 0; i0 < pieces; i0 += U * STEP) {
        float2 ml[U];
        float v[U][E];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int i = i0 + k * STEP;
            ml[k] = make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int e = 0; e < E; ++e) v[k][e] = 0.0f;
            if (i < pieces) {
                ml[k] = P.part_ml[slot(i)];
                const float *src = P.part + slot(i) * D + lane * E;
                if constexpr (E == 4) {
                    const float4 t = *reinterpret_cast<const float4 *>(src);
                    v[k][0] = t.x; v[k][1] = t.y; v[k][2] = t.z; v[k][3] = t.w;
                } else {
                    const float2 t = *reinterpret_cast<const float2 *>(src);
                    v[k][0] = t.x; v[k][1] = t.y;
                }
            }
        }
        float mn = m;
#pragma unroll
        for (int k = 0; k < U; ++k) mn = fmaxf(mn, ml[k].x);
        const float f = m == mn ? 1.0f : exp2f(m - mn);
        l *= f;
#pragma unroll
        for (int e = 0; e < E; ++e) a[e] *= f;
#pragma unroll
        for (int k = 0; k < U; ++k) {      // a piece in which the row saw nothing has sum 0
            const float w_k = ml[k].y == 0.0f ? 0.0f : ml[k].y * exp2f(ml[k].x - mn);
            l += w_k;
#pragma unroll
            for (int e = 0; e < E; ++e) a[e] = fmaf(w_k, v[k][e], a[e]);
        }
        m = mn;
    }
    if (PAIRS) {     // the eight warps' shares, in their order
#pragma unroll
        for (int e = 0; e < E; ++e) acc_s[warp][lane * E + e] = a[e];
        if (lane == 0) ml_s[warp] = make_float2(m, l);
        __syncthreads();
        if (warp) return;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = fmaxf(m, ml_s[PAIRS ? k : 0].x);
        l = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) a[e] = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float2 o = ml_s[PAIRS ? k : 0];
            const float f = o.y == 0.0f ? 0.0f : exp2f(o.x - m);
            l = fmaf(f, o.y, l);
#pragma unroll
            for (int e = 0; e < E; ++e) a[e] = fmaf(f, acc_s[PAIRS ? k : 0][lane * E + e], a[e]);
        }
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < E; ++e) a[e] *= inv;
    const int32_t r = it.row0 + row, tok = it.tok0 + r / P.kv.group, hq = head * P.kv.group + r % P.kv.group;
    // (a row whose sum is no number has inv = NaN, and so has every column)
#pragma unroll
    for (int e = 0; e < E; ++e) a[e] = isnan(l) ? l : a[e];
    __nv_bfloat162 h[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) h[e] = __floats2bfloat162_rn(a[2 * e], a[2 * e + 1]);
    __nv_bfloat16 *dst = P.out + tok * P.ldo + (int64_t)hq * D + lane * E;
    if constexpr (E == 4) *reinterpret_cast<uint2 *>(dst) = *reinterpret_cast<const uint2 *>(h);
    else *reinterpret_cast<uint32_t *>(dst) = *reinterpret_cast<const uint32_t *>(h);
    if (P.lse && lane == 0) P.lse[(int64_t)tok * P.kv.hq + hq] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718f;
}

}  // namespace lora
