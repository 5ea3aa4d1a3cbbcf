// Attention of single tokens (and of a few tokens at once) over the 4-bit cache, and the joining of
// pieces that both attention kernels leave.
//
//   o = sum_t p_t v_t / sum_t p_t ,  p_t = 2^(x_t - m) ,  x_t = log2(e) scale q . k_t
//   k_t = low_t + s_t c_t :   q . k_t = s_t (q . (c_t - 8)) + (low_t + 8 s_t) sum(q)
//   sum_t p_t v_t = sum_t (p_t s_t) (c_t - 8) + sum_t p_t (low_t + 8 s_t)
// so a code is widened to c - 8 (exact in bf16 and fp16) and never multiplied by its scale: the scale
// enters once per score and once per probability, and the low values of the values add one number per row.
//
// What bounds it: every key costs head_dim + 8 bytes and each of its codes about 1.4 instructions of
// widening, whatever the number of query heads, so the memory and the instruction issue are close to
// each other (about 0.7 of the issue slots at full memory speed).  Hence:
//   - a warp works alone: its own ring of chunks (32 keys, two cells) filled by bulk copies, its own
//     maximum and sums; no block barrier anywhere;
//   - the matrix instructions take the keys as their 16 rows and up to eight query rows as their 8
//     columns (S^T = K q^T, o^T = V^T p^T): the codes of a cell go from shared memory through one widening
//     straight into a fragment, the probabilities through one movmatrix;
//   - all (item, head, chunk) triples of the batch form one walk that is cut into equal spans, one per
//     resident warp: no tail, whatever the lengths.  A span that ends inside an (item, head) leaves a
//     piece (maximum, sum, normalised output) in the workspace, at most two per warp.
// The running maximum is raised only when a score passes it by 2^8: the probabilities then stay below 256
// and the accumulators are rescaled once in a while instead of once a chunk.  p_t s_t is rounded to fp16
// (11 bits, where bf16 would add as much error as the output's own rounding has); its exponent range is
// kept by a common power of two of the value rows seen so far, raised like the maximum.
#pragma once

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
constexpr float KV_RAISE = 8.0f;        // a score may pass the running maximum by this (log2)
constexpr int KV_RAISE_E = 7;           // a value row may pass the common exponent by this

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
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma16816_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// nibbles at bits 0..3 and 16..19 -> two numbers c - 8.  bf16: 0x4300 | c is 128 + c.
__device__ __forceinline__ uint32_t widen_bf16(uint32_t w) {
    uint32_t v = (w & 0x000f000fu) | 0x43004300u, r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(0x43084308u));
    return r;
}
// fp16: 0x6400 | c is 1024 + c; the nibble above it, left in place, is 1024 + 16 c.
__device__ __forceinline__ uint32_t widen_f16_lo(uint32_t w) {
    uint32_t v = (w & 0x000f000fu) | 0x64006400u, r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(0x64086408u));
    return r;
}
__device__ __forceinline__ uint32_t widen_f16_hi(uint32_t w) {
    uint32_t v = (w & 0x00f000f0u) | 0x64006400u, r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(v), "r"(0x2c002c00u), "r"(0xd480d480u));   // v / 16 - 72
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t lds_u32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ void lds_v2(uint32_t addr, uint32_t (&v)[2]) {
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(addr));
}
__device__ __forceinline__ void lds_v4(uint32_t addr, uint32_t (&v)[4]) {
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(addr));
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

// The common exponent of the value rows: what their scales and lows are divided by.  A row whose
// magnitude is 2^a needs e >= a - KV_RAISE_E; a new exponent is set to the row's own.
__device__ __forceinline__ int raise_exponent(int e, uint32_t most_bits) {
    const int a = (int)(most_bits >> 23) - 126;      // magnitude < 2^a
    return a > e + KV_RAISE_E ? min(a, 126) : e;
}
constexpr int KV_NO_EXPONENT = -126;

template <int D, int NT>
__global__ void __launch_bounds__(32 * DK_WARPS, NT == 1 ? 4 : 3) decode_attention_kernel(const AttnParams P) {
    using C = DecCfg<D>;
    constexpr int S = C::STAGES, KW = D / 32, MT = D / 16, ROWS = 8 * NT;   // words of K a lane, column tiles
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
    int32_t f_head = (int32_t)((s0 - hkv * fi.start) / fi.n), f_chunk = (int32_t)(s0 - hkv * fi.start - (int64_t)f_head * fi.n);
    int64_t f_pos = s0;
    int32_t pages = -1, pages_at = -1;       // lane i: the page of cell pages_at + i of the cursor's request
    int32_t pages_item = -1;
    uint32_t issued = 0;
    auto request = [&]() {
        if (f_pos >= s1) return;
        const int s = issued % S;
        const int32_t key = fi.k_lo + f_chunk * KV_DEC_CHUNK, cell = key / KV_CELL;
        const int32_t end = fi.lim0 + (fi.row0 + fi.nrows - 1) / group;      // keys below this are there
        if (pages_item != f_item || cell < pages_at || cell + 2 > pages_at + 32) {
            pages_at = cell;
            pages_item = f_item;
            const int32_t k = (cell + lane) * KV_CELL;
            pages = -1;
            if (k < end) {
                pages = __ldg(P.block_table + fi.req * P.ld_table + (k >> P.kv.page_shift));
                if (pages < 0 || pages >= P.kv.num_pages) pages = -1;
            }
        }
        const int32_t p0 = __shfl_sync(0xffffffffu, pages, cell - pages_at);
        const int32_t p1 = __shfl_sync(0xffffffffu, pages, cell + 1 - pages_at);
        if (lane == 0) {
            unsigned char *dst = ring + s * C::STAGE;
            flags[s] = (p0 >= 0 ? 1u : 0u) | (p1 >= 0 ? 2u : 0u);
            mbar_expect_tx(&full[s], ((p0 >= 0) + (p1 >= 0)) * C::CELL);
            const int32_t off = key & (P.kv.page_size - 1);
            if (P.kv.page_size > KV_CELL) {      // both cells lie in one page
                if (p0 >= 0) bulk_g2s(dst, kv_cell(P.kv, p0, f_head, off, C::CELL), (1 + (p1 >= 0)) * C::CELL, &full[s]);
            } else {
                if (p0 >= 0) bulk_g2s(dst, kv_cell(P.kv, p0, f_head, 0, C::CELL), C::CELL, &full[s]);
                if (p1 >= 0) bulk_g2s(dst + C::CELL, kv_cell(P.kv, p1, f_head, 0, C::CELL), C::CELL, &full[s]);
            }
        }
        ++issued;
        ++f_pos;
        if (++f_chunk == fi.n) {
            f_chunk = 0;
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
    int32_t head = (int32_t)((s0 - hkv * it.start) / it.n), chunk = (int32_t)(s0 - hkv * it.start - (int64_t)head * it.n);
    int64_t pos = s0;
    uint32_t done = 0;
    while (pos < s1) {
        // one (item, head): its chunks from `chunk` to the end of the item or of the span
        const int32_t c0 = chunk, c1 = (int32_t)min((int64_t)it.n, chunk + (s1 - pos));
        uint32_t qf[NT][4 * KW];
        float qs[NT][2];
        int32_t lim[NT][2];
        int32_t lim_min = 0x7fffffff, lim_max = -0x7fffffff;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int32_t row = n * 8 + g;
            float sum = 0.0f;
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
                for (int i = 0; i < 4 * KW; ++i)
                    sum += __uint_as_float(qf[n][i] << 16) + __uint_as_float(qf[n][i] & 0xffff0000u);
            } else {
#pragma unroll
                for (int i = 0; i < 4 * KW; ++i) qf[n][i] = 0u;
            }
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                qs[n][j] = __shfl_sync(0xffffffffu, sum, (2 * c + j) * 4);
                const int32_t rr = min(n * 8 + 2 * c + j, it.nrows - 1);
                lim[n][j] = it.lim0 + (it.row0 + rr) / group;
            }
        }
        lim_min = it.lim0 + it.row0 / group;
        lim_max = it.lim0 + (it.row0 + it.nrows - 1) / group;
        float o[NT][MT][4], m[NT][2], l[NT][2], z[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][t][i] = 0.0f;
            m[n][0] = m[n][1] = -INFINITY;
            l[n][0] = l[n][1] = z[n][0] = z[n][1] = 0.0f;
        }
        int ve = KV_NO_EXPONENT;
        for (chunk = c0; chunk < c1; ++chunk, ++done) {
            const int s = done % S;
            request();       // refills the stage that was finished in the previous round
            const bool ok = mbar_wait(&full[s], (done / S) & 1u);
            if (!__all_sync(0xffffffffu, ok)) {      // give up: nothing more is stored
                if (lane == 0) {
                    atomicAdd(&P.kv.status[STATUS_TIMEOUTS], 1);
                    for (uint32_t i = done + 1; i < issued; ++i) mbar_wait(&full[i % S], (i / S) & 1u);
                }
                return;
            }
            const uint32_t base = ring_u + s * C::STAGE, valid = flags[s];
            const int32_t key0 = it.k_lo + chunk * KV_DEC_CHUNK;
            const bool whole = valid == 3u && key0 + KV_DEC_CHUNK <= lim_min && (P.window == 0 || key0 >= lim_max - P.window);

            // scores of both cells: x[n][cell][i]: i 0, 1: row pr, columns 2c, 2c+1; i 2, 3: row pr + 8
            float x[NT][2][4];
            float vs[2][2], vz[2][2];
            uint32_t most = 0;
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
                for (int i = 0; i < KW; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t a[4] = {widen_bf16(ka[i] >> (8 * j)), widen_bf16(kb[i] >> (8 * j)),
                                               widen_bf16(ka[i] >> (8 * j + 4)), widen_bf16(kb[i] >> (8 * j + 4))};
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            mma16816(acc[n], a, qf[n][4 * i + 2 * j], qf[n][4 * i + 2 * j + 1]);
                    }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t par = cell + kv_cell_params(D) + (pr + 8 * r) * 4;
                    const uint32_t kp = lds_u32(par), vp = lds_u32(par + KV_CELL * 4);
                    const float ks = __uint_as_float(kp << 16), kl = __uint_as_float(kp & 0xffff0000u);
                    const float kz = fmaf(8.0f, ks, kl) * P.scale2, kf = ks * P.scale2;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        x[n][b][2 * r] = fmaf(acc[n][2 * r], kf, qs[n][0] * kz);
                        x[n][b][2 * r + 1] = fmaf(acc[n][2 * r + 1], kf, qs[n][1] * kz);
                    }
                    vs[b][r] = __uint_as_float(vp << 16);
                    const float vl = __uint_as_float(vp & 0xffff0000u);
                    vz[b][r] = fmaf(8.0f, vs[b][r], vl);
                    // magnitude of the value row, for the common exponent (rows that do not count: none)
                    const uint32_t mag = max(vp << 16, vp & 0x7fff0000u);
                    const int32_t key = key0 + b * KV_CELL + pr + 8 * r;
                    const bool seen = whole || (((valid >> b) & 1u) && key < lim_max);
                    if (seen && mag < 0x7f800000u) most = max(most, mag);
                    if (!seen) vs[b][r] = vz[b][r] = 0.0f;
                }
            }
            if (!whole) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int32_t key = key0 + b * KV_CELL + pr + 8 * (i >> 1), lm = lim[n][i & 1];
                            const bool seen = ((valid >> b) & 1u) && key < lm && (P.window == 0 || key >= lm - P.window);
                            if (!seen) x[n][b][i] = -INFINITY;
                        }
            }
            // maximum and exponent: raised when a score or a value row passes them by the margin
            bool up = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float mx = fmaxf(fmaxf(x[n][0][j], x[n][0][2 + j]), fmaxf(x[n][1][j], x[n][1][2 + j]));
                    up |= mx > m[n][j] + KV_RAISE;      // (also the first time: m is -inf)
                }
            const int ve_lane = raise_exponent(ve, most);
            up |= ve_lane != ve;
            if (__any_sync(0xffffffffu, up)) {
                const int ve_new = raise_exponent(ve, __reduce_max_sync(0xffffffffu, most));
                const float fe = pow2(max(ve - ve_new, -126));
                ve = ve_new;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float mx = fmaxf(fmaxf(x[n][0][j], x[n][0][2 + j]), fmaxf(x[n][1][j], x[n][1][2 + j]));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                        const float mn = mx > m[n][j] + KV_RAISE ? mx : m[n][j];
                        const float f = mn == m[n][j] ? 1.0f : exp2_approx(m[n][j] - mn);
                        m[n][j] = mn;
                        l[n][j] *= f;
                        z[n][j] *= f * fe;
#pragma unroll
                        for (int t = 0; t < MT; ++t) {
                            o[n][t][j] *= f * fe;
                            o[n][t][2 + j] *= f * fe;
                        }
                    }
            }
            // probabilities, and the second product
            const float unit = pow2(-ve);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint32_t cell = base + b * C::CELL + KV_CELL * (D / 2);
                uint32_t pb[NT][2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float fs = vs[b][r] * unit, fz = vz[b][r] * unit;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float p0 = exp2_approx(x[n][b][2 * r] - m[n][0]), p1 = exp2_approx(x[n][b][2 * r + 1] - m[n][1]);
                        float q0 = p0 * fs, q1 = p1 * fs, z0 = p0 * fz, z1 = p1 * fz;
                        if (!whole) {    // a row that nothing counts in has no maximum; a row's NaN counts only where it is seen
                            const bool a0 = x[n][b][2 * r] == -INFINITY, a1 = x[n][b][2 * r + 1] == -INFINITY;
                            p0 = a0 ? 0.0f : p0; q0 = a0 ? 0.0f : q0; z0 = a0 ? 0.0f : z0;
                            p1 = a1 ? 0.0f : p1; q1 = a1 ? 0.0f : q1; z1 = a1 ? 0.0f : z1;
                        }
                        l[n][0] += p0;
                        l[n][1] += p1;
                        z[n][0] += z0;
                        z[n][1] += z1;
                        pb[n][r] = movmatrix_trans(pack_f16(q0, q1));
                    }
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
                        const uint32_t a[4] = {widen_f16_lo(lo), widen_f16_hi(lo), widen_f16_lo(hi), widen_f16_hi(hi)};
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma16816_f16(o[n][u * 4 + j], a, pb[n][0], pb[n][1]);
                    }
            }
            __syncwarp();     // every lane has read the stage: it may be requested again
        }
        // ---- this (item, head) is over, or the span is -----------------------------------------
        const bool complete = c0 == 0 && c1 == it.n;
        const int64_t slot = 2 * (int64_t)w + (c0 == 0 ? 1 : 0);
        const float back = pow2(ve);
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
                const float inv = m[n][j] == -INFINITY && ls == 0.0f ? 0.0f : 1.0f / ls;
                // a lane's columns are g D/8 .. g D/8 + D/8 - 1, in the order of the codes' nibbles
                float f[D / 8];
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const int u = t >> 2, jj = t & 3;
                    f[u * 8 + (jj < 2 ? 4 * jj : 4 * (jj - 2) + 1)] = (o[n][t][j] + zs) * inv * back;
                    f[u * 8 + (jj < 2 ? 4 * jj + 2 : 4 * (jj - 2) + 3)] = (o[n][t][2 + j] + zs) * inv * back;
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
                        P.lse[(int64_t)tok * P.kv.hq + hq] = inv == 0.0f ? -INFINITY : (m[n][j] + log2f(ls)) * 0.69314718f;
                } else {
                    float4 *dst = reinterpret_cast<float4 *>(P.part + (slot * ROWS + row) * D + g * (D / 8));
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) dst[i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
                    if (g == 0) P.part_ml[slot * ROWS + row] = make_float2(m[n][j], ls);
                }
            }
        pos += c1 - c0;
        if (c1 == it.n) {
            chunk = 0;
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
// loads of 16 pieces are in flight together.  Two ways to share it out:
//   PAIRS = false  block x looks at the end of walker x's span and takes the pair that begins in the span and
//                  crosses it; a warp per row (rows 8 y .. 8 y + 7): many pairs of few pieces
//   PAIRS = true   block x is a pair, y its row, whose pieces the eight warps share: few pairs of many pieces
//                  (four requests of 100k keys: 75 pieces each)
template <int D, int ROWS, bool PROMPT, bool PAIRS>
__global__ void __launch_bounds__(256) join_kernel(const AttnParams P) {
    constexpr int E = D / 32, U = 16;
    __shared__ float acc_s[PAIRS ? 8 : 1][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int4 *wk = reinterpret_cast<const int4 *>(reinterpret_cast<const KvWalk *>(P.tables + P.L.walk) + (PROMPT ? 1 : 0));
    const int4 w01 = __ldg(wk), w23 = __ldg(wk + 1);
    const int64_t total = (int64_t)(uint32_t)w01.x | ((int64_t)w01.y << 32), span = (int64_t)(uint32_t)w01.z | ((int64_t)w01.w << 32);
    const KvItem *items = reinterpret_cast<const KvItem *>(P.tables + (PROMPT ? P.L.pr_items : P.L.dec_items));
    KvItem it;
    int32_t head;
    int64_t begin, w;
    if (PAIRS) {
        const int32_t item = blockIdx.x / P.kv.hkv;
        if (item >= w23.x) return;
        it = load_item(items + item);
        head = blockIdx.x % P.kv.hkv;
        begin = P.kv.hkv * it.start + (int64_t)head * it.n;
        w = begin / span;
        if (begin + it.n <= (w + 1) * span) return;
    } else {
        w = blockIdx.x;
        const int64_t cut = (w + 1) * span;
        if (cut >= total) return;
        it = load_item(items + __ldg(P.tables + (PROMPT ? P.L.pr_first : P.L.dec_first) + w + 1));
        const int64_t off = cut - P.kv.hkv * it.start;
        head = (int32_t)(off / it.n);
        begin = P.kv.hkv * it.start + (int64_t)head * it.n;
        if (begin == cut || begin < w * span) return;      // nothing crosses this end, or another block has it
    }
    const int32_t row = PAIRS ? (int32_t)blockIdx.y : (int32_t)blockIdx.y * 8 + warp;
    if (row >= it.nrows) return;
    const int32_t pieces = (int32_t)((begin + it.n - 1) / span - w) + 1;
    // piece i is walker w + i's: its second slot where it begins the pair (i = 0), else its first
    auto slot = [&](int i) { return (2 * (w + i) + (i == 0 ? 1 : 0)) * ROWS + row; };
    griddep_wait();
    float m = -INFINITY, l = 0.0f;
    for (int i = lane; i < pieces; i += 32) m = fmaxf(m, P.part_ml[slot(i)].x);
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    for (int i = lane; i < pieces; i += 32) {      // a piece in which the row saw nothing has sum 0
        const float2 v = P.part_ml[slot(i)];
        l += v.y == 0.0f ? 0.0f : v.y * exp2f(v.x - m);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    float a[E];
#pragma unroll
    for (int e = 0; e < E; ++e) a[e] = 0.0f;
    for (int i0 = PAIRS ? warp : 0; i0 < pieces; i0 += U * (PAIRS ? 8 : 1)) {
        float f[U], v[U][E];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int i = i0 + k * (PAIRS ? 8 : 1);
            if (i < pieces) {
                const float2 ml = P.part_ml[slot(i)];
                f[k] = ml.y == 0.0f ? 0.0f : ml.y * exp2f(ml.x - m) * inv;
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
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (i0 + k * (PAIRS ? 8 : 1) < pieces)
#pragma unroll
                for (int e = 0; e < E; ++e) a[e] = fmaf(f[k], v[k][e], a[e]);
    }
    const int32_t r = it.row0 + row, tok = it.tok0 + r / P.kv.group, hq = head * P.kv.group + r % P.kv.group;
    if (PAIRS) {
#pragma unroll
        for (int e = 0; e < E; ++e) acc_s[warp][lane * E + e] = a[e];
        __syncthreads();
        if (warp) return;
#pragma unroll
        for (int e = 0; e < E; ++e) a[e] = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) a[e] += acc_s[PAIRS ? k : 0][lane * E + e];
    }
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
