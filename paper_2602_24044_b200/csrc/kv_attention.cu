// Attention of a batch over one layer of the 4-bit cache.
#include "kv_decode.cuh"

namespace lora {

// One warp per (token, query head): a lane takes a key for the scores, then head_dim / 32 columns for the
// products with the values.
template <int D>
__global__ void __launch_bounds__(128) attention_plain_kernel(const AttnParams P, int32_t T) {
    __shared__ float qs[4][D];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t unit = (int64_t)blockIdx.x * 4 + w;
    const int32_t t = (int32_t)(unit / P.kv.hq), h = (int32_t)(unit % P.kv.hq);
    if (t >= T) return;
    constexpr int E = D / 32;
    for (int e = lane; e < D; e += 32) qs[w][e] = __bfloat162float(P.q[t * P.ldq + h * D + e]);
    __syncwarp();
    const int32_t *start = P.tables + P.L.start;
    const int32_t slot = P.tables[P.L.slot + t];
    int lo = 0, hi = P.tables[KVH_R];   // the request: last r with start[r] <= t < start[r + 1]
    while (lo < hi) {
        const int m = (lo + hi) >> 1;
        if (start[m + 1] > t) hi = m; else lo = m + 1;
    }
    if (lo >= P.tables[KVH_R] || slot == -1 || (int64_t)(start[lo + 1] - start[lo]) * P.kv.group <= KV_DEC_MAX_ROWS) return;
    const int32_t limit = P.tables[P.L.position + t] + 1;
    const int32_t from = P.window > 0 ? max(0, limit - P.window) : 0;
    float m = -INFINITY, l = 0.0f, acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
    for (int32_t k0 = from & ~31; k0 < limit; k0 += 32) {
        const int32_t key = k0 + lane;
        float x = -INFINITY;
        const unsigned char *cell = nullptr;
        if (key >= from && key < limit) {
            const int32_t page = P.block_table[lo * P.ld_table + (key >> P.kv.page_shift)];
            if (page >= 0 && page < P.kv.num_pages)
                cell = kv_cell(P.kv, page, h / P.kv.group, key & (P.kv.page_size - 1), kv_cell_bytes(D));
        }
        if (cell) {
            const uint32_t p = *reinterpret_cast<const uint32_t *>(cell + kv_cell_params(D) + (key % 16) * 4);
            const float s = __uint_as_float(p << 16), low = __uint_as_float(p & 0xffff0000u);
            float dot = 0.0f;
            for (int wd = 0; wd < D / 8; ++wd) {
                const uint32_t c = *reinterpret_cast<const uint32_t *>(cell + (key % 16) * (D / 2) + wd * 4);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    dot = fmaf(qs[w][wd * 8 + e], fmaf((float)((c >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15u), s, low), dot);
            }
            x = dot * P.scale2 * 0.69314718f;
        }
        float mx = x;
#pragma unroll
        for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        const float mn = fmaxf(m, mx);
        const float c = m == -INFINITY ? 0.0f : __expf(m - mn);
        const float p = cell ? __expf(x - mn) : 0.0f;
        l = l * c + p;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= c;
        m = mn;
        for (int i = 0; i < 32; ++i) {
            const float pi = __shfl_sync(0xffffffffu, p, i);
            const unsigned char *ci = reinterpret_cast<const unsigned char *>(
                __shfl_sync(0xffffffffu, (unsigned long long)cell, i));
            if (!ci) continue;
            const int r = (k0 + i) % 16;
            const uint32_t pv = *reinterpret_cast<const uint32_t *>(ci + kv_cell_params(D) + (16 + r) * 4);
            const float s = __uint_as_float(pv << 16), low = __uint_as_float(pv & 0xffff0000u);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int col = lane * E + e;
                const uint32_t wv = *reinterpret_cast<const uint32_t *>(ci + (16 + r) * (D / 2) + (col / 8) * 4);
                const int n = ((col & 7) >> 1) + 4 * (col & 1);
                acc[e] = fmaf(pi, fmaf((float)((wv >> (4 * n)) & 15u), s, low), acc[e]);
            }
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
    const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < E; ++e) P.out[t * P.ldo + h * D + lane * E + e] = __float2bfloat16_rn(acc[e] * inv);
    if (P.lse && lane == 0) P.lse[(int64_t)t * P.kv.hq + h] = m == -INFINITY ? -INFINITY : m + logf(l);
}

// Space for the pieces of one walk: outputs, then maximum and sum.
static size_t part_bytes(int32_t walkers, int32_t rows, int32_t d) {
    return (size_t)2 * walkers * rows * (d * sizeof(float) + sizeof(float2));
}

template <int D, int NT>
static lora_status_t launch_decode(lora_kv *kv, AttnParams P, cudaStream_t stream) {
    using C = DecCfg<D>;
    bool &done = kv->decode_attr[(D == 128 ? 2 : 0) + NT - 1];
    if (!done) {
        LORA_CUDA_TRY(cudaFuncSetAttribute(decode_attention_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                           C::SMEM));
        done = true;
    }
    decode_attention_kernel<D, NT><<<P.walkers / DK_WARPS, 32 * DK_WARPS, C::SMEM, stream>>>(P);
    lora_status_t s = count_launch();
    if (s != LORA_OK) return s;
    join_kernel<D, 8 * NT, false><<<P.walkers, 256, 0, stream>>>(P);
    return count_launch();
}

}  // namespace lora

using namespace lora;

extern "C" {

lora_status_t lora_kv_workspace_bytes(const lora_kv_t *kv, size_t *bytes) {
    if (!kv || !bytes) return LORA_ERR_INVALID_ARG;
    size_t most = 0;
    for (int rows = 8; rows <= 16; rows += 8) {
        const size_t b = part_bytes(kv->dec_walkers(rows), rows, kv->d);
        if (b > most) most = b;
    }
    *bytes = (most + 255) / 256 * 256;
    return LORA_OK;
}

lora_status_t lora_kv_attention(lora_kv_t *kv, int32_t layer, const void *q, int64_t ldq, void *out, int64_t ldo,
                                float *lse, float scale, const void *tables, int32_t R, int32_t T,
                                const int32_t *block_table, int64_t ld_table, void *workspace,
                                size_t workspace_bytes, void *stream) {
    if (!kv) return LORA_ERR_INVALID_ARG;
    if (layer < 0 || layer >= kv->num_layers) return LORA_ERR_SLOT_RANGE;
    if (R < 0 || T < 0 || ld_table < 0) return LORA_ERR_SHAPE;
    if (T == 0) return LORA_OK;
    if (!q || !out || !tables || (R > 0 && !block_table)) return LORA_ERR_INVALID_ARG;
    const int64_t width = (int64_t)kv->hq * kv->d;
    if (ldq < width || ldo < width || ldq % 8 || ldo % 8) return LORA_ERR_SHAPE;
    if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)tables) & 15) return LORA_ERR_INVALID_ARG;
    const char *a = (const char *)q, *b = (const char *)out;
    if (a < b + ((T - 1) * ldo + width) * 2 && b < a + ((T - 1) * ldq + width) * 2) return LORA_ERR_INVALID_ARG;
    size_t need = 0;
    lora_kv_workspace_bytes(kv, &need);
    if (!workspace || ((uintptr_t)workspace & 15)) return LORA_ERR_INVALID_ARG;
    if (workspace_bytes < need) return LORA_ERR_BUFFER_TOO_SMALL;
    const KvTableRecord *rec = kv->find(tables, R, T);
    if (!rec) return LORA_ERR_INVALID_ARG;
    AttnParams P;
    P.q = (const __nv_bfloat16 *)q;
    P.out = (__nv_bfloat16 *)out;
    P.lse = lse;
    P.ldq = ldq;
    P.ldo = ldo;
    P.tables = (const int32_t *)tables;
    P.block_table = block_table;
    P.ld_table = ld_table;
    const int32_t rows = kv->dec_rows(rec->max_q);
    P.L = kv_tables(R, T, kv->group, kv->dec_walkers(rows), kv->pr_walkers());
    P.kv = kv->view(layer);
    P.window = rec->window;
    P.scale2 = scale * 1.4426950408889634f;
    P.walkers = kv->dec_walkers(rows);
    P.part = (float *)workspace;
    P.part_ml = (float2 *)(P.part + (size_t)2 * P.walkers * rows * kv->d);
    DeviceGuard g(kv->device);
    lora_status_t s = kv->d == 64 ? (rows == 8 ? launch_decode<64, 1>(kv, P, (cudaStream_t)stream)
                                               : launch_decode<64, 2>(kv, P, (cudaStream_t)stream))
                                  : (rows == 8 ? launch_decode<128, 1>(kv, P, (cudaStream_t)stream)
                                               : launch_decode<128, 2>(kv, P, (cudaStream_t)stream));
    if (s != LORA_OK) return s;
    // a batch whose requests all have few rows needs no more
    if ((int64_t)rec->max_q * kv->group <= KV_DEC_MAX_ROWS) return LORA_OK;
    const int64_t blocks = ((int64_t)T * kv->hq + 3) / 4;
    if (blocks > 0x7fffffff) return LORA_ERR_SHAPE;
    if (kv->d == 64) attention_plain_kernel<64><<<(unsigned)blocks, 128, 0, (cudaStream_t)stream>>>(P, T);
    else attention_plain_kernel<128><<<(unsigned)blocks, 128, 0, (cudaStream_t)stream>>>(P, T);
    return count_launch();
}

}  // extern "C"
