// Attention of a batch over one layer of the 4-bit cache.
#include <cmath>

#include "kv_decode.cuh"
#include "kv_prompt.cuh"

namespace lora {

// Space for the pieces of one walk: outputs, then maximum and sum.
static size_t part_bytes(int32_t walkers, int32_t rows, int32_t d) {
    return (size_t)2 * walkers * rows * (d * sizeof(float) + sizeof(float2));
}

// The joining kernel may become resident while the one before it runs.
template <typename K>
static lora_status_t launch_join(K kernel, dim3 grid, const AttnParams &P, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    LORA_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, P));
    return count_launch();
}

template <int D, int NT>
static lora_status_t launch_decode(lora_kv *kv, AttnParams P, int64_t pairs, cudaStream_t stream) {
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
    // few pairs are cut into many pieces each: a block per pair and row
    if (pairs <= 4 * kv->sm_count)
        return launch_join(join_kernel<D, 8 * NT, false, true>, dim3((unsigned)pairs, 8 * NT), P, stream);
    return launch_join(join_kernel<D, 8 * NT, false, false>, dim3(P.walkers, NT), P, stream);
}

template <int D>
static lora_status_t launch_prompt(lora_kv *kv, AttnParams P, cudaStream_t stream) {
    using C = PromptCfg<D>;
    bool &done = kv->prompt_attr[D == 128];
    if (!done) {
        LORA_CUDA_TRY(cudaFuncSetAttribute(prompt_attention_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                           C::SMEM));
        done = true;
    }
    prompt_attention_kernel<D><<<P.walkers, PK_THREADS, C::SMEM, stream>>>(P);
    lora_status_t s = count_launch();
    if (s != LORA_OK) return s;
    return launch_join(join_kernel<D, KV_PROMPT_ROWS, true, false>, dim3(P.walkers, KV_PROMPT_ROWS / 8), P, stream);
}

}  // namespace lora

using namespace lora;

extern "C" {

lora_status_t lora_kv_workspace_bytes(const lora_kv_t *kv, size_t *bytes) {
    if (!kv || !bytes) return LORA_ERR_INVALID_ARG;
    size_t most = part_bytes(kv->dec_walkers(), kv->dec_rows(), kv->d);
    const size_t b = part_bytes(kv->pr_walkers(), KV_PROMPT_ROWS, kv->d);
    if (b > most) most = b;
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
    if (rows_overlap(q, width * 2, ldq * 2, out, width * 2, ldo * 2, T)) return LORA_ERR_INVALID_ARG;
    const float scale2 = scale * 1.4426950408889634f;
    if (!std::isfinite(scale2)) return LORA_ERR_INVALID_ARG;
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
    const int32_t rows = kv->dec_rows();
    P.L = kv_tables(R, T, kv->group, kv->dec_walkers(), kv->pr_walkers());
    P.kv = kv->view(layer);
    P.window = rec->window;
    P.scale2 = scale2;
    P.walkers = kv->dec_walkers();
    P.part = (float *)workspace;
    P.part_ml = (float2 *)(P.part + (size_t)2 * P.walkers * rows * kv->d);
    // (item, head) pairs that can be in the list (a failed request's rows are items too, however many)
    const int64_t pairs = (R + 1 + (int64_t)T * kv->group / rows) * kv->hkv;
    DeviceGuard g(kv->device);
    lora_status_t s = kv->d == 64 ? (rows == 8 ? launch_decode<64, 1>(kv, P, pairs, (cudaStream_t)stream)
                                               : launch_decode<64, 2>(kv, P, pairs, (cudaStream_t)stream))
                                  : (rows == 8 ? launch_decode<128, 1>(kv, P, pairs, (cudaStream_t)stream)
                                               : launch_decode<128, 2>(kv, P, pairs, (cudaStream_t)stream));
    if (s != LORA_OK) return s;
    // a batch whose requests all have few rows needs no more
    if ((int64_t)rec->max_q * kv->group <= KV_DEC_MAX_ROWS) return LORA_OK;
    P.walkers = kv->pr_walkers();
    P.part_ml = (float2 *)(P.part + (size_t)2 * P.walkers * KV_PROMPT_ROWS * kv->d);
    return kv->d == 64 ? launch_prompt<64>(kv, P, (cudaStream_t)stream) : launch_prompt<128>(kv, P, (cudaStream_t)stream);
}

}  // extern "C"
