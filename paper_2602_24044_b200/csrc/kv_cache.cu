// The paged 4-bit key/value cache: handle, sizes, status words.
#include <new>

#include "kv_common.cuh"

lora::KvView lora_kv::view(int32_t layer) const {
    lora::KvView v;
    v.cells = base + 256 + (int64_t)layer * layer_bytes;
    v.page_bytes = page_bytes;
    v.head_bytes = page_bytes / hkv;
    v.num_pages = num_pages;
    v.page_size = page_size;
    v.page_shift = page_shift;
    v.hq = hq;
    v.hkv = hkv;
    v.group = group;
    v.status = status_dev;
    return v;
}

namespace lora {
static lora_status_t validate(const lora_kv_desc_t *d) {
    if (!d) return LORA_ERR_INVALID_ARG;
    if (d->num_layers < 1 || d->num_pages < 1) return LORA_ERR_INVALID_ARG;
    if (d->page_size != 16 && d->page_size != 32 && d->page_size != 64 && d->page_size != 128) return LORA_ERR_SHAPE;
    if (d->head_dim != 64 && d->head_dim != 128) return LORA_ERR_SHAPE;
    if (d->num_kv_heads < 1 || d->num_q_heads < 1 || d->num_q_heads % d->num_kv_heads) return LORA_ERR_SHAPE;
    if (d->num_q_heads / d->num_kv_heads > 128 || d->num_kv_heads > 4096) return LORA_ERR_SHAPE;
    if ((int64_t)d->num_pages * d->page_size > 0x7fffffff) return LORA_ERR_SHAPE;   // slots are int32
    return LORA_OK;
}
static int64_t page_bytes_of(const lora_kv_desc_t *d) {
    return (int64_t)d->num_kv_heads * (d->page_size / KV_CELL) * kv_cell_bytes(d->head_dim);
}
// the control block (status words) comes first, 256 bytes; every layer starts on 256 bytes
static int64_t layer_bytes_of(const lora_kv_desc_t *d) { return (page_bytes_of(d) * d->num_pages + 255) / 256 * 256; }
}  // namespace lora

using namespace lora;

extern "C" {

lora_status_t lora_kv_bytes(const lora_kv_desc_t *desc, size_t *bytes) {
    if (!bytes) return LORA_ERR_INVALID_ARG;
    lora_status_t s = validate(desc);
    if (s != LORA_OK) return s;
    *bytes = 256 + (size_t)layer_bytes_of(desc) * (size_t)desc->num_layers;
    return LORA_OK;
}

lora_status_t lora_kv_layer_range(const lora_kv_desc_t *desc, int32_t layer, size_t *offset, size_t *bytes) {
    if (!offset || !bytes) return LORA_ERR_INVALID_ARG;
    lora_status_t s = validate(desc);
    if (s != LORA_OK) return s;
    if (layer < 0 || layer >= desc->num_layers) return LORA_ERR_SLOT_RANGE;
    *offset = 256 + (size_t)layer_bytes_of(desc) * (size_t)layer;
    *bytes = (size_t)page_bytes_of(desc) * (size_t)desc->num_pages;
    return LORA_OK;
}

lora_status_t lora_kv_create(const lora_kv_desc_t *desc, lora_kv_t **out) {
    if (!out) return LORA_ERR_INVALID_ARG;
    *out = nullptr;
    size_t need = 0;
    lora_status_t s = lora_kv_bytes(desc, &need);
    if (s != LORA_OK) return s;
    if (!desc->device_buf || ((uintptr_t)desc->device_buf & 255)) return LORA_ERR_INVALID_ARG;
    if (desc->device_buf_bytes < need) return LORA_ERR_BUFFER_TOO_SMALL;
    lora_kv *kv = new (std::nothrow) lora_kv;
    if (!kv) return LORA_ERR_INVALID_ARG;
    kv->device = desc->device;
    kv->num_layers = desc->num_layers;
    kv->num_pages = desc->num_pages;
    kv->page_size = desc->page_size;
    while ((1 << kv->page_shift) < desc->page_size) ++kv->page_shift;
    kv->hq = desc->num_q_heads;
    kv->hkv = desc->num_kv_heads;
    kv->group = kv->hq / kv->hkv;
    kv->d = desc->head_dim;
    kv->base = (unsigned char *)desc->device_buf;
    kv->status_dev = (int32_t *)kv->base;
    kv->page_bytes = page_bytes_of(desc);
    kv->layer_bytes = layer_bytes_of(desc);
    DeviceGuard g(desc->device);
    cudaError_t e = g.ok ? cudaSuccess : cudaErrorInvalidDevice;
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&kv->sm_count, cudaDevAttrMultiProcessorCount, desc->device);
    if (e == cudaSuccess) e = cudaMemset(kv->base, 0, 256);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) {
        delete kv;
        return cuda_fail(e);
    }
    *out = kv;
    return LORA_OK;
}

lora_status_t lora_kv_destroy(lora_kv_t *kv) {
    if (!kv) return LORA_ERR_INVALID_ARG;
    delete kv;
    return LORA_OK;
}

lora_status_t lora_kv_check_status(lora_kv_t *kv, void *stream, int32_t *words_out) {
    if (!kv) return LORA_ERR_INVALID_ARG;
    DeviceGuard g(kv->device);
    int32_t w[STATUS_WORDS];
    LORA_CUDA_TRY(cudaMemcpyAsync(w, kv->status_dev, sizeof(w), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
    LORA_CUDA_TRY(cudaStreamSynchronize((cudaStream_t)stream));
    if (words_out)
        for (int i = 0; i < STATUS_WORDS; ++i) words_out[i] = w[i];
    return w[STATUS_TIMEOUTS] ? LORA_ERR_TIMEOUT : LORA_OK;
}

}  // extern "C"
