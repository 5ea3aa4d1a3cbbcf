// Shared declarations of the 4-bit paged key/value cache: host handle, cell format, batch tables.
#pragma once

#include "common.cuh"

namespace lora {

constexpr int KV_CELL = 16;            // tokens of one cell
constexpr int KV_MAX_REQUESTS = 4096;  // of one batch (the table builder keeps them in shared memory)

// One cell: [16 x D/2 K codes][16 x D/2 V codes][16 x (scale, low) of K][16 x (scale, low) of V].
__host__ __device__ constexpr int kv_cell_bytes(int d) { return KV_CELL * (d + 8); }
__host__ __device__ constexpr int kv_cell_params(int d) { return KV_CELL * d; }   // offset of K's (scale, low)

struct KvView {                 // one layer, passed to kernels by value
    unsigned char *cells;       // page 0 of the layer
    int64_t page_bytes;         // heads * cells of a page * bytes of a cell
    int64_t head_bytes;         // cells of a page * bytes of a cell
    int32_t num_pages, page_size, page_shift;
    int32_t hq, hkv, group;
    int32_t *status;            // [STATUS_WORDS]
};

// Address of the cell that holds token `offset` (a multiple of 16 inside page `page`) of a head.
__device__ __forceinline__ unsigned char *kv_cell(const KvView &v, int32_t page, int32_t head, int32_t offset,
                                                  int cell_bytes) {
    return v.cells + page * v.page_bytes + head * v.head_bytes + (int64_t)(offset / KV_CELL) * cell_bytes;
}

// Two floats at once, each rounded by itself.
__device__ __forceinline__ uint64_t pack2f(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2f(uint64_t v, float &a, float &b) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// ---------------------------------------------------------------------------------------------
// batch tables (int32 words): public part as documented, then the attention's work lists
// ---------------------------------------------------------------------------------------------
constexpr int KVH_WORDS = 16;      // of the header, the first six in use

// A piece of attention work before it is multiplied by the key/value heads: some rows of one request
// (row = token * group + query head inside its group) against a run of key chunks.  An item of n
// chunks stands for hkv pairs (item, head) of over + n places each in the list's walk, the first at hkv *
// start: `over` empty places for what a pair costs whatever its length is (queries in, outputs out), then its
// chunks.
struct __align__(16) KvItem {
    int64_t start;     // places of the items before it (one head's)
    int32_t req;
    int32_t row0, nrows;
    int32_t k_lo;      // first key, a multiple of the chunk
    int32_t n;         // chunks, at least one
    int32_t tok0;      // the request's first token
    int32_t lim0;      // its token i sees keys below lim0 + i
    int32_t reserved[3];
};
static_assert(sizeof(KvItem) == 48, "three 16-byte words");

// The walk over a list (all items, heads and places in order) is cut into equal spans, one per walker:
// a warp of the single-token kernel, a block of the prompt kernel.
struct __align__(16) KvWalk {
    int64_t total;     // hkv * places
    int64_t span;
    int32_t n_items;
    int32_t reserved[3];
};

// Empty places of a pair.  32 prompts of 32..2048 tokens (pairs of one to sixteen chunks), 0 / 2 / 3 / 6 places:
// 435 / 275 / 262 / 303 us.  256 single tokens on 256..8192 keys, 0 / 1 / 2 / 4 places: 157 / 152 / 149 / 150 us.
constexpr int KV_DEC_OVER = 2, KV_PROMPT_OVER = 3;
constexpr int KV_DEC_CHUNK = 32;       // keys of a chunk of the single-token walk
constexpr int KV_PROMPT_CHUNK = 128;   // keys of a chunk of the prompt walk
constexpr int KV_PROMPT_ROWS = 256;    // rows of an item of the prompt walk
constexpr int KV_DEC_MAX_ROWS = 64;    // requests with more rows than this go to the prompt walk

struct KvTables {
    int64_t start, kv_len, position, slot;         // word offsets
    int64_t walk;                                  // two KvWalk: single tokens, prompts
    int64_t dec_items, pr_items;                   // KvItem lists
    int64_t dec_first, pr_first;                   // first item of each walker
    int64_t words;
};

__host__ __device__ inline KvTables kv_tables(int32_t R, int32_t T, int32_t group, int32_t dec_walkers,
                                              int32_t pr_walkers) {
    KvTables L;
    int64_t o = KVH_WORDS;
    L.start = o;    o += (int64_t)R + 1;
    L.kv_len = o;   o += R;
    L.position = o; o += T;
    L.slot = o;     o += T;
    o = (o + 3) & ~(int64_t)3;
    // a request of q tokens has ceil(q * group / rows) items: at most one more than q * group / rows
    const int64_t rows = (int64_t)T * group;
    // (the tokens of no request count as one more)
    const int64_t cd = R + 1 + rows / 8, cp = R + rows / KV_PROMPT_ROWS;
    L.walk = o;      o += 2 * (int64_t)(sizeof(KvWalk) / 4);
    L.dec_items = o; o += cd * (int64_t)(sizeof(KvItem) / 4);
    L.pr_items = o;  o += cp * (int64_t)(sizeof(KvItem) / 4);
    L.dec_first = o; o += dec_walkers;
    L.pr_first = o;  o += pr_walkers;
    L.words = (o + 3) & ~(int64_t)3;
    return L;
}

// Do T rows of `wa` bytes at pitch `lda` and T rows of `wb` bytes at pitch `ldb` touch?  Rows of one
// pitch may interleave (parts of a fused projection's rows).
inline bool rows_overlap(const void *a, int64_t wa, int64_t lda, const void *b, int64_t wb, int64_t ldb, int32_t T) {
    const char *pa = (const char *)a, *pb = (const char *)b;
    const char *ea = pa + (T - 1) * lda + wa, *eb = pb + (T - 1) * ldb + wb;
    if (ea <= pb || eb <= pa) return false;
    if (lda != ldb) return true;
    int64_t d = (pb - pa) % lda;
    if (d < 0) d += lda;
    return d < wa || d + wb > lda;
}

struct KvTableRecord {        // what the host knows of a table it built
    const void *ptr;
    int32_t R, T, max_q, window;
    uint64_t written;         // the how-manieth build through the handle
};

}  // namespace lora

struct lora_kv {
    int32_t device = 0, num_layers = 0, num_pages = 0, page_size = 0, page_shift = 0;
    int32_t hq = 0, hkv = 0, group = 0, d = 0;
    unsigned char *base = nullptr;
    int32_t *status_dev = nullptr;
    int64_t page_bytes = 0, layer_bytes = 0;
    int32_t sm_count = 148;
    bool decode_attr[4] = {false, false, false, false};   // attributes set: head_dim 64 / 128, 8 / 16 rows
    bool prompt_attr[2] = {false, false};
    bool tables_attr = false;
    // tables built through this handle, the one written longest ago forgotten first (a fixed array: no call
    // allocates)
    static constexpr int32_t MAX_TABLES = 256;
    lora::KvTableRecord tables[MAX_TABLES];
    int32_t n_tables = 0;
    uint64_t builds = 0;

    void remember(const void *ptr, int32_t R, int32_t T, int32_t max_q, int32_t window) {
        int32_t at = -1, oldest = 0;
        for (int32_t i = 0; i < n_tables && at < 0; ++i) {
            if (tables[i].ptr == ptr) at = i;
            if (tables[i].written < tables[oldest].written) oldest = i;
        }
        if (at < 0) at = n_tables < MAX_TABLES ? n_tables++ : oldest;
        tables[at] = {ptr, R, T, max_q, window, ++builds};
    }
    const lora::KvTableRecord *find(const void *ptr, int32_t R, int32_t T) const {
        for (int32_t i = 0; i < n_tables; ++i)
            if (tables[i].ptr == ptr && tables[i].R == R && tables[i].T == T) return &tables[i];
        return nullptr;
    }
    lora::KvView view(int32_t layer) const;
    // Rows of one item of the single-token walk: 8 (one column tile of the matrix instructions), or 16 where
    // a token alone has more than 8 rows.  (16 for requests of several tokens would halve their reads of the
    // cache, but the wider kernel costs every request of one token more: the single tokens of a batch of 512
    // beside four prompt chunks 229 us against 143.)
    int32_t dec_rows() const { return group <= 8 ? 8 : 16; }
    // Warps of the single-token kernel that are resident at once (its registers: 128 a thread at 8 rows,
    // 168 at 16).
    int32_t dec_walkers() const { return sm_count * (dec_rows() == 8 ? 16 : 12); }
    int32_t pr_walkers() const { return sm_count; }
};
