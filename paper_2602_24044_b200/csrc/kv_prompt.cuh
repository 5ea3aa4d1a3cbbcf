// Attention of prompts (many query rows a request) over the 4-bit cache on the 5th-generation tensor cores.
//
//   x = scale q . k_t ,  k_t = z_t + s_t (c_t - 8) ,  z_t = low_t + 8 s_t
// enters the tensor cores whole, so that a score needs nothing of its key afterwards: s_t has 8 significant
// bits and c_t - 8 three (or is a power of two), so s_t (c_t - 8) is exact in fp16, and sum(q) z_t is one
// more step of 16 columns with both factors split into fp16 parts.  Queries (8 bits) are exact in fp16 once
// a row is divided by a power of two; keys and values of a block are divided by a common power of two,
// raised like the maximum.  Values enter as fp16(low_t + s_t c_t), rounded once to 11 bits like the
// probabilities (by way of z_t, which is rounded to 11 bits itself, a small value beside a large scale was off by
// several per cent).
//
// What bounds it: a block of 128 keys against 256 rows is 2100 cycles of tensor pipe, 2048 of the
// exponential unit, about 2300 of shared memory (operands of the products 1650, widened tiles in and out
// 650) and about 1400 issue slots a scheduler: all near each other.  A version that kept the codes as they
// are and applied scale and low to every score read 4 numbers a key and row from shared memory, 4096 cycles
// more.  Hence 256 rows a block of threads, as two tiles of 128 whose softmax and matrix products
// alternate, and everything else on warps of its own:
//   warps 0-3, 4-7   softmax of tile 0, tile 1: a thread is a row; scores from tensor memory to registers,
//                    probabilities back to the same tensor-memory columns, which the second product reads
//                    as its A operand; rescales the accumulator itself when its maximum was raised; brings its
//                    row of the next (item, head)'s queries while the last products of this one run (a warp that
//                    brought them for 128 rows was 4.5 us a pair)
//   warps 8-11       widen the codes of a block of keys, K and V, into three swizzled tiles (order K0 V0 K1 ..)
//   warp 12          issues the matrix products
//   warp 13          requests the cells (bulk copies), two blocks ahead
// The (item, head, block) triples form one walk cut into equal spans, one per SM; what a span's ends cut is
// joined afterwards.  Tensor memory: scores of both tiles (2 x 128 columns), accumulators (2 x head_dim).
//
// Measured: 2048 tokens on 30001 cached keys 1.24 ms (840 TFLOP/s), 5400 cycles a block: the issuing warp is in
// the products 43 % of them and waits for probabilities 20 % and for widened tiles 24 %.  32 prompts of 32..2048
// tokens 263 us, of which the blocks at that pace are 143.  Measured and not faster (the first case, 1.22..1.27 ms at the time): two threads a row 1.30..1.33,
// eight widening warps 1.28, all scores in registers 1.33, an eighth or a quarter of the exponentials as
// polynomials 1.26, 1.31.
#pragma once

#include <cuda_fp16.h>

#include "kv_decode.cuh"

namespace lora {

namespace tcp {
__device__ __forceinline__ void tmem_alloc(uint32_t *dst_smem, uint32_t ncols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst_smem)),
                 "r"(ncols)
                 : "memory");
}
__device__ __forceinline__ void tmem_relinquish() {
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t ncols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D[tmem] (+)= A[smem] . B[smem]; A[tmem] . B[smem].  Descriptors come as their low words (start address and
// leading offset); the high word is the layout's.
template <uint32_t HI>
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(HI)
        : "memory");
}
template <uint32_t HI>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(HI)
        : "memory");
}
// one lane of the (converged) warp
__device__ __forceinline__ bool elect() {
    uint32_t is;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(is));
    return is != 0;
}
// one arrival on the mbarrier when every product issued so far by this thread has completed
__device__ __forceinline__ void commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
                 : "memory");
}
#define LORA_R32(r, o)                                                                                             \
    "=r"(r[o + 0]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), \
        "=r"(r[o + 7]), "=r"(r[o + 8]), "=r"(r[o + 9]), "=r"(r[o + 10]), "=r"(r[o + 11]), "=r"(r[o + 12]),           \
        "=r"(r[o + 13]), "=r"(r[o + 14]), "=r"(r[o + 15]), "=r"(r[o + 16]), "=r"(r[o + 17]), "=r"(r[o + 18]),        \
        "=r"(r[o + 19]), "=r"(r[o + 20]), "=r"(r[o + 21]), "=r"(r[o + 22]), "=r"(r[o + 23]), "=r"(r[o + 24]),        \
        "=r"(r[o + 25]), "=r"(r[o + 26]), "=r"(r[o + 27]), "=r"(r[o + 28]), "=r"(r[o + 29]), "=r"(r[o + 30]),        \
        "=r"(r[o + 31])
// 32 lanes x 32 columns -> registers o .. o + 31 of every thread (lane = thread)
#define LORA_TMEM_LD32(addr, r, o)                                                                                \
    asm volatile(                                                                                                 \
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, " \
        "%15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"              \
        : LORA_R32(r, o)                                                                                          \
        : "r"(addr)                                                                                               \
        : "memory")
template <int N>
__device__ __forceinline__ void st32(uint32_t addr, const uint32_t (&r)[N], int o) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
        "%14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[o + 0]),
        "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7]),
        "r"(r[o + 8]), "r"(r[o + 9]), "r"(r[o + 10]), "r"(r[o + 11]), "r"(r[o + 12]), "r"(r[o + 13]), "r"(r[o + 14]),
        "r"(r[o + 15]), "r"(r[o + 16]), "r"(r[o + 17]), "r"(r[o + 18]), "r"(r[o + 19]), "r"(r[o + 20]), "r"(r[o + 21]),
        "r"(r[o + 22]), "r"(r[o + 23]), "r"(r[o + 24]), "r"(r[o + 25]), "r"(r[o + 26]), "r"(r[o + 27]), "r"(r[o + 28]),
        "r"(r[o + 29]), "r"(r[o + 30]), "r"(r[o + 31]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void ld16(uint32_t addr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
        "[%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
}
template <int N>
__device__ __forceinline__ void st16(uint32_t addr, const uint32_t (&r)[N]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
        : "memory");
}
// Shared-memory matrix descriptors.  Low word: start address and leading offset in 16-byte units.  High
// word: stride offset, version, layout (2: 128-byte swizzle, 0: 8 x 8 core matrices).
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lead) { return ((addr & 0x3FFFFu) >> 4) | (lead >> 4) << 16; }
constexpr uint32_t desc_hi(uint32_t stride, uint32_t layout) { return (stride >> 4) | 1u << 14 | layout << 29; }
constexpr uint32_t HI_SWIZZLED = desc_hi(1024, 2), HI_CORES = desc_hi(128, 0);
// fp32 accumulator; a, b: 0 = fp16, 1 = bf16; b_n: B's rows run along N
__host__ __device__ constexpr uint32_t instr(uint32_t type, uint32_t N, uint32_t b_n) {
    return (1u << 4) | (type << 7) | (type << 10) | (b_n << 16) | ((N >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void sts_v4(uint32_t addr, const uint32_t (&v)[4]) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3])
                 : "memory");
}
}  // namespace tcp

__device__ __forceinline__ uint32_t half2_of(float x) { return pack_f16(x, x); }
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ float f16_round(float x) { return __half2float(__float2half_rn(x)); }
// x as three fp16 parts
struct Split { float h, l, t; };
__device__ __forceinline__ Split split_f16(float x) {
    Split s;
    s.h = f16_round(x);
    s.l = f16_round(x - s.h);
    s.t = f16_round(x - s.h - s.l);
    return s;
}

// the n lowest bits (n may lie outside 0 .. 32)
__device__ __forceinline__ uint32_t low_bits(int32_t n) {
    return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
}

constexpr int PK_THREADS = 448, PK_TILES = 3, PK_RAW = 2, PK_INFO = 3;
// A score may pass the running maximum by PK_RAISE (log2), a row of keys or values the common exponent by
// PK_RAISE_E.  Probabilities come with a power of two, so that the largest is 2^15, half of what fp16 holds: 11
// bits then reach down to 2^-23 of the largest, and smaller ones are off by 2^-34 of it at most.  (With the largest
// at 2^8, 8000 keys 2^-25 below one whose value is zero had 35 % of their weight misrounded.)
constexpr float PK_RAISE = 6.0f, PK_UNIT = 15.0f - PK_RAISE;
constexpr int PK_RAISE_E = 7;
constexpr int PK_NO_EXPONENT = -126, PK_MOST_EXPONENT = 126;
constexpr int PK_EXTRA = 128 * 16 * 2;       // 16 more columns of 128 rows, as core matrices

struct PromptInfo {          // of a block of keys, from the widening warps to the softmax
    int32_t ek, ev;          // exponents taken out of the keys, of the values
    uint32_t valid;          // cells that are there
    uint32_t bad[4];         // value rows that are no numbers (their tile rows are zero)
    uint32_t reserved;
};

template <int D>
struct PromptCfg {
    static constexpr int CELL = kv_cell_bytes(D);
    static constexpr int RAW = 8 * CELL;                    // a block of 128 keys as it lies in the cache
    static constexpr int TILE = 128 * D * 2;                // 128 rows of 16-bit values
    static constexpr int OFF_KV = 2 * TILE;                 // behind the queries of both tiles
    static constexpr int OFF_QX = OFF_KV + PK_TILES * TILE; // the further columns: queries of both tiles,
    static constexpr int OFF_KX = OFF_QX + 2 * PK_EXTRA;    // keys of the tiles
    static constexpr int OFF_RAW = OFF_KX + PK_TILES * PK_EXTRA;
    static constexpr int OFF_INFO = OFF_RAW + PK_RAW * RAW;
    static constexpr int OFF_BAR = OFF_INFO + PK_INFO * (int)sizeof(PromptInfo);
    static constexpr int SMEM = OFF_BAR + 512 + 1024;       // 1024: the swizzled tiles' alignment
};

// A walker's cursor over its span: (item, head, block) in order.
struct PromptCursor {
    static constexpr int OVER = KV_PROMPT_OVER;
    const KvItem *items;
    KvItem it;
    int64_t left;             // places of the span that are left, from the pair's first chunk or the span's start on
    int32_t index, head, chunk, hkv;
    __device__ __forceinline__ PromptCursor(const KvItem *list, int32_t first, int64_t s0, int64_t s1, int32_t heads)
        : items(list), index(first), hkv(heads) {
        it = load_item(items + index);
        const int64_t off = s0 - hkv * it.start;
        head = (int32_t)(off / (it.n + OVER));
        const int32_t place = (int32_t)(off - (int64_t)head * (it.n + OVER));
        chunk = max(place - OVER, 0);
        left = s1 - s0 - max(OVER - place, 0);
    }
    __device__ __forceinline__ bool more() const { return left > 0; }
    // blocks of the current (item, head) that belong to the span
    __device__ __forceinline__ int32_t last_chunk() const { return (int32_t)min((int64_t)it.n, chunk + left); }
    // is there a block behind the current pair's?
    __device__ __forceinline__ bool another_pair() const { return left > it.n - chunk + OVER; }
    __device__ __forceinline__ void next_pair(int32_t blocks) {
        left -= blocks + OVER;
        chunk = 0;
        if (++head == hkv) {
            head = 0;
            if (left > 0) it = load_item(items + ++index);
        }
    }
};

template <int D>
__global__ void __launch_bounds__(PK_THREADS, 1) prompt_attention_kernel(const AttnParams P) {
    using C = PromptCfg<D>;
    extern __shared__ __align__(1024) unsigned char pk_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>(((uintptr_t)pk_raw + 1023) & ~(uintptr_t)1023);
    uint64_t *raw_full = reinterpret_cast<uint64_t *>(smem + C::OFF_BAR);
    uint64_t *raw_empty = raw_full + PK_RAW;
    uint64_t *kv_full = raw_empty + PK_RAW;
    uint64_t *kv_empty = kv_full + PK_TILES;
    uint64_t *s_full = kv_empty + PK_TILES;       // [2] scores of a tile are in tensor memory
    uint64_t *p_ready = s_full + 2;               // [2] probabilities are
    uint64_t *o_full = p_ready + 2;               // [2] the accumulator of an (item, head) is complete
    uint64_t *q_ready = o_full + 2;               // [2] queries are in shared memory
    uint64_t *q_free = q_ready + 2;               // [2] the last score product of an (item, head) is done
    uint64_t *info_full = q_free + 2;
    uint64_t *info_empty = info_full + PK_INFO;
    uint64_t *drained = info_empty + PK_INFO;     // every product has completed
    uint32_t *valid_s = reinterpret_cast<uint32_t *>(drained + 1);      // [PK_RAW] cells that are there
    uint32_t *most_s = valid_s + PK_RAW;          // [2][8] largest key and value row of a block, per warp
    uint32_t *tmem_slot = most_s + 16;
    PromptInfo *infos = reinterpret_cast<PromptInfo *>(smem + C::OFF_INFO);
    volatile uint32_t *failed = tmem_slot + 1;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const KvWalk *walk = reinterpret_cast<const KvWalk *>(P.tables + P.L.walk) + 1;
    const int64_t s0 = blockIdx.x * walk->span, s1 = min(s0 + walk->span, walk->total);
    if (s0 >= s1) return;
    const KvItem *items = reinterpret_cast<const KvItem *>(P.tables + P.L.pr_items);
    const int32_t first = __ldg(P.tables + P.L.pr_first + blockIdx.x);
    const int32_t group = P.kv.group;
    PromptCursor cur(items, first, s0, s1, P.kv.hkv);
    if (!cur.more()) return;      // only empty places (the same for the whole block)

    if (tid == 0) {
        for (int i = 0; i < PK_RAW; ++i) { mbar_init(&raw_full[i], 1); mbar_init(&raw_empty[i], 4); }
        for (int i = 0; i < PK_TILES; ++i) { mbar_init(&kv_full[i], 4); mbar_init(&kv_empty[i], 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&p_ready[i], 128);
            mbar_init(&o_full[i], 1);
            mbar_init(&q_ready[i], 128);
            mbar_init(&q_free[i], 1);
        }
        for (int i = 0; i < PK_INFO; ++i) { mbar_init(&info_full[i], 4); mbar_init(&info_empty[i], 8); }
        mbar_init(drained, 1);
        *failed = 0;
        fence_mbar_init();
    }
    // the columns that no part fills stay zero
    for (int i = tid; i < (2 + PK_TILES) * PK_EXTRA / 16; i += PK_THREADS)
        *reinterpret_cast<uint4 *>(smem + C::OFF_QX + i * 16) = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async();
    if (warp == 12) {
        tcp::tmem_alloc(tmem_slot, 512);
        tcp::tmem_relinquish();
    }
    tcp::fence_before();
    __syncthreads();
    tcp::fence_after();
    const uint32_t tmem = *tmem_slot;
    griddep_launch_dependents();
    // a wait gives up after a limit, or when another warp has
    auto wait = [&](uint64_t *bar, uint32_t parity) -> bool {
        for (uint32_t i = 0; i < WAIT_POLLS; ++i) {
            if (mbar_try_wait(bar, parity)) return true;
            if (*failed) return false;
        }
        *failed = 1;
        return false;
    };
    if (warp < 8) {
        // =========================== softmax: a thread is a row ====================================
        const int t = warp >> 2, row = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + lanes + t * 128, o_at = tmem + lanes + 256 + t * D;
        // The queries of a pair.  A warp requests its 32 rows (whole lines; before the wait for the pair before
        // it), lays them out as they came, and then every thread takes its own row: as fp16 divided by a power of
        // two, in place, and its sum in parts.  Returns log2(e) |scale| times that power.  (A negative scale turns
        // the queries.)
        auto take_queries = [&](const KvItem &it, int32_t head, uint32_t pair, bool &ok) -> float {
            constexpr int LPR = D / 8, RPI = 32 / LPR;       // lanes of a row, rows of a request
            const int run = lane % LPR;
            const uint32_t tile = smem_u32(smem) + t * C::TILE;
            {
                uint4 v[LPR];
                const int32_t my0 = t * 128 + (warp & 3) * 32 + lane / LPR;
                const int32_t r0 = it.row0 + my0;
                int32_t tok = r0 / group, h = r0 - tok * group;
                const __nv_bfloat16 *src = P.q + it.tok0 * P.ldq + (int64_t)head * group * D + run * 8;
#pragma unroll
                for (int i = 0; i < LPR; ++i) {
                    v[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (my0 + i * RPI < it.nrows) v[i] = __ldg(reinterpret_cast<const uint4 *>(src + tok * P.ldq + h * D));
                    h += RPI;
                    while (h >= group) { h -= group; ++tok; }
                }
                if (pair > 0) ok = ok && wait(&q_free[t], (pair - 1) & 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) return 0.0f;
#pragma unroll
                for (int i = 0; i < LPR; ++i) {
                    const int rr = (warp & 3) * 32 + lane / LPR + i * RPI;
                    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                    tcp::sts_v4(tile + (run >> 3) * 16384 + rr * 128 + (((run & 7) ^ (rr & 7)) << 4), w);
                }
            }
            __syncwarp();
            const uint32_t q_at = tile + row * 128;
            uint32_t most = 0;
#pragma unroll 4
            for (int i = 0; i < D / 8; ++i) {
                uint32_t v[4];
                lds_v4(q_at + (i >> 3) * 16384 + (((i & 7) ^ (row & 7)) << 4), v);
                most = max_u16x2(most, max_u16x2(max_u16x2(v[0] & 0x7fff7fffu, v[1] & 0x7fff7fffu),
                                                 max_u16x2(v[2] & 0x7fff7fffu, v[3] & 0x7fff7fffu)));
            }
            most = max(most << 16, most & 0xffff0000u);
            const int a = most >= 0x7f800000u ? 0 : max((int)(most >> 23) - 126, -126);     // |q| < 2^a
            const float unit = copysignf(pow2(max(-a, -126)), P.scale2);
            float sum = 0.0f;
#pragma unroll 4
            for (int i = 0; i < D / 8; ++i) {
                const uint32_t at = q_at + (i >> 3) * 16384 + (((i & 7) ^ (row & 7)) << 4);
                uint32_t v[4];
                lds_v4(at, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float lo = __uint_as_float(v[e] << 16) * unit, hi = __uint_as_float(v[e] & 0xffff0000u) * unit;
                    sum += lo + hi;
                    v[e] = pack_f16(lo, hi);
                }
                tcp::sts_v4(at, v);
            }
            const Split q = split_f16(sum);
            const uint32_t qx[4] = {pack_f16(q.h, q.h), pack_f16(q.l, q.l), pack_f16(q.h, q.t), 0u};
            tcp::sts_v4(smem_u32(smem) + C::OFF_QX + t * PK_EXTRA + (row >> 3) * 128 + (row & 7) * 16, qx);
            fence_proxy_async();
            mbar_arrive(&q_ready[t]);
            return fabsf(P.scale2) * pow2(min(max(a, -126), 126));
        };
        uint32_t j = 0, pair = 0;
        bool ok = true;
        float q_unit = take_queries(cur.it, cur.head, 0, ok);
        for (; ok && cur.more(); ++pair) {
            const int32_t c0 = cur.chunk, c1 = cur.last_chunk();
            const int32_t r = cur.it.row0 + t * 128 + row;
            const int32_t my = t * 128 + row;
            // rows past the item's end (their queries are zero) follow the last one's limit
            const int32_t last_row = cur.it.row0 + cur.it.nrows - 1;
            const int32_t lim = cur.it.lim0 + min(r, last_row) / group;
            const int32_t lo = P.window > 0 ? lim - P.window : 0;
            const int32_t lim_min = cur.it.lim0 + min(cur.it.row0 + t * 128, last_row) / group;
            const int32_t lo_max = P.window > 0 ? cur.it.lim0 + min(cur.it.row0 + t * 128 + 127, last_row) / group - P.window : 0;
            float m = -INFINITY, l = 0.0f;      // m: a maximum less PK_UNIT
            int ve = PK_NO_EXPONENT;
            for (int32_t ch = c0; ch < c1; ++ch, ++j) {
                const uint32_t ps = j % PK_INFO;
                ok = wait(&info_full[ps], (j / PK_INFO) & 1u) && wait(&s_full[t], j & 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tcp::fence_after();
                const PromptInfo *info = infos + ps;
                const int ve_new = info->ev;
                const uint32_t valid = info->valid;
                const float f = fminf(fmaxf(q_unit * pow2(info->ek), 1.17549435e-38f), 3e38f);     // never 0 or inf: masked scores stay -inf
                const int32_t key0 = cur.it.k_lo + ch * KV_PROMPT_CHUNK;
                const bool whole = valid == 0xffu && key0 + 128 <= lim_min && key0 >= lo_max;
                const bool any_bad = (info->bad[0] | info->bad[1] | info->bad[2] | info->bad[3]) != 0;
                // The scores are read twice (tensor memory is fast; 128 registers of them are not there), 32
                // columns at a time, the next on their way while these are worked on.
                float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                uint32_t xa[32];
                auto largest = [&](uint32_t (&x)[32], int h) {
                    if (!whole) {      // what a row does not see goes back as -inf
                        const int32_t k = key0 + h;       // bit i is key k + i
                        const uint32_t cells = valid >> (h >> 4);
                        const uint32_t seen = low_bits(lim - k) & ~low_bits(lo - k) &
                                              (((cells & 1u) ? 0xffffu : 0u) | ((cells & 2u) ? 0xffff0000u : 0u));
                        // a value row that is no number makes the rows that see it no numbers
                        if (any_bad && (seen & info->bad[h >> 5])) l = NAN;
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = (seen >> i) & 1u ? x[i] : 0xff800000u;
                        tcp::st32(s_at + h, x, 0);
                    }
#pragma unroll
                    for (int i = 0; i < 32; i += 2)
                        mx4[(i >> 1) & 3] = fmaxf(fmaxf(mx4[(i >> 1) & 3], __uint_as_float(x[i])), __uint_as_float(x[i + 1]));
                };
#pragma unroll 1
                for (int h = 0; h < 128; h += 32) {
                    LORA_TMEM_LD32(s_at + h, xa, 0);
                    tcp::wait_ld();
                    largest(xa, h);
                }
                if (!whole) tcp::wait_st();
                else if (any_bad) l = NAN;
                float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
                mx = mx == -INFINITY ? mx : mx * f;
                if (__any_sync(0xffffffffu, mx > m + (PK_UNIT + PK_RAISE) || ve_new != ve)) {
                    const float mn = mx > m + (PK_UNIT + PK_RAISE) ? mx - PK_UNIT : m;
                    const float fm = mn == m ? 1.0f : exp2_approx(m - mn), fe = fm * pow2(max(ve - ve_new, -126));
                    m = mn;
                    ve = ve_new;
                    l *= fm;
                    if (ch > c0) {     // the products of the blocks before have completed: their scores' successor is here
#pragma unroll
                        for (int cc = 0; cc < D; cc += 16) {
                            uint32_t o[16];
                            tcp::ld16(o_at + cc, o);
                            tcp::wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * fe);
                            tcp::st16(o_at + cc, o);
                        }
                        tcp::wait_st();
                    }
                }
                // a row that sees nothing has no maximum: its probabilities are 2^(-inf - 0)
                const float mm = m == -INFINITY ? 0.0f : m;
                const uint64_t f2 = pack2f(f, f), nm = pack2f(-mm, -mm);
                uint64_t l2[2] = {0, 0};
                auto spread = [&](uint32_t (&x)[32], int h) {     // (probabilities h / 2 .. overwrite scores that have been read)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float a, b;
                        unpack2f(fma2(pack2f(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), f2, nm),
                                      a, b);
                        a = exp2_approx(a);
                        b = exp2_approx(b);
                        l2[i & 1] = add2(l2[i & 1], pack2f(a, b));
                        x[i] = pack_f16(a, b);
                    }
                    tcp::st16(s_at + h / 2, x);
                };
#pragma unroll 1
                for (int h = 0; h < 128; h += 32) {
                    LORA_TMEM_LD32(s_at + h, xa, 0);
                    tcp::wait_ld();
                    spread(xa, h);
                }
                float a, b;
                unpack2f(add2(l2[0], l2[1]), a, b);
                l += a + b;
                tcp::wait_st();
                tcp::fence_before();
                mbar_arrive(&p_ready[t]);
                __syncwarp();
                if (lane == 0) mbar_arrive(&info_empty[ps]);
            }
            if (!ok) break;
            // the next pair's queries, while the last product runs
            float next_unit = 0.0f;
            if (cur.another_pair()) {
                const bool same = cur.head + 1 < cur.hkv;
                const KvItem next = same ? cur.it : load_item(items + cur.index + 1);
                next_unit = take_queries(next, same ? cur.head + 1 : 0, pair + 1, ok);
            }
            if (!ok) break;
            // ---- the (item, head) is over, or the span is ------------------------------------------
            ok = wait(&o_full[t], pair & 1u);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tcp::fence_after();
            const bool live = my < cur.it.nrows, complete = c0 == 0 && c1 == cur.it.n;
            const float inv = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l, back = pow2(ve);
            const int32_t tok = cur.it.tok0 + r / group, hq = cur.head * group + r % group;
            const int64_t slot = (2 * (int64_t)blockIdx.x + (c0 == 0 ? 1 : 0)) * KV_PROMPT_ROWS + my;
#pragma unroll
            for (int cc = 0; cc < D; cc += 32) {
                uint32_t o[32];
                LORA_TMEM_LD32(o_at + cc, o, 0);
                tcp::wait_ld();
                if (live) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * inv * back);
                    if (complete) {
                        uint4 *dst = reinterpret_cast<uint4 *>(P.out + tok * P.ldo + (int64_t)hq * D + cc);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t h[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const __nv_bfloat162 b2 = __floats2bfloat162_rn(__uint_as_float(o[8 * e + 2 * k]),
                                                                                __uint_as_float(o[8 * e + 2 * k + 1]));
                                h[k] = *reinterpret_cast<const uint32_t *>(&b2);
                            }
                            dst[e] = make_uint4(h[0], h[1], h[2], h[3]);
                        }
                    } else {
                        uint4 *dst = reinterpret_cast<uint4 *>(P.part + slot * D + cc);
#pragma unroll
                        for (int e = 0; e < 8; ++e) dst[e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                    }
                }
            }
            if (live) {
                if (!complete) P.part_ml[slot] = make_float2(m, l);
                else if (P.lse) P.lse[(int64_t)tok * P.kv.hq + hq] = inv == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718f;
            }
            tcp::fence_before();
            q_unit = next_unit;
            cur.next_pair(c1 - c0);
        }
    } else if (warp < 12) {
        // =========================== widening ======================================================
        const int id = tid - 256, wq = warp - 8, kr = id >> 2, c = id & 3;
        uint32_t j = 0, u = 0;        // blocks, tiles
        // a warp whose wait failed still takes part in the named barrier of the next block, where all four
        // learn of it and leave together
        bool ok = true, dead = false;
        while (!dead && cur.more()) {
            const int32_t c0 = cur.chunk, c1 = cur.last_chunk();
            const int32_t end = cur.it.lim0 + (cur.it.row0 + cur.it.nrows - 1) / group;
            int ek = PK_NO_EXPONENT, ev = PK_NO_EXPONENT;
            for (int32_t ch = c0; ch < c1; ++ch, ++j) {
                const uint32_t rs = j % PK_RAW, ps = j % PK_INFO;
                const uint32_t raw = smem_u32(smem) + C::OFF_RAW + rs * C::RAW;
                ok = ok && wait(&raw_full[rs], (j / PK_RAW) & 1u);
                if (ok && j >= PK_INFO) ok = wait(&info_empty[ps], (j / PK_INFO - 1) & 1u);
                // the common exponents: a thread is a key
                const uint32_t valid = valid_s[rs];
                const int32_t left = end - (cur.it.k_lo + ch * KV_PROMPT_CHUNK);     // keys of the block that are there
                float ks = 0.0f, kl = 0.0f;
                uint32_t kmag = 0, vmag = 0;
                bool bad = false;
                if (((valid >> (id >> 4)) & 1u) && id < left) {
                    const uint32_t at = raw + (id >> 4) * C::CELL + kv_cell_params(D) + (id & 15) * 4;
                    const uint32_t kp = lds_u32(at), vp = lds_u32(at + KV_CELL * 4);
                    ks = __uint_as_float(kp << 16);
                    kl = __uint_as_float(kp & 0xffff0000u);
                    kmag = max(kp << 16, kp & 0x7fff0000u);
                    vmag = max(vp << 16, vp & 0x7fff0000u);
                    bad = vmag >= 0x7f800000u;
                    if (kmag >= 0x7f800000u) kmag = 0;
                    if (bad) vmag = 0;
                }
                kmag = __reduce_max_sync(0xffffffffu, kmag);
                vmag = __reduce_max_sync(0xffffffffu, vmag);
                const uint32_t bad_keys = __ballot_sync(0xffffffffu, bad);
                uint32_t *most = most_s + (j & 1u) * 8;
                if (lane == 0) {
                    most[wq] = kmag;
                    most[4 + wq] = vmag;
                }
                uint32_t any_bad;      // all four warps take the same decision
                asm volatile(
                    "{\n\t.reg .pred p, q;\n\t"
                    "setp.ne.u32 p, %1, 0;\n\t"
                    "bar.red.or.pred q, 1, 128, p;\n\t"
                    "selp.u32 %0, 1, 0, q;\n\t}"
                    : "=r"(any_bad)
                    : "r"(ok ? 0u : 1u)
                    : "memory");
                if (any_bad) { dead = true; break; }
                ek = raise_exponent<PK_RAISE_E, PK_MOST_EXPONENT>(ek, max(max(most[0], most[1]), max(most[2], most[3])));
                ev = raise_exponent<PK_RAISE_E, PK_MOST_EXPONENT>(ev, max(max(most[4], most[5]), max(most[6], most[7])));
                const float k_unit = pow2(-ek), v_unit = pow2(-ev);
                if (lane == 0) {
                    PromptInfo *info = infos + ps;
                    info->bad[wq] = bad_keys;
                    if (wq == 0) {
                        info->ek = ek;
                        info->ev = ev;
                        info->valid = valid;
                    }
                    mbar_arrive(&info_full[ps]);
                }
                // codes: K, then V.  Four lanes share a row; those of the second pair take their two halves
                // in the other order, so that the eight lanes of a store phase hit eight different banks
                // (one small loop for both: the roles' code together has to fit the instruction cache)
#pragma unroll 1
                for (int kv = 0; kv < 2; ++kv, ++u) {
                    const uint32_t b = u % PK_TILES, tile = smem_u32(smem) + C::OFF_KV + b * C::TILE;
                    if (u >= PK_TILES) ok = ok && wait(&kv_empty[b], (u / PK_TILES - 1) & 1u);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (kv == 0) {     // sum(q) z_t: parts (h, l, h, l, t, h) against the queries' (h, h, l, l, h, t)
                        const Split z = split_f16(fmaf(8.0f, ks, kl) * k_unit);
                        const uint32_t kx[4] = {pack_f16(z.h, z.l), pack_f16(z.h, z.l), pack_f16(z.t, z.h), 0u};
                        tcp::sts_v4(smem_u32(smem) + C::OFF_KX + b * PK_EXTRA + (id >> 3) * 128 + (id & 7) * 16, kx);
                    }
                    const float unit = kv ? v_unit : k_unit;
                    // keys become s (c - 8), values low + s c: codes less 8 or as they are
                    const uint32_t off_lo = kv ? 0x64006400u : 0x64086408u, off_hi = kv ? 0xd400d400u : 0xd480d480u;
#pragma unroll 1
                    for (int i = 0; i < 4; ++i) {
                        const int key = i * 32 + kr;
                        const uint32_t cell = raw + (key >> 4) * C::CELL + kv * KV_CELL * (D / 2);
                        const uint32_t src = cell + (key & 15) * (D / 2) + c * (D / 8);
                        // a row that is not there, or whose values are no numbers, becomes zero
                        const uint32_t par = lds_u32(raw + (key >> 4) * C::CELL + kv_cell_params(D) + (kv * KV_CELL + (key & 15)) * 4);
                        uint32_t w[D / 32];
                        if constexpr (D == 128) lds_v4(src, w);
                        else lds_v2(src, w);
                        const float sf = __uint_as_float(par << 16), lf = __uint_as_float(par & 0xffff0000u);
                        const bool there = ((valid >> (key >> 4)) & 1u) && key < left &&
                                           (kv == 0 || max(par << 16, par & 0x7fff0000u) < 0x7f800000u);
                        const uint32_t s2 = half2_of(there ? sf * unit : 0.0f);
                        const uint32_t z2 = half2_of(there && kv ? lf * unit : 0.0f);      // (keys get theirs in the further columns)
                        const uint32_t dst = tile + (c * (D / 32) >> 3) * 16384 + key * 128;
#pragma unroll
                        for (int e = 0; e < D / 32; ++e) {
                            // lanes 2 and 3 of a row begin with their second half
                            const int we = D == 128 ? e ^ (c & 2) : e;
                            const uint32_t we_w = D == 128 ? ((c & 2) ? w[e ^ 2] : w[e]) : w[e];
                            uint32_t v[4] = {widen_f16_lo(we_w, off_lo), widen_f16_hi(we_w, off_hi), widen_f16_lo(we_w >> 8, off_lo),
                                             widen_f16_hi(we_w >> 8, off_hi)};
#pragma unroll
                            for (int q = 0; q < 4; ++q) v[q] = fma_f16x2(v[q], s2, z2);
                            tcp::sts_v4(dst + (((c * (D / 32) + we) & 7) ^ (key & 7)) * 16, v);
                        }
                    }
                    fence_proxy_async();     // ordinary stores, read by the matrix unit
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&kv_full[b]);
                        if (kv == 1) mbar_arrive(&raw_empty[rs]);
                    }
                }
            }
            cur.next_pair(c1 - c0);
        }
        if (dead || !ok) *failed = 1;
    } else {
        if (warp == 12) {
            // ======================= matrix products ===============================================
            // The whole warp follows the same path (so that descriptors live in uniform registers); one
            // elected lane issues.
            constexpr uint32_t QK = tcp::instr(0, 128, 0), PV = tcp::instr(0, D, 1);
            const uint32_t base = smem_u32(smem);
            const uint32_t q_lo = tcp::desc_lo(base, 16), kv_lo = tcp::desc_lo(base + C::OFF_KV, 16);
            const uint32_t v_lo = tcp::desc_lo(base + C::OFF_KV, 16384);
            const uint32_t qx_lo = tcp::desc_lo(base + C::OFF_QX, 2048), kx_lo = tcp::desc_lo(base + C::OFF_KX, 2048);
            bool ok = true;
            // scores of tile t with the keys in tile buffer b; `done`: more barriers that learn of its end
            auto scores = [&](int t, uint32_t b, uint64_t *also, uint64_t *and_also) {
                if (tcp::elect()) {
                    const uint32_t qa = q_lo + t * (C::TILE >> 4), ka = kv_lo + b * (C::TILE >> 4);
                    // rolled: the code of all roles has to fit the instruction caches of an SM
#pragma unroll 1
                    for (int h = 0; h < D / 64; ++h)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            tcp::mma_ss<tcp::HI_SWIZZLED>(tmem + t * 128, qa + h * 1024 + k * 2, ka + h * 1024 + k * 2, QK, (h | k) > 0);
                    tcp::mma_ss<tcp::HI_CORES>(tmem + t * 128, qx_lo + t * (PK_EXTRA >> 4), kx_lo + b * (PK_EXTRA >> 4), QK, 1);
                    tcp::commit(&s_full[t]);
                    if (also) tcp::commit(also);
                    if (and_also) tcp::commit(and_also);
                }
                __syncwarp();
            };
            uint32_t j = 0, pair = 0, b = 0, b_phase = 0;      // b: the tile buffer of the block's values
            int32_t left = cur.last_chunk() - cur.chunk;      // blocks left of the current (item, head)
            bool fresh = true;                                // its first block
            ok = __all_sync(0xffffffffu, wait(&kv_full[0], 0));
#pragma unroll 1
            for (int t = 0; t < 2 && ok; ++t) {
                ok = __all_sync(0xffffffffu, wait(&q_ready[t], 0));
                tcp::fence_after();
                if (!ok) break;
                scores(t, 0, left == 1 ? &q_free[t] : nullptr, t == 1 ? &kv_empty[0] : nullptr);
            }
            b = 1;
            while (ok) {
                const bool last = left == 1;
                if (last) cur.next_pair(cur.last_chunk() - cur.chunk);
                const bool another = !last || cur.more();     // one more block follows
                const int32_t next_left = last ? (another ? cur.last_chunk() - cur.chunk : 0) : left - 1;
                const uint32_t kb = b + 1 == PK_TILES ? 0 : b + 1, kb_phase = b + 1 == PK_TILES ? b_phase ^ 1u : b_phase;
                ok = __all_sync(0xffffffffu, wait(&kv_full[b], b_phase));
#pragma unroll 1
                for (int t = 0; t < 2 && ok; ++t) {
                    ok = __all_sync(0xffffffffu, wait(&p_ready[t], j & 1u));
                    if (!ok) break;
                    tcp::fence_after();
                    if (tcp::elect()) {
                        const uint32_t va = v_lo + b * (C::TILE >> 4);
#pragma unroll 2
                        for (int k = 0; k < 8; ++k)
                            tcp::mma_ts<tcp::HI_SWIZZLED>(tmem + 256 + t * D, tmem + t * 128 + k * 8, va + k * 128, PV,
                                                          (k > 0 || !fresh) ? 1u : 0u);
                        if (last) tcp::commit(&o_full[t]);
                        if (t == 1) tcp::commit(&kv_empty[b]);
                    }
                    __syncwarp();
                    if (another) {
                        if (t == 0) ok = __all_sync(0xffffffffu, wait(&kv_full[kb], kb_phase));
                        if (ok && last) ok = __all_sync(0xffffffffu, wait(&q_ready[t], (pair + 1) & 1u));
                        if (!ok) break;
                        tcp::fence_after();
                        scores(t, kb, next_left == 1 ? &q_free[t] : nullptr, t == 1 ? &kv_empty[kb] : nullptr);
                    }
                }
                if (!ok || !another) break;
                fresh = last;
                pair += last;
                left = next_left;
                ++j;
                b = kb + 1 == PK_TILES ? 0 : kb + 1;
                b_phase = kb + 1 == PK_TILES ? kb_phase ^ 1u : kb_phase;
            }
            if (!ok) *failed = 1;
            // nothing of this block's memory may be given back while a product is in flight
            if (tcp::elect()) tcp::commit(drained);
            __syncwarp();
            mbar_wait(drained, 0);
        } else if (warp == 13) {
            // ======================= cells from the cache ==========================================
            uint32_t j = 0;
            bool ok = true;
            for (; ok && cur.more();) {
                const int32_t c0 = cur.chunk, c1 = cur.last_chunk();
                const int32_t end = cur.it.lim0 + (cur.it.row0 + cur.it.nrows - 1) / group;
                for (int32_t ch = c0; ch < c1; ++ch, ++j) {
                    const uint32_t rs = j % PK_RAW;
                    const int32_t key = cur.it.k_lo + ch * KV_PROMPT_CHUNK + lane * KV_CELL;
                    int32_t page = -1;
                    if (lane < 8 && key < end) {
                        page = __ldg(P.block_table + cur.it.req * P.ld_table + (key >> P.kv.page_shift));
                        if (page < 0 || page >= P.kv.num_pages) page = -1;
                    }
                    const uint32_t valid = __ballot_sync(0xffffffffu, page >= 0);
                    if (j >= PK_RAW) ok = wait(&raw_empty[rs], (j / PK_RAW - 1) & 1u);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (lane == 0) {
                        valid_s[rs] = valid;
                        mbar_expect_tx(&raw_full[rs], __popc(valid) * C::CELL);
                    }
                    __syncwarp();
                    if (page >= 0)
                        bulk_g2s(smem + C::OFF_RAW + rs * C::RAW + lane * C::CELL,
                                 kv_cell(P.kv, page, cur.head, key & (P.kv.page_size - 1), C::CELL), C::CELL, &raw_full[rs]);
                }
                if (!ok) break;
                cur.next_pair(c1 - c0);
            }
            if (!ok) {
                *failed = 1;
                // copies on their way must land before the block leaves
                for (uint32_t i = j > PK_RAW ? j - PK_RAW : 0; i < j; ++i) mbar_wait(&raw_full[i % PK_RAW], (i / PK_RAW) & 1u);
            }
        }
    }
    tcp::fence_before();
    __syncthreads();
    if (tid == 0 && *failed) atomicAdd(&P.kv.status[STATUS_TIMEOUTS], 1);
    if (warp == 12) tcp::tmem_dealloc(tmem, 512);
}

}  // namespace lora
