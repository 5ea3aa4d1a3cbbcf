// Block tables, positions, slot maps and the attention's work lists, from the requests' lengths.
//
// Integer work on a few thousand words: what bounds it is the chain of dependent steps (lengths in,
// prefix sums, tables out), not bytes.  One cluster of eight blocks, each of which recomputes all
// prefix sums for itself in shared memory (they are short), so the only exchange between blocks is the
// cluster barrier that separates the reads of the inputs from the writes (lengths and stack may be
// updated in place) and, where there are prompts, the one after which their walkers' first items are looked
// up in the list.
#include "fused_ptx.cuh"
#include "kv_common.cuh"

namespace lora {

constexpr int TB_BLOCKS = 8, TB_THREADS = 512;
constexpr int TB_WARPS = TB_THREADS / 32;

struct TableParams {
    const int32_t *kv_len, *q_len, *free_pages, *free_count;
    int32_t *block_table, *kv_len_out, *free_count_out, *out, *status;
    int64_t ld;
    int32_t R, T, max_q, window;
    int32_t num_pages, page_shift, hkv, group;
    int32_t dec_rows, dec_walkers, pr_walkers;
    KvTables L;
};

// Dynamic shared memory of a batch of R requests, as the kernel carves it up.
constexpr size_t tables_smem(int32_t R) { return (size_t)R * (2 * 8 + 6 * 4) + 2 * 32 * 8 + 2 * 32 * 4; }

// Sums that stay at the largest int32 once they pass it (with lengths that are not negative: associative).
__device__ __forceinline__ int32_t plus(int32_t a, int32_t b) {
    return (int32_t)min((uint32_t)a + (uint32_t)b, 0x7fffffffu);
}
__device__ __forceinline__ int64_t plus(int64_t a, int64_t b) { return a + b; }

template <typename I>
__device__ __forceinline__ I warp_incl(I v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const I o = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v = plus(v, o);
    }
    return v;
}

// In place: a[0 .. n) -> its inclusive prefix sums.  A thread takes consecutive entries.  In three steps, so
// that several arrays share the block's barriers: the threads' sums, the warps' sums (one warp an array), the
// entries.
template <typename I>
struct Scan {
    I *a, *warp_sum;      // [TB_WARPS]
    I sum, incl;
    __device__ __forceinline__ Scan(I *array, I *sums) : a(array), warp_sum(sums) {}
    __device__ __forceinline__ void threads(int i0, int i1) {
        sum = 0;
        for (int i = i0; i < i1; ++i) sum = plus(sum, a[i]);
        incl = warp_incl(sum);
        if ((threadIdx.x & 31) == 31) warp_sum[threadIdx.x >> 5] = incl;
    }
    __device__ __forceinline__ void warps(int warp) {
        if ((int)(threadIdx.x >> 5) != warp) return;
        const int lane = threadIdx.x & 31;
        const I v = warp_incl(lane < TB_WARPS ? warp_sum[lane] : (I)0);
        __syncwarp();
        if (lane < TB_WARPS) warp_sum[lane] = v;
    }
    __device__ __forceinline__ void entries(int i0, int i1) {
        // what lies before this thread: the warps before, the lanes before
        const I before = __shfl_up_sync(0xffffffffu, incl, 1);
        I run = plus(threadIdx.x >= 32 ? warp_sum[(threadIdx.x >> 5) - 1] : (I)0, (threadIdx.x & 31) ? before : (I)0);
        for (int i = i0; i < i1; ++i) {
            run = plus(run, a[i]);
            a[i] = run;
        }
    }
};
__device__ __forceinline__ void share_of(int n, int &i0, int &i1) {
    const int per = (n + TB_THREADS - 1) / TB_THREADS;
    i0 = min((int)threadIdx.x * per, n);
    i1 = min(i0 + per, n);
}
template <typename I>
__device__ void block_scan(I *a, int n, I *warp_sum) {
    int i0, i1;
    share_of(n, i0, i1);
    Scan<I> s(a, warp_sum);
    s.threads(i0, i1);
    __syncthreads();
    s.warps(0);
    __syncthreads();
    s.entries(i0, i1);
    __syncthreads();
}

// first i with a[i] > x, in a non-decreasing a[0 .. n)
template <typename I>
__device__ __forceinline__ int upper_bound(const I *a, int n, I x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int m = (lo + hi) >> 1;
        if (a[m] > x) hi = m; else lo = m + 1;
    }
    return lo;
}

__device__ __forceinline__ int32_t pages_for(int32_t tokens, int32_t shift) {
    return (int32_t)(((int64_t)tokens + (1 << shift) - 1) >> shift);
}

// Keys that rows row0 .. row0 + rows - 1 of a request see: [k_lo, k_hi), k_lo rounded down to a chunk.
__device__ __forceinline__ void item_range(int32_t lim0, int32_t group, int32_t window, int32_t chunk, int32_t row0,
                                           int32_t nrows, int32_t *k_lo, int32_t *n) {
    const int64_t hi = (int64_t)lim0 + (row0 + nrows - 1) / group;
    int64_t lo = window > 0 ? (int64_t)lim0 + row0 / group - window : 0;
    if (lo < 0) lo = 0;
    lo -= lo % chunk;
    *k_lo = (int32_t)(hi > lo ? lo : 0);
    *n = hi > lo ? (int32_t)((hi - lo + chunk - 1) / chunk) : 1;
}

__global__ void __launch_bounds__(TB_THREADS) build_tables_kernel(const TableParams P) {
    extern __shared__ __align__(16) unsigned char tb_smem[];
    const int R = P.R, T = P.T, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int64_t *chunks_d = reinterpret_cast<int64_t *>(tb_smem);   // prefix sums: places of the single-token list
    int64_t *chunks_p = chunks_d + R;                            // and of the prompt list
    int64_t *warp64 = chunks_p + R;                              // [2][32]
    int32_t *kv = reinterpret_cast<int32_t *>(warp64 + 64);
    int32_t *end = kv + R;        // prefix sums of the new tokens, cut at T
    int32_t *pages = end + R;     // of the pages needed
    int32_t *items_d = pages + R; // of the items
    int32_t *items_p = items_d + R;
    int32_t *failed = items_p + R;   // 1: failed
    int32_t *warp32 = failed + R;    // [2][32]
    __shared__ int32_t n_failed, n_negative, taken, sum_q;
    __shared__ int64_t walk_total[2], walk_span[2];

    if (tid == 0) n_failed = n_negative = taken = sum_q = 0;
    __syncthreads();
    for (int r = tid; r < R; r += TB_THREADS) {
        const int32_t k = P.kv_len[r], q = P.q_len[r];
        if (k < 0 || q < 0) atomicAdd(&n_negative, 1);
        kv[r] = max(k, 0);
        end[r] = max(q, 0);
        items_d[r] = max(q, 0);
    }
    const int32_t count = P.free_count ? min(max(*P.free_count, 0), P.num_pages) : 0;
    __syncthreads();
    block_scan(end, R, warp32);
    for (int r = tid; r < R; r += TB_THREADS) {
        const int32_t q = items_d[r];
        const int64_t all = (int64_t)kv[r] + q;
        // (a sum that stopped at the largest number is over T in any case: T * group is below it)
        const bool fits = end[r] <= T && q <= P.max_q && all <= (P.ld << P.page_shift) && all < 0x7fffff00;
        failed[r] = !fits;
        pages[r] = items_p[r] = fits ? pages_for((int32_t)all, P.page_shift) - pages_for(kv[r], P.page_shift) : 0;
    }
    __syncthreads();
    block_scan(pages, R, warp32);
    const int32_t all_q = R ? end[R - 1] : 0;
    for (int r = tid; r < R; r += TB_THREADS) {
        const int32_t need = items_p[r];
        if (need > 0 && pages[r] > count) failed[r] = 1;
        if (failed[r]) atomicAdd(&n_failed, 1);
        else if (need > 0) atomicMax(&taken, pages[r]);
    }
    __syncthreads();
    for (int r = tid; r < R; r += TB_THREADS) end[r] = min(end[r], T);
    if (tid == 0) sum_q = all_q;
    __syncthreads();
    const int32_t tokens = R ? end[R - 1] : 0;

    // items and chunks of every request: few for a request of single tokens, one warp each for prompts.
    // A failed request's rows, however many, are items of one empty chunk in the single-token list;
    // behind all requests' items come those of the tokens that belong to none.
    for (int r = tid; r < R; r += TB_THREADS) {
        const int32_t q = end[r] - (r ? end[r - 1] : 0);
        const int64_t rows = (int64_t)q * P.group;
        const int32_t lim0 = kv[r] + 1;
        int64_t c = 0;
        int32_t n_items = 0;
        if (failed[r])
            c = (1 + KV_DEC_OVER) * (int64_t)(n_items = (int32_t)((rows + P.dec_rows - 1) / P.dec_rows));
        else if (rows <= KV_DEC_MAX_ROWS)
            for (int32_t row0 = 0; row0 < rows; row0 += P.dec_rows, ++n_items) {
                int32_t lo, n;
                item_range(lim0, P.group, P.window, KV_DEC_CHUNK, row0, min(P.dec_rows, (int32_t)rows - row0), &lo, &n);
                c += n + KV_DEC_OVER;
            }
        chunks_d[r] = c;
        items_d[r] = n_items;
        chunks_p[r] = 0;
        items_p[r] = 0;
    }
    __syncthreads();
    // (max_q bounds every request that did not fail; a warp looks at 32 requests and takes the prompts among them)
    const bool may_prompt = (int64_t)P.max_q * P.group > KV_DEC_MAX_ROWS;
    for (int r0 = warp * 32; may_prompt && r0 < R; r0 += TB_WARPS * 32) {
        const int mine = r0 + lane;
        uint32_t mask = __ballot_sync(0xffffffffu, mine < R && !failed[mine] &&
            (int64_t)(end[mine] - (mine ? end[mine - 1] : 0)) * P.group > KV_DEC_MAX_ROWS);
        for (; mask; mask &= mask - 1) {
            const int r = r0 + __ffs(mask) - 1;
            const int64_t rows = (int64_t)(end[r] - (r ? end[r - 1] : 0)) * P.group;
            const int32_t tiles = (int32_t)((rows + KV_PROMPT_ROWS - 1) / KV_PROMPT_ROWS);
            int64_t c = 0;
            for (int32_t t = lane; t < tiles; t += 32) {
                int32_t lo, n;
                item_range(kv[r] + 1, P.group, P.window, KV_PROMPT_CHUNK, t * KV_PROMPT_ROWS,
                           (int32_t)min((int64_t)KV_PROMPT_ROWS, rows - (int64_t)t * KV_PROMPT_ROWS), &lo, &n);
                c += n + KV_PROMPT_OVER;
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) c += __shfl_xor_sync(0xffffffffu, c, d);
            if (lane == 0) {
                chunks_p[r] = c;
                items_p[r] = tiles;
            }
        }
    }
    __syncthreads();
    {
        int i0, i1;
        share_of(R, i0, i1);
        Scan<int64_t> a(chunks_d, warp64), b(chunks_p, warp64 + 32);
        Scan<int32_t> c(items_d, warp32), d(items_p, warp32 + 32);
        a.threads(i0, i1); b.threads(i0, i1); c.threads(i0, i1); d.threads(i0, i1);
        __syncthreads();
        a.warps(0); b.warps(1); c.warps(2); d.warps(3);
        __syncthreads();
        a.entries(i0, i1); b.entries(i0, i1); c.entries(i0, i1); d.entries(i0, i1);
        __syncthreads();
    }
    const int64_t spare_rows = (int64_t)(T - tokens) * P.group;
    const int32_t spare = (int32_t)((spare_rows + P.dec_rows - 1) / P.dec_rows);
    if (tid < 2) {
        const int64_t total = P.hkv * ((R ? (tid ? chunks_p : chunks_d)[R - 1] : 0) + (tid ? 0 : (1 + KV_DEC_OVER) * (int64_t)spare));
        const int32_t walkers = tid ? P.pr_walkers : P.dec_walkers;
        int64_t span = (total + walkers - 1) / walkers;
        // single tokens: no fewer than four chunks per warp, or joining the pieces costs more than
        // the split saves
        if (tid == 0 && span < 4 + KV_DEC_OVER) span = 4 + KV_DEC_OVER;
        if (span < 1) span = 1;
        walk_total[tid] = total;
        walk_span[tid] = span;
    }
    cluster_arrive();   // every block has read the lengths and the stack's count
    cluster_wait();

    const int gt = blockIdx.x * TB_THREADS + tid;
    const int all_threads = gridDim.x * TB_THREADS;
    if (gt < KVH_WORDS) {
        const int32_t h[6] = {R, T, sum_q, n_failed, n_negative, taken};
        P.out[gt] = gt < 6 ? h[gt] : 0;
    }
    if (gt == 0) {
        if (P.free_count_out) *P.free_count_out = count - taken;
        P.out[P.L.start] = 0;
    }
    if (gt < 2) {
        KvWalk w;
        w.total = walk_total[gt];
        w.span = walk_span[gt];
        w.n_items = (R ? (gt ? items_p : items_d)[R - 1] : 0) + (gt ? 0 : spare);
        w.reserved[0] = w.reserved[1] = w.reserved[2] = 0;
        reinterpret_cast<KvWalk *>(P.out + P.L.walk)[gt] = w;
    }
    for (int r = gt; r < R; r += all_threads) {
        const int32_t q = end[r] - (r ? end[r - 1] : 0);
        const int32_t after = failed[r] ? kv[r] : kv[r] + q;
        P.out[P.L.start + 1 + r] = end[r];
        P.out[P.L.kv_len + r] = after;
        if (P.kv_len_out) P.kv_len_out[r] = after;
    }
    // Half of each block's threads write what belongs to tokens and pages, the other half the work lists and
    // the walkers' first items: their chains of loads and divisions run beside each other.
    KvItem *dec = reinterpret_cast<KvItem *>(P.out + P.L.dec_items);
    KvItem *pr = reinterpret_cast<KvItem *>(P.out + P.L.pr_items);
    const int half_threads = gridDim.x * (TB_THREADS / 2);
    const int half = blockIdx.x * (TB_THREADS / 2) + tid % (TB_THREADS / 2);
    if (tid < TB_THREADS / 2) {
        // tokens.  A page of the batch is taken from the stack directly; an old one from the block table
        for (int t = half; t < T; t += half_threads) {
            int32_t pos = 0, slot = -1;
            if (t < tokens) {
                const int r = upper_bound(end, R, t);
                const int64_t p64 = (int64_t)kv[r] + (t - (r ? end[r - 1] : 0));
                pos = (int32_t)min(p64, (int64_t)0x7fffffff);
                if (!failed[r]) {
                    const int32_t i = pos >> P.page_shift, old = pages_for(kv[r], P.page_shift);
                    int32_t page;
                    if (i < old) {
                        page = P.block_table[r * P.ld + i];
                    } else {
                        const int32_t k = (r ? pages[r - 1] : 0) + i - old;
                        page = P.free_pages[count - 1 - k];
                    }
                    if (page >= 0 && page < P.num_pages) slot = (page << P.page_shift) + (pos & ((1 << P.page_shift) - 1));
                    else atomicAdd(&P.status[STATUS_INVALID_TOKENS], 1);
                }
            }
            P.out[P.L.position + t] = pos;
            P.out[P.L.slot + t] = slot;
        }
        for (int k = half; k < taken; k += half_threads) {
            const int r = upper_bound(pages, R, k);
            const int32_t i = pages_for(kv[r], P.page_shift) + k - (r ? pages[r - 1] : 0);
            P.block_table[r * P.ld + i] = P.free_pages[count - 1 - k];
        }
    } else {
        // work lists
        for (int r = half; r < R; r += half_threads) {      // requests of single tokens: at most eight items, a thread each
            const int32_t tok0 = r ? end[r - 1] : 0;
            const int64_t rows = (int64_t)(end[r] - tok0) * P.group;
            if (rows > KV_DEC_MAX_ROWS || failed[r]) continue;
            KvItem it;
            it.req = r;
            it.tok0 = tok0;
            it.lim0 = kv[r] + 1;
            it.reserved[0] = it.reserved[1] = it.reserved[2] = 0;
            it.start = r ? chunks_d[r - 1] : 0;
            KvItem *to = dec + (r ? items_d[r - 1] : 0);
            for (it.row0 = 0; it.row0 < rows; it.row0 += P.dec_rows) {
                it.nrows = min(P.dec_rows, (int32_t)rows - it.row0);
                item_range(it.lim0, P.group, P.window, KV_DEC_CHUNK, it.row0, it.nrows, &it.k_lo, &it.n);
                *to++ = it;
                it.start += it.n + KV_DEC_OVER;
            }
        }
        for (int r = half >> 5; r < R && (n_failed > 0 || items_p[R - 1] > 0); r += half_threads >> 5) {      // the others: a warp each
            const int32_t tok0 = r ? end[r - 1] : 0, q = end[r] - tok0;
            const int64_t rows = (int64_t)q * P.group;
            if (rows == 0 || (rows <= KV_DEC_MAX_ROWS && !failed[r])) continue;
            const bool single = failed[r];
            const int32_t per = single ? P.dec_rows : KV_PROMPT_ROWS;
            const int32_t n_items = (int32_t)((rows + per - 1) / per);
            const int32_t first = single ? (r ? items_d[r - 1] : 0) : (r ? items_p[r - 1] : 0);
            int64_t before = single ? (r ? chunks_d[r - 1] : 0) : (r ? chunks_p[r - 1] : 0);
            KvItem it;
            it.req = r;
            it.tok0 = tok0;
            it.lim0 = failed[r] ? -0x40000000 : kv[r] + 1;
            it.reserved[0] = it.reserved[1] = it.reserved[2] = 0;
            for (int32_t b = 0; b < n_items; b += 32) {
                const int32_t i = b + lane;
                it.row0 = i * per;
                it.nrows = (int32_t)min((int64_t)per, rows - it.row0);
                it.n = 0;
                it.k_lo = 0;
                if (i < n_items)
                    item_range(it.lim0, P.group, P.window, single ? KV_DEC_CHUNK : KV_PROMPT_CHUNK, it.row0, it.nrows,
                               &it.k_lo, &it.n);
                const int64_t places = i < n_items ? it.n + (single ? KV_DEC_OVER : KV_PROMPT_OVER) : 0;
                const int64_t incl = warp_incl(places);
                it.start = before + incl - places;
                if (i < n_items) (single ? dec : pr)[first + i] = it;
                before += __shfl_sync(0xffffffffu, incl, 31);
            }
        }
        for (int i = half; i < spare; i += half_threads) {
            KvItem it;
            it.start = (R ? chunks_d[R - 1] : 0) + (1 + KV_DEC_OVER) * (int64_t)i;
            it.req = 0;
            it.row0 = i * P.dec_rows;
            it.nrows = (int32_t)min((int64_t)P.dec_rows, spare_rows - it.row0);
            it.k_lo = 0;
            it.n = 1;
            it.tok0 = tokens;
            it.lim0 = -0x40000000;
            it.reserved[0] = it.reserved[1] = it.reserved[2] = 0;
            dec[(R ? items_d[R - 1] : 0) + i] = it;
        }
    }
    // The first item of each walker.  A request of single tokens has at most eight items, whose places are
    // counted again; a prompt's are looked up in the list, once that is complete.
    const bool prompts = R && items_p[R - 1] > 0;
    if (prompts) {
        cluster_arrive();
        cluster_wait();
    }
    for (int w = prompts ? gt : half; w < P.dec_walkers + P.pr_walkers; w += prompts ? all_threads : half_threads) {
        if (!prompts && tid < TB_THREADS / 2) break;
        const bool single = w < P.dec_walkers;
        const int32_t i = single ? w : w - P.dec_walkers;
        const int64_t pos = i * walk_span[single ? 0 : 1];
        int32_t found = -1;
        if (pos < walk_total[single ? 0 : 1]) {
            int64_t at = pos >> 31 ? pos / P.hkv : (int64_t)((uint32_t)pos / (uint32_t)P.hkv);   // hkv * start <= pos  <=>  start <= at
            const int r = upper_bound(single ? chunks_d : chunks_p, R, at);
            const int32_t *items = single ? items_d : items_p;
            found = r ? items[r - 1] : 0;
            if (single) {
                at -= r ? chunks_d[r - 1] : 0;
                if (r == R || failed[r]) {
                    found += (int32_t)(at / (1 + KV_DEC_OVER));      // items of one empty chunk each
                } else {
                    const int32_t rows = (end[r] - (r ? end[r - 1] : 0)) * P.group;
                    for (int32_t row0 = 0;; row0 += P.dec_rows, ++found) {
                        int32_t lo, n;
                        item_range(kv[r] + 1, P.group, P.window, KV_DEC_CHUNK, row0, min(P.dec_rows, rows - row0), &lo, &n);
                        at -= n + KV_DEC_OVER;
                        if (at < 0 || row0 + P.dec_rows >= rows) break;
                    }
                }
            } else {
                int32_t hi = items[r];
                while (hi - found > 1) {   // last item that starts at or before `at`
                    const int32_t m = (found + hi) >> 1;
                    if (pr[m].start <= at) found = m; else hi = m;
                }
            }
        }
        P.out[(single ? P.L.dec_first : P.L.pr_first) + i] = found;
    }
}

// One block: the number of pages before each named request by a prefix sum, then one warp per request.
__global__ void __launch_bounds__(TB_THREADS) release_kernel(const int32_t *requests, int32_t n, int32_t R,
                                                             int32_t *kv_len, int32_t *block_table, int64_t ld,
                                                             int32_t *free_pages, int32_t *free_count,
                                                             int32_t num_pages, int32_t page_shift, int32_t *status) {
    extern __shared__ __align__(16) unsigned char tb_smem[];
    int32_t *count = reinterpret_cast<int32_t *>(tb_smem);   // [n] pages of the entry, then prefix sums
    int32_t *lens = count + n;                               // [n]
    int32_t *warp_sum = lens + n;
    unsigned char *take = reinterpret_cast<unsigned char *>(warp_sum + 32);   // [n] the entry counts
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // the first mention of a request takes it: an entry is skipped when an earlier one names the same
    for (int i = tid; i < n; i += TB_THREADS) lens[i] = requests[i];
    __syncthreads();
    for (int i = warp; i < n; i += TB_WARPS) {
        const int32_t r = lens[i];
        bool dup = false;
        for (int j = lane; j < i; j += 32) dup |= lens[j] == r;
        dup = __any_sync(0xffffffffu, dup);
        const bool ok = r >= 0 && r < R && !dup;
        int32_t pages = 0, good = 0;
        if (ok) pages = (int32_t)min((int64_t)pages_for(max(kv_len[r], 0), page_shift), ld);
        for (int j = lane; j < pages; j += 32) {
            const int32_t p = block_table[r * ld + j];
            good += p >= 0 && p < num_pages;
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) good += __shfl_xor_sync(0xffffffffu, good, d);
        if (lane == 0) {
            count[i] = good;
            take[i] = ok;
        }
    }
    __syncthreads();
    block_scan(count, n, warp_sum);
    const int32_t have = min(max(*free_count, 0), num_pages);
    __syncthreads();
    int32_t lost = 0;
    for (int i = warp; i < n; i += TB_WARPS) {
        const int32_t r = lens[i];
        if (!take[i]) continue;
        const int32_t pages = (int32_t)min((int64_t)pages_for(max(kv_len[r], 0), page_shift), ld);
        int32_t at = have + (i ? count[i - 1] : 0);
        for (int j0 = 0; j0 < pages; j0 += 32) {
            const int j = j0 + lane;
            const int32_t p = j < pages ? block_table[r * ld + j] : -1;
            const bool good = p >= 0 && p < num_pages;
            const uint32_t m = __ballot_sync(0xffffffffu, good);
            const int32_t to = at + __popc(m & ((1u << lane) - 1u));
            if (good) {
                if (to < num_pages) free_pages[to] = p; else ++lost;
            }
            if (j < pages) block_table[r * ld + j] = -1;
            at += __popc(m);
        }
        __syncwarp();
        if (lane == 0) kv_len[r] = 0;
    }
    if (lost) atomicAdd(&status[STATUS_INVALID_TOKENS], lost);
    __syncthreads();
    if (tid == 0) *free_count = (int32_t)min((int64_t)have + (n ? count[n - 1] : 0), (int64_t)num_pages);
}

// Positions of the batch's tokens on three axes.  A thread a token: its request is looked up in the starts,
// which every block brings into shared memory (three loads in a row instead of twelve), then the last of the
// request's spans that begins at or before it.  What bounds it is that chain of dependent loads: 6 us for 12936
// tokens of 32 prompts, and hardly less for 256.
constexpr int AP_THREADS = 256;
__global__ void __launch_bounds__(AP_THREADS)
axis_positions_kernel(const int32_t *start_dev, const int32_t *position, int32_t R, int32_t T, const int32_t *spans,
                      const int32_t *span_begin, int32_t num_spans, int32_t *out, int64_t ld) {
    __shared__ int32_t start[KV_MAX_REQUESTS + 1];
    const int64_t t = (int64_t)blockIdx.x * AP_THREADS + threadIdx.x;
    const int64_t p = t < T ? __ldg(position + t) : 0;
    for (int i = threadIdx.x; i <= R; i += AP_THREADS) start[i] = __ldg(start_dev + i);
    __syncthreads();
    if (t >= T) return;
    int64_t a0 = p, a1 = p, a2 = p;
    const int r = upper_bound(start + 1, R, (int32_t)t);
    if (r < R) {
        const int lo = min(max(__ldg(span_begin + r), 0), num_spans), hi = min(__ldg(span_begin + r + 1), num_spans);
        int i = lo, j = hi;                      // first span that begins behind the token
        while (i < j) {
            const int m = (i + j) >> 1;
            if (__ldg(spans + (int64_t)m * 8) > p) j = m; else i = m + 1;
        }
        if (i > lo) {
            const int4 *s = reinterpret_cast<const int4 *>(spans + (int64_t)(i - 1) * 8);
            const int4 u = __ldg(s), v = __ldg(s + 1);               // first, frames, rows, columns; base, step
            const int64_t k = p - u.x, hw = (int64_t)u.z * u.w, size = hw * u.y;
            if (k < size) {
                a0 = v.x + k / hw * v.y;
                a1 = v.x + k / u.w % u.z;
                a2 = v.x + k % u.w;
            } else {
                a0 = a1 = a2 = k - size + v.x + max(max(((int64_t)u.y - 1) * v.y + 1, (int64_t)u.z), (int64_t)u.w);
            }
        }
    }
    out[t] = (int32_t)a0;
    out[ld + t] = (int32_t)a1;
    out[2 * ld + t] = (int32_t)a2;
}

}  // namespace lora

using namespace lora;

extern "C" {

static lora_status_t tables_shape(const lora_kv_t *kv, int32_t R, int32_t T, KvTables *L) {
    if (!kv) return LORA_ERR_INVALID_ARG;
    if (R < 0 || T < 0 || R > KV_MAX_REQUESTS) return LORA_ERR_SHAPE;
    if ((int64_t)T * kv->group > 0x7ffffff0) return LORA_ERR_SHAPE;
    *L = kv_tables(R, T, kv->group, kv->dec_walkers(), kv->pr_walkers());
    return LORA_OK;
}

lora_status_t lora_kv_tables_bytes(const lora_kv_t *kv, int32_t R, int32_t T, size_t *bytes) {
    if (!bytes) return LORA_ERR_INVALID_ARG;
    KvTables L;
    lora_status_t s = tables_shape(kv, R, T, &L);
    if (s != LORA_OK) return s;
    *bytes = (size_t)L.words * 4;
    return LORA_OK;
}

lora_status_t lora_kv_build_tables(lora_kv_t *kv, const int32_t *kv_len, const int32_t *q_len, int32_t R, int32_t T,
                                   int32_t max_q, int32_t window, const int32_t *free_pages,
                                   const int32_t *free_count, int32_t *block_table, int64_t ld_table,
                                   int32_t *kv_len_out, int32_t *free_count_out, void *tables, size_t tables_bytes,
                                   void *stream) {
    TableParams P;
    if (max_q == 0 || max_q > T) max_q = T;
    lora_status_t s = tables_shape(kv, R, T, &P.L);
    if (s != LORA_OK) return s;
    if (max_q < 0 || window < 0 || ld_table < 0) return LORA_ERR_SHAPE;
    if (!tables || ((uintptr_t)tables & 15)) return LORA_ERR_INVALID_ARG;
    if (tables_bytes < (size_t)P.L.words * 4) return LORA_ERR_BUFFER_TOO_SMALL;
    if (R > 0 && (!kv_len || !q_len || !free_pages || !free_count || !block_table)) return LORA_ERR_INVALID_ARG;
    DeviceGuard g(kv->device);
    P.kv_len = kv_len;
    P.q_len = q_len;
    P.free_pages = free_pages;
    P.free_count = free_count;
    P.block_table = block_table;
    P.kv_len_out = kv_len_out;
    P.free_count_out = free_count_out;
    P.out = (int32_t *)tables;
    P.status = kv->status_dev;
    P.ld = ld_table;
    P.R = R;
    P.T = T;
    P.max_q = max_q;
    P.window = window;
    P.num_pages = kv->num_pages;
    P.page_shift = kv->page_shift;
    P.hkv = kv->hkv;
    P.group = kv->group;
    P.dec_rows = kv->dec_rows();
    P.dec_walkers = kv->dec_walkers();
    P.pr_walkers = kv->pr_walkers();
    // The limit belongs to the function, so every handle sets the same one: what the largest batch needs.
    if (!kv->tables_attr) {
        LORA_CUDA_TRY(cudaFuncSetAttribute(build_tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                           (int)tables_smem(KV_MAX_REQUESTS)));
        kv->tables_attr = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(TB_BLOCKS);
    cfg.blockDim = dim3(TB_THREADS);
    cfg.dynamicSmemBytes = tables_smem(R);
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = TB_BLOCKS;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    LORA_CUDA_TRY(cudaLaunchKernelEx(&cfg, build_tables_kernel, P));
    kv->remember(tables, R, T, max_q, window);
    return count_launch();
}

lora_status_t lora_kv_axis_positions(lora_kv_t *kv, const void *tables, int32_t R, int32_t T, const int32_t *spans,
                                     const int32_t *span_begin, int32_t num_spans, int32_t *positions,
                                     int64_t ld_positions, void *stream) {
    if (!kv) return LORA_ERR_INVALID_ARG;
    if (R < 0 || T < 0 || num_spans < 0) return LORA_ERR_SHAPE;
    if (T == 0) return LORA_OK;
    if (ld_positions < T) return LORA_ERR_SHAPE;
    if (!tables || !positions || (R > 0 && !span_begin) || (num_spans > 0 && !spans)) return LORA_ERR_INVALID_ARG;
    if ((uintptr_t)spans & 15) return LORA_ERR_INVALID_ARG;
    if (!kv->find(tables, R, T)) return LORA_ERR_INVALID_ARG;
    const KvTables L = kv_tables(R, T, kv->group, kv->dec_walkers(), kv->pr_walkers());
    const int32_t *words = (const int32_t *)tables;
    DeviceGuard g(kv->device);
    axis_positions_kernel<<<(unsigned)(((int64_t)T + AP_THREADS - 1) / AP_THREADS), AP_THREADS, 0, (cudaStream_t)stream>>>(
        words + L.start, words + L.position, R, T, spans, span_begin, num_spans, positions, ld_positions);
    return count_launch();
}

lora_status_t lora_kv_release(lora_kv_t *kv, const int32_t *requests, int32_t n, int32_t R, int32_t *kv_len,
                              int32_t *block_table, int64_t ld_table, int32_t *free_pages, int32_t *free_count,
                              void *stream) {
    if (!kv) return LORA_ERR_INVALID_ARG;
    if (n < 0 || n > KV_MAX_REQUESTS || R < 0 || ld_table < 0) return LORA_ERR_SHAPE;
    if (n == 0) return LORA_OK;
    if (!requests || !kv_len || !block_table || !free_pages || !free_count) return LORA_ERR_INVALID_ARG;
    DeviceGuard g(kv->device);
    const size_t smem = (size_t)n * 9 + 32 * 4;   // at most 37 KB
    release_kernel<<<1, TB_THREADS, smem, (cudaStream_t)stream>>>(requests, n, R, kv_len, block_table, ld_table,
                                                                  free_pages, free_count, kv->num_pages,
                                                                  kv->page_shift, kv->status_dev);
    return count_launch();
}

}  // extern "C"
