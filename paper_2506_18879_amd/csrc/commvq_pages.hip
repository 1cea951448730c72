// Paged caches: block tables and slots from the requests' lengths, and stores of new records into the pages.
#include "commvq_internal.hpp"

namespace {

constexpr int kTableThreads = 1024;  // requests of a round, and new tokens of a workgroup of k_page_tables
constexpr int kStoreThreads = 256;

struct TableArgs {
    const int32_t *cached, *fresh, *free_blocks;
    int32_t *table, *seq_lens, *cu_new, *slots, *token_pos, *taken;
    int batch, n_free, n_slots, n_blocks, max_blocks, block_bits;
};

// Exclusive prefix sums of two numbers a thread over the workgroup, with the totals.
struct Sums {
    long long tokens, pages;
};
__device__ __forceinline__ Sums scan_exclusive(Sums v, Sums *waves, Sums &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Sums incl = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const long long t = __shfl_up(incl.tokens, d);
        const long long p = __shfl_up(incl.pages, d);
        if (lane >= d) { incl.tokens += t; incl.pages += p; }
    }
    if (lane == 63) waves[wave] = incl;
    __syncthreads();
    Sums before = {0, 0};
    total = Sums{0, 0};
#pragma unroll
    for (int w = 0; w < kTableThreads / 64; ++w) {
        if (w < wave) { before.tokens += waves[w].tokens; before.pages += waves[w].pages; }
        total.tokens += waves[w].tokens;
        total.pages += waves[w].pages;
    }
    __syncthreads();
    return Sums{before.tokens + incl.tokens - v.tokens, before.pages + incl.pages - v.pages};
}

// Pages, slots and offsets of new tokens.  With held_b = ceil(cached_b / P) and need_b = ceil((cached_b + new_b) / P) - held_b the
// pages of request b are entries sum_{c < b} need_c .. of the free list, and token i of its new ones has index t = cached_b + i
// and lies in page t / P of its row, from the table if t / P < held_b and from the list otherwise.  Every page that is taken begins with a new
// token, whose thread writes the table's entry: nothing is read that the launch writes, so one launch does and its workgroups need not
// wait for each other.  Every workgroup sums up the requests by itself, 1024 a round, and serves 1024 slots.
// Bound by latency: a launch, the lengths' load, two barriers, the search and the page's load; a few bytes a token.  Measured: 24 requests 6.6 us, 1000
// requests with 254 000 new tokens 7.4.
__global__ __launch_bounds__(kTableThreads) void k_page_tables(TableArgs a)
{
    __shared__ Sums waves[kTableThreads / 64];
    __shared__ int starts[kTableThreads + 1];   // first new token of the round's requests, from the workgroup's first slot; clamped
    __shared__ int firsts[kTableThreads];       // first entry of the free list, or -1: not granted
    __shared__ int lens[kTableThreads];         // cached tokens
    const int tid = threadIdx.x;
    const long long slot0 = (long long)blockIdx.x * kTableThreads;
    const int page_mask = (1 << a.block_bits) - 1;
    const bool writer = blockIdx.x == 0;        // lengths, offsets and counts
    Sums done = {0, 0};                         // of the rounds before
    long long granted_pages = 0, refused = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kTableThreads) {
        const int b = b0 + tid;
        const long long cached = b < a.batch ? max(a.cached[b], 0) : 0, fresh = b < a.batch ? max(a.fresh[b], 0) : 0;
        const long long held = (cached + page_mask) >> a.block_bits, after = (cached + fresh + page_mask) >> a.block_bits;
        const bool fits = after <= a.max_blocks && cached + fresh <= 0x7fffffff;
        Sums total;
        const Sums own = {fresh, fits ? after - held : 0};
        const Sums at = scan_exclusive(own, waves, total);
        const long long first_token = done.tokens + at.tokens;
        const long long first_page = done.pages + at.pages;
        const bool granted = fits && (own.pages == 0 || first_page + own.pages <= a.n_free) && first_token + fresh <= a.n_slots;
        const long long rel = first_token - slot0;
        starts[tid] = (int)(rel < -0x40000000ll ? -0x40000000ll : rel > 0x40000000ll ? 0x40000000ll : rel);
        firsts[tid] = granted ? (int)first_page : -1;
        lens[tid] = (int)cached;
        if (tid == 0) {
            const long long end = done.tokens + total.tokens - slot0;
            starts[kTableThreads] = (int)(end < -0x40000000ll ? -0x40000000ll : end > 0x40000000ll ? 0x40000000ll : end);
        }
        if (writer && b < a.batch) {
            a.seq_lens[b] = (int)(granted ? cached + fresh : cached);
            a.cu_new[b + 1] = (int)(first_token + fresh);
            granted_pages += granted ? own.pages : 0;
            refused += granted ? 0 : 1;
        }
        __syncthreads();
        const long long slot = slot0 + tid;
        if (slot < a.n_slots && tid >= starts[0] && tid < starts[kTableThreads]) {
            int lo = 0, hi = kTableThreads - 1;      // the last request that begins at or before the slot (empty ones share their start with the next)
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (starts[mid] <= tid) lo = mid;
                else hi = mid - 1;
            }
            // (a start before the workgroup's first slot by more than 2^30 tokens cannot be: n_slots is an int)
            const long long t = (long long)lens[lo] + tid - starts[lo];
            const int page_at = (int)(t >> a.block_bits), kept = (int)(((long long)lens[lo] + page_mask) >> a.block_bits);
            int out = -1;
            if (firsts[lo] >= 0) {
                int32_t *row = a.table + (size_t)(b0 + lo) * a.max_blocks;
                const int page = page_at < kept ? row[page_at] : a.free_blocks[firsts[lo] + page_at - kept];
                if (page_at >= kept && (t & page_mask) == 0) row[page_at] = page;
                if (page >= 0 && page < a.n_blocks) out = (page << a.block_bits) + (int)(t & page_mask);
            }
            a.slots[slot] = out;
            if (a.token_pos) a.token_pos[slot] = (int)min(t, 0x7fffffffll);
        }
        done.tokens += total.tokens;
        done.pages += total.pages;
        if (!writer && done.tokens >= slot0 + kTableThreads) return;  // (the same for the whole workgroup)
        __syncthreads();
    }
    const long long slot = slot0 + tid;
    if (slot >= done.tokens && slot < a.n_slots) a.slots[slot] = -1;
    if (!writer) return;
    Sums total;
    scan_exclusive(Sums{refused, granted_pages}, waves, total);
    if (tid == 0) {
        a.cu_new[0] = 0;
        a.taken[0] = (int)total.pages;
        a.taken[1] = (int)total.tokens;
    }
}

struct StoreArgs {
    const int32_t *slots, *token_pos;
    const uint4 *keys, *vals;
    uint4 *key_pages, *val_pages;
    int32_t *page_pos;
    int pieces;                     // 16-byte pieces of all tokens' records
    int per, key_per;               // pieces of a token (keys, then values), of its keys
    int key_shift, val_shift;       // pieces of a record of one head: 1 << shift
    int heads, block_bits, n_slots, n_axes;
    Divisor by_per;
};

// One 16-byte piece a thread: record h of token t to page slot / P, head h, row slot % P.  Bound by memory: every record is read
// once and written once, in runs of M bytes.  Measured: 90 001 tokens of 8 heads, 16 and 32 codebooks, three axes 13.8 us, 5.2 TB/s; 27 tokens 2.2.
__global__ __launch_bounds__(kStoreThreads) void k_store_pages(StoreArgs a)
{
    const long long id = (long long)blockIdx.x * kStoreThreads + threadIdx.x;
    if (id >= a.pieces) return;
    const int i = (int)id, t = quotient(i, a.by_per), x = i - t * a.per;
    const int slot = a.slots[t];
    if (slot < 0 || slot >= a.n_slots) return;
    const size_t page = (size_t)(slot >> a.block_bits);
    const int row = slot & ((1 << a.block_bits) - 1);
    const bool key = x < a.key_per;
    const int y = key ? x : x - a.key_per, shift = key ? a.key_shift : a.val_shift;
    const int h = y >> shift, piece = y & ((1 << shift) - 1);
    const size_t to = (((((page * a.heads + h) << a.block_bits) + row)) << shift) + piece;
    if (key) a.key_pages[to] = a.keys[(size_t)t * a.key_per + y];
    else a.val_pages[to] = a.vals[(size_t)t * (a.per - a.key_per) + y];
    if (a.page_pos)  // (a layer of one head has fewer pieces than a position has numbers)
        for (int k = x; k < a.n_axes; k += a.per) a.page_pos[(size_t)slot * a.n_axes + k] = a.token_pos[(size_t)t * a.n_axes + k];
}

}  // namespace

// Host-only check of a pool's geometry; shared with the attention call.
commvq_status commvq_check_pages(const commvq_pages *p)
{
    if (!p) return COMMVQ_ERR_NULL;
    if (p->block_size < 16 || p->block_size > 1024 || (p->block_size & (p->block_size - 1))) return COMMVQ_ERR_SHAPE;
    if (p->n_blocks < 1 || (int64_t)p->n_blocks * p->block_size > (int64_t)0x7fffffff) return COMMVQ_ERR_SHAPE;
    if (p->max_blocks < 1 || p->n_axes < 1 || p->n_axes > 4) return COMMVQ_ERR_SHAPE;
    return COMMVQ_OK;
}

extern "C" {

commvq_status commvq_page_tables(const commvq_pages *pages, int32_t batch, const int32_t *cached_lens, const int32_t *new_lens,
                                 const int32_t *free_blocks, int32_t n_free, int32_t *block_tables, int32_t *seq_lens,
                                 int32_t *cu_new, int32_t *slots, int32_t *token_pos, int32_t n_slots, int32_t *taken,
                                 void *stream)
{
    if (!cached_lens || !new_lens || !block_tables || !seq_lens || !cu_new || !taken) return COMMVQ_ERR_NULL;
    if ((n_free > 0 && !free_blocks) || (n_slots > 0 && !slots)) return COMMVQ_ERR_NULL;
    const commvq_status st = commvq_check_pages(pages);
    if (st != COMMVQ_OK) return st;
    if (batch < 1 || n_free < 0 || n_slots < 0 || n_slots > 1 << 30) return COMMVQ_ERR_SHAPE;
    TableArgs a{cached_lens, new_lens, free_blocks, block_tables, seq_lens, cu_new, slots, token_pos, taken,
                batch, n_free, n_slots, pages->n_blocks, pages->max_blocks, __builtin_ctz((unsigned)pages->block_size)};
    const int wgs = n_slots > 0 ? (n_slots + kTableThreads - 1) / kTableThreads : 1;
    k_page_tables<<<dim3((unsigned)wgs), kTableThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
    return hipGetLastError() == hipSuccess ? COMMVQ_OK : COMMVQ_ERR_LAUNCH;
}

commvq_status commvq_store_pages(commvq_handle *h, const commvq_pages *pages, int32_t n_tokens, const int32_t *slots,
                                 const uint8_t *key_codes, const uint8_t *val_codes, const int32_t *token_pos,
                                 uint8_t *key_pages, uint8_t *val_pages, int32_t *page_pos, void *stream)
{
    if (!h || !slots || !key_codes || !val_codes || !key_pages || !val_pages) return COMMVQ_ERR_NULL;
    if (!token_pos != !page_pos) return COMMVQ_ERR_NULL;
    const commvq_status st = commvq_check_pages(pages);
    if (st != COMMVQ_OK) return st;
    const commvq_config &c = h->cfg;
    if (c.key_format != COMMVQ_KEYS_INDEXED || c.value_format != COMMVQ_VALUES_INDEXED) return COMMVQ_ERR_CONFIG;
    if (n_tokens < 1) return COMMVQ_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(key_codes) | reinterpret_cast<uintptr_t>(val_codes) | reinterpret_cast<uintptr_t>(key_pages) |
         reinterpret_cast<uintptr_t>(val_pages)) & 15u)
        return COMMVQ_ERR_SHAPE;
    const int kp = c.m_key / 16, vp = c.m_val / 16;
    const int64_t per = (int64_t)c.n_kv_heads * (kp + vp);
    if (per * n_tokens > 0x7fffffff) return COMMVQ_ERR_SHAPE;  // (pieces are counted in 31 bits)
    if (h->device < 0) return COMMVQ_ERR_NO_DEVICE;
    StoreArgs a{slots, token_pos, reinterpret_cast<const uint4 *>(key_codes), reinterpret_cast<const uint4 *>(val_codes),
                reinterpret_cast<uint4 *>(key_pages), reinterpret_cast<uint4 *>(val_pages), page_pos, (int)(per * n_tokens), (int)per,
                c.n_kv_heads * kp, kp / 2, vp / 2, c.n_kv_heads, __builtin_ctz((unsigned)pages->block_size),
                pages->n_blocks * pages->block_size, pages->n_axes, divisor((unsigned)per)};
    const unsigned wgs = (unsigned)((per * n_tokens + kStoreThreads - 1) / kStoreThreads);
    k_store_pages<<<dim3(wgs), kStoreThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
    return hipGetLastError() == hipSuccess ? COMMVQ_OK : COMMVQ_ERR_LAUNCH;
}

}  // extern "C"
