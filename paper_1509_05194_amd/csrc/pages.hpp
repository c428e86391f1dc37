// Pages of a cache: which are in use follows from the tables and lengths of its sequences alone, so that a fork is a copied row
// of the tables and a sequence is given up by setting its length to zero.
//   k_pages_clear, k_pages_mark   bitmaps of the pages that are named once or more, and twice or more
//   k_extend_plan, k_extend_rows  pages for new rows, in the order of the sequences, the lowest free page first
//   k_compact_plan, k_compact_tables   the last pages in use go to the first holes
//   k_extend_block, k_compact_block   all of it in one block, bitmaps in LDS, where tables and cache are small enough
//   k_pages_copy                  rows of pages
// None of it moves much memory: a call is its launches and a few chains of loads.
#pragma once
#include "decode.hpp"
#include "serve.hpp"

namespace hclae {

constexpr int kPageThreads = 256, kPlanThreads = 1024;

// Entries of a table that hold rows.
__host__ __device__ constexpr int pages_of(int64_t length, int page) { return (int)((length + page - 1) / page); }
__host__ __device__ constexpr int64_t held(int64_t length, int max_pages, int page)
{
    const int64_t most = (int64_t)max_pages * page;
    return length < 0 ? 0 : length > most ? most : length;
}
__host__ __device__ constexpr int64_t words_of(int64_t n_pages) { return (n_pages + 31) / 32; }

// What a sequence asks for.
struct Growth {
    int64_t length;                                 // rows it has
    int64_t first, add;                             // its new rows: of the batch, their number
    int64_t old_pages, new_pages;                   // before and after
    bool fits;                                      // the table has entries for them, and `lengths` holds their number
    __host__ __device__ constexpr Growth(const PageArgs &a, int b)
        : length(held(a.lengths[b], a.max_pages, a.page)), first(0), add(0), old_pages(0), new_pages(0), fits(false)
    {
        const int64_t from = a.starts[b] < 0 ? 0 : a.starts[b] > a.n ? a.n : a.starts[b], to = a.starts[b + 1] < 0 ? 0 : a.starts[b + 1] > a.n ? a.n : a.starts[b + 1];
        first = from;
        add = to > from ? to - from : 0;
        old_pages = (length + a.page - 1) / a.page;
        new_pages = (length + add + a.page - 1) / a.page;
        fits = new_pages <= a.max_pages && length + add <= 0x7fffffff;
    }
};

__global__ __launch_bounds__(kPageThreads) void k_pages_clear(unsigned *words, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * kPageThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kPageThreads) words[i] = 0u;
}

constexpr int kMarkEntries = 1024;                  // entries of one table that a block looks at at a time
__host__ __device__ constexpr int table_chunks(int max_pages) { return (int)(((int64_t)max_pages + kMarkEntries - 1) / kMarkEntries); }

// The live entries of a table from j0 on, those of one thread of `threads`: f(entry's place, page).
template <typename F>
__device__ __forceinline__ void live_entries(const PageArgs &a, int b, int64_t j0, int64_t j1, int live, int thread, int threads, F f)
{
    const int32_t *table = a.tables + (int64_t)b * a.max_pages;
    const int64_t end = j1 < live ? j1 : live;
    for (int64_t j = j0 + thread; j < end; j += 4 * threads) {
        int32_t p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = j + i * threads < end ? table[j + i * threads] : -1;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (p[i] >= 0 && p[i] < a.n_pages) f((int)(j + i * threads), p[i]);
    }
}
// shared: or null, where nobody asks which pages are named twice
__device__ __forceinline__ void mark_page(unsigned *used, unsigned *shared, int32_t p)
{
    const unsigned bit = 1u << (p & 31), old = atomicOr(&used[p >> 5], bit);
    if (shared && (old & bit)) atomicOr(&shared[p >> 5], bit);
}

__global__ __launch_bounds__(kPageThreads) void k_pages_mark(const PageArgs a, unsigned *used, unsigned *shared)
{
    const int chunks = table_chunks(a.max_pages);
    const int64_t jobs = (int64_t)a.B * chunks;
    for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
        const int b = (int)(job / chunks);
        const int64_t j0 = (job - (int64_t)b * chunks) * kMarkEntries;
        const int live = pages_of(held(a.lengths[b], a.max_pages, a.page), a.page);
        live_entries(a, b, j0, j0 + kMarkEntries, live, threadIdx.x, kPageThreads, [&](int, int32_t p) { mark_page(used, shared, p); });
    }
}

// Inclusive sum over the block; *total: that of all.  sums: 16 numbers in LDS.
template <typename N>
__device__ __forceinline__ N block_scan(N v, N *sums, N *total)
{
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    N x = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const N y = __shfl_up(x, o, kWave);
        if (lane >= o) x += y;
    }
    if (lane == kWave - 1) sums[wave] = x;
    __syncthreads();
    N before = 0, all = 0;
    const int waves = blockDim.x >> 6;
    for (int w = 0; w < waves; ++w) {
        if (w < wave) before += sums[w];
        all += sums[w];
    }
    __syncthreads();
    *total = all;
    return x + before;
}

struct ExtendScratch {
    unsigned *used, *shared, *upto, *free, *found;  // found: [0]
    unsigned room;                                  // pages that all sequences together can ask for
};

__device__ __forceinline__ bool last_page_shared(const PageArgs &a, int b, const Growth &g, const unsigned *shared, int32_t *at)
{
    if (g.add == 0 || g.length % a.page == 0) return false;
    const int32_t p = a.tables[(int64_t)b * a.max_pages + g.length / a.page];
    *at = p;
    return p >= 0 && p < a.n_pages && (shared[p >> 5] >> (p & 31) & 1u);
}

// By one block: how many pages the sequences up to each ask for, and that many free pages, the lowest first.  Whatever `starts` holds, no more than `room`
// pages are given: sums are in 64 bits, and those beyond 32 are more than there are.
__device__ __forceinline__ void extend_plan(const PageArgs &a, const ExtendScratch &s, unsigned long long *sums)
{
    typedef unsigned long long u64;
    u64 asked = 0;
    for (int64_t b0 = 0; b0 < a.B; b0 += kPlanThreads) {
        const int b = (int)(b0 + threadIdx.x);
        u64 need = 0, all;
        if (b < a.B) {
            const Growth g(a, b);
            int32_t at;
            if (g.fits) need = (u64)(g.new_pages - g.old_pages) + (last_page_shared(a, b, g, s.shared, &at) ? 1u : 0u);
        }
        const u64 upto = asked + block_scan(need, sums, &all);
        if (b < a.B) s.upto[b] = (unsigned)min(upto, (u64)0xffffffffu);
        asked += all;
    }
    u64 found = 0;
    const int64_t words = words_of(a.n_pages);
    for (int64_t w0 = 0; w0 < words && found < asked; w0 += kPlanThreads) {
        const int64_t w = w0 + threadIdx.x;
        unsigned left = 0;
        u64 all;
        if (w < words) {
            left = ~s.used[w];
            if (w == words - 1 && (a.n_pages & 31)) left &= (1u << (a.n_pages & 31)) - 1u;
        }
        const u64 here = (u64)__popc(left);
        u64 at = found + block_scan(here, sums, &all) - here;
        while (left && at < asked && at < s.room) {
            s.free[at++] = (unsigned)(w * 32 + (__ffs(left) - 1));
            left &= left - 1u;
        }
        found += all;
    }
    if (threadIdx.x == 0) *s.found = (unsigned)min(found, (u64)s.room);
}

// By one thread or wave: a sequence's rows' slots, its new entries, its length.  What is read of its table is read before anything is written.
template <int LANES>
__device__ __forceinline__ void extend_sequence(const PageArgs &a, const ExtendScratch &s, int b, int lane)
{
    const Growth g(a, b);
    int32_t at = -1;
    const bool split = last_page_shared(a, b, g, s.shared, &at);
    const unsigned need = g.fits ? (unsigned)(g.new_pages - g.old_pages) + (split ? 1u : 0u) : 0u, begin = s.upto[b] - need;
    const bool served = g.add > 0 && g.fits && (need == 0 || s.upto[b] <= *s.found);
    int32_t *table = a.tables + (int64_t)b * a.max_pages;
    const int64_t last = g.length / a.page;             // entry of the row that is next
    const int32_t copy = served && split ? (int32_t)s.free[begin] : -1;
    const int32_t tail = copy >= 0 ? copy : g.length % a.page ? at : -1;    // page of that entry, if it holds rows already
    const unsigned *fresh = s.free + begin + (copy >= 0 ? 1 : 0);
    for (int64_t i = lane; i < g.add; i += LANES) {
        int64_t slot = -1;
        if (served) {
            const int64_t pos = g.length + i, e = pos / a.page, off = pos - e * a.page;
            const int32_t p = e < g.old_pages ? tail : (int32_t)fresh[e - g.old_pages];
            if (p >= 0 && p < a.n_pages) slot = (int64_t)p * a.page + off;
        }
        a.slots[g.first + i] = slot;
    }
    if (served)
        for (int64_t e = g.old_pages + lane; e < g.new_pages; e += LANES) table[e] = (int32_t)fresh[e - g.old_pages];
    if (lane == 0) {
        if (copy >= 0) table[last] = copy;
        if (served) a.lengths[b] = (int32_t)(g.length + g.add);
        a.src[b] = copy >= 0 ? at : -1;
        a.dst[b] = copy;
        a.rows[b] = copy >= 0 ? (int32_t)(g.length % a.page) : 0;
    }
}
// Rows that are of no sequence.
__device__ __forceinline__ void extend_others(const PageArgs &a, int64_t at, int64_t step)
{
    const int64_t front = a.starts[0] < 0 ? 0 : a.starts[0] > a.n ? a.n : a.starts[0], back = a.starts[a.B] < 0 ? 0 : a.starts[a.B] > a.n ? a.n : a.starts[a.B];
    for (int64_t i = at; i < front; i += step) a.slots[i] = -1;
    for (int64_t i = back + at; i < a.n; i += step) a.slots[i] = -1;
}

__global__ __launch_bounds__(kPlanThreads) void k_extend_plan(const PageArgs a, const ExtendScratch s)
{
    __shared__ unsigned long long sums[kPlanThreads / kWave];
    extend_plan(a, s, sums);
}

__global__ __launch_bounds__(kPageThreads) void k_extend_rows(const PageArgs a, const ExtendScratch s)
{
    const int wave = threadIdx.x >> 6, waves = kPageThreads / kWave;
    for (int64_t b = (int64_t)blockIdx.x * waves + wave; b < a.B; b += (int64_t)gridDim.x * waves) extend_sequence<kWave>(a, s, (int)b, lane_id());
    extend_others(a, (int64_t)blockIdx.x * kPageThreads + threadIdx.x, (int64_t)gridDim.x * kPageThreads);
}

// All of it by one block: bitmaps, sums and the list of free pages in LDS.  64 sequences of 1000 to 2000 rows in pages of 16 take 10 us (the four kernels 15, and three
// launches more), 256 of 2000 to 4000 in pages of 64 14 us; with a wave a table in place of all entries at once 17 and 50.
constexpr int kBlockLds = 128 * 1024, kBlockEntries = 32768, kBlockRows = 16384, kFewNew = 16;
__host__ __device__ constexpr int64_t extend_lds(const PageArgs &a, int64_t room) { return 4 * (2 * words_of(a.n_pages) + 2 * (int64_t)a.B + room); }
__host__ __device__ constexpr bool extend_in_block(const PageArgs &a, int64_t room)
{
    return (int64_t)a.B * a.max_pages <= kBlockEntries && a.B <= kBlockEntries && a.n <= kBlockRows && extend_lds(a, room) <= kBlockLds;
}
// f(sequence, entry, page) for all live entries of all tables: the block's threads take them one after another, eight loads on their way at a time.
// live: how many entries of a sequence hold rows.
template <typename F>
__device__ __forceinline__ void all_entries(const PageArgs &a, const unsigned *live, F f)
{
    const unsigned total = (unsigned)(a.B * a.max_pages), mul = page_mul(max(a.max_pages, 1));
    const int shift = page_shift(max(a.max_pages, 1));
    for (unsigned i0 = threadIdx.x; i0 < total; i0 += 8 * kPlanThreads) {
        int32_t p[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) p[k] = a.tables[min(i0 + k * kPlanThreads, total - 1u)];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const unsigned i = i0 + k * kPlanThreads;
            if (i >= total || p[k] < 0 || p[k] >= a.n_pages) continue;
            const unsigned b = (unsigned)((uint64_t)i * mul >> (31 + shift)), j = i - b * (unsigned)a.max_pages;
            if (j < live[b]) f((int)b, (int)j, p[k]);
        }
    }
}
__device__ __forceinline__ void live_of(const PageArgs &a, unsigned *live)
{
    for (int b = threadIdx.x; b < a.B; b += kPlanThreads) live[b] = (unsigned)pages_of(held(a.lengths[b], a.max_pages, a.page), a.page);
}
__global__ __launch_bounds__(kPlanThreads) void k_extend_block(const PageArgs a, unsigned room)
{
    extern __shared__ unsigned page_lds[];
    __shared__ unsigned long long sums[kPlanThreads / kWave];
    __shared__ unsigned found;
    const int words = (int)words_of(a.n_pages);
    const ExtendScratch s = {page_lds, page_lds + words, page_lds + 2 * words, page_lds + 2 * words + 2 * a.B, &found, room};
    unsigned *live = page_lds + 2 * words + a.B;
    for (int i = threadIdx.x; i < 2 * words; i += kPlanThreads) page_lds[i] = 0u;
    live_of(a, live);
    __syncthreads();
    all_entries(a, live, [&](int, int, int32_t p) { mark_page(s.used, s.shared, p); });
    __syncthreads();
    extend_plan(a, s, sums);
    __syncthreads();
    // a thread a sequence with few new rows, then a wave one with many
    for (int b = threadIdx.x; b < a.B; b += kPlanThreads) {
        const bool few = a.starts[b + 1] - (int64_t)a.starts[b] <= kFewNew;
        live[b] = few ? 1u : 0u;
        if (few) extend_sequence<1>(a, s, b, 0);
    }
    __syncthreads();
    for (int b = threadIdx.x >> 6; b < a.B; b += kPlanThreads / kWave)
        if (!live[b]) extend_sequence<kWave>(a, s, b, lane_id());
    extend_others(a, threadIdx.x, kPlanThreads);
}

struct CompactScratch {
    unsigned *used, *before;                        // before: pages in use in earlier words
};

// By one block: the pages in use are counted; the i-th hole below that number takes the i-th page from that number on.
__device__ __forceinline__ void compact_plan(const PageArgs &a, const CompactScratch &s, unsigned *sums)
{
    const int64_t words = words_of(a.n_pages);
    unsigned n = 0;
    for (int64_t w0 = 0; w0 < words; w0 += kPlanThreads) {
        const int64_t w = w0 + threadIdx.x;
        const unsigned here = w < words ? (unsigned)__popc(s.used[w]) : 0u;
        unsigned all;
        const unsigned upto = n + block_scan(here, sums, &all);
        if (w < words) s.before[w] = upto - here;
        n += all;
    }
    if (threadIdx.x == 0 && a.used) *a.used = (int32_t)n;
    __syncthreads();
    // of the pages below n so many are in use: the others from n on have to move
    const int64_t wn = n >> 5;
    const unsigned low = wn < words ? s.before[wn] + (unsigned)__popc(s.used[wn] & ((1u << (n & 31)) - 1u)) : n;
    const unsigned moves = n - low;
    for (int64_t p = threadIdx.x; p < a.n_pages; p += kPlanThreads) {
        const unsigned used = s.used[p >> 5], bit = (unsigned)(p & 31), upto = s.before[p >> 5] + (unsigned)__popc(used & ((1u << bit) - 1u));    // pages in use before it
        if (used >> bit & 1u) {
            if (p >= n) a.src[upto - low] = (int32_t)p;
        } else if (p < n) a.dst[p - upto] = (int32_t)p;     // as many holes are before it
    }
    for (int64_t i = moves + threadIdx.x; i < a.n_pages / 2; i += kPlanThreads) a.src[i] = a.dst[i] = -1;
}
// Where a page from n on goes, `low` pages below n being in use; n and low as compact_plan has them.
struct NewPlaces {
    unsigned n, low;
    __device__ __forceinline__ NewPlaces(const PageArgs &a, const CompactScratch &s)
    {
        const int64_t words = words_of(a.n_pages);
        n = s.before[words - 1] + (unsigned)__popc(s.used[words - 1]);
        const int64_t wn = n >> 5;
        low = wn < words ? s.before[wn] + (unsigned)__popc(s.used[wn] & ((1u << (n & 31)) - 1u)) : n;
    }
    __device__ __forceinline__ void entry(const PageArgs &a, const CompactScratch &s, int b, int j, int32_t p) const
    {
        if (p >= (int64_t)n) a.tables[(int64_t)b * a.max_pages + j] = a.dst[s.before[p >> 5] + (unsigned)__popc(s.used[p >> 5] & ((1u << (p & 31)) - 1u)) - low];
    }
};

__global__ __launch_bounds__(kPlanThreads) void k_compact_plan(const PageArgs a, const CompactScratch s)
{
    __shared__ unsigned sums[kPlanThreads / kWave];
    compact_plan(a, s, sums);
}

__global__ __launch_bounds__(kPageThreads) void k_compact_tables(const PageArgs a, const CompactScratch s)
{
    const NewPlaces places(a, s);
    const int chunks = table_chunks(a.max_pages);
    const int64_t jobs = (int64_t)a.B * chunks;
    for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
        const int b = (int)(job / chunks);
        const int64_t j0 = (job - (int64_t)b * chunks) * kMarkEntries;
        const int live = pages_of(held(a.lengths[b], a.max_pages, a.page), a.page);
        live_entries(a, b, j0, j0 + kMarkEntries, live, threadIdx.x, kPageThreads, [&](int j, int32_t p) { places.entry(a, s, b, j, p); });
    }
}

// All of it by one block, as k_extend_block: 24600 pages and 128 tables of 128 entries 18 us, 250 pages 5 us (the four kernels 19 and 10).
__host__ __device__ constexpr bool compact_in_block(const PageArgs &a)
{
    return (int64_t)a.B * a.max_pages <= kBlockEntries && a.B <= 8192 && a.n_pages <= 65536;
}
__global__ __launch_bounds__(kPlanThreads) void k_compact_block(const PageArgs a)
{
    extern __shared__ unsigned page_lds[];
    __shared__ unsigned sums[kPlanThreads / kWave];
    const int words = (int)words_of(a.n_pages);
    const CompactScratch s = {page_lds, page_lds + words};
    unsigned *live = page_lds + 2 * words;
    for (int i = threadIdx.x; i < words; i += kPlanThreads) page_lds[i] = 0u;
    live_of(a, live);
    __syncthreads();
    all_entries(a, live, [&](int, int, int32_t p) { mark_page(s.used, nullptr, p); });
    __syncthreads();
    compact_plan(a, s, sums);
    __syncthreads();
    const NewPlaces places(a, s);
    all_entries(a, live, [&](int b, int j, int32_t p) { places.entry(a, s, b, j, p); });
}

// V: bytes of a load.  Rows of a page lie side by side in both arrays, so that the rows of a copy are two stretches of memory.
template <typename V>
__device__ __forceinline__ void copy_stretch(char *to, const char *from, int64_t bytes)
{
    const int64_t whole = bytes / (int64_t)sizeof(V);
    for (int64_t i = threadIdx.x; i < whole; i += kPageThreads) reinterpret_cast<V *>(to)[i] = reinterpret_cast<const V *>(from)[i];
    for (int64_t i = whole * (int64_t)sizeof(V) + threadIdx.x; i < bytes; i += kPageThreads) to[i] = from[i];
}

// parts: blocks a page, each a part of its rows.  5800 pages of 12 KB among 12300 entries, most of the others -1: 27 us, 5.2 TB/s read and written (a large copy: 5.0).
__global__ __launch_bounds__(kPageThreads) void k_pages_copy(const CopyArgs a, int parts)
{
    const int64_t jobs = a.n * parts;
    for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
        const int64_t i = job / parts;
        const int part = (int)(job - i * parts);
        const int32_t from = a.src[i], to = a.dst[i];
        if (from < 0 || to < 0 || from >= a.n_pages || to >= a.n_pages || from == to) continue;
        int rows = a.rows ? a.rows[i] : a.page;
        rows = rows < 0 ? 0 : rows > a.page ? a.page : rows;
        const int r0 = (int)((int64_t)rows * part / parts), r1 = (int)((int64_t)rows * (part + 1) / parts);
        if (r0 == r1) continue;
        const int64_t f = (int64_t)from * a.page + r0, t = (int64_t)to * a.page + r0;
        char *tc = reinterpret_cast<char *>(a.codes) + t * a.row_codes;
        const char *fc = reinterpret_cast<const char *>(a.codes) + f * a.row_codes;
        const int64_t bytes = (int64_t)(r1 - r0) * a.row_codes;
        const uintptr_t odd = reinterpret_cast<uintptr_t>(tc) | reinterpret_cast<uintptr_t>(fc);
        if (odd % 16 == 0) copy_stretch<uint4>(tc, fc, bytes);
        else if (odd % 4 == 0) copy_stretch<unsigned>(tc, fc, bytes);
        else copy_stretch<char>(tc, fc, bytes);
        if (a.scale) {
            char *ts = reinterpret_cast<char *>(a.scale + t * a.row_scales);
            const char *fs = reinterpret_cast<const char *>(a.scale + f * a.row_scales);
            const int64_t sb = (int64_t)(r1 - r0) * a.row_scales * 4;
            if ((reinterpret_cast<uintptr_t>(ts) | reinterpret_cast<uintptr_t>(fs)) % 16 == 0) copy_stretch<uint4>(ts, fs, sb);
            else copy_stretch<unsigned>(ts, fs, sb);
        }
    }
}

}  // namespace hclae
