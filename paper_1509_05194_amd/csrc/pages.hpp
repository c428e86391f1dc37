// Pages of a cache: which are in use follows from the tables and lengths of its sequences alone, so that a fork is a copied row
// of the tables and a sequence is given up by setting its length to zero.
//   k_pages_clear, k_pages_mark   bitmaps of the pages that are named once or more, and twice or more
//   k_extend_plan, k_extend_rows  pages for new rows, in the order of the sequences, the lowest free page first
//   k_compact_plan, k_compact_tables   the last pages in use go to the first holes
//   k_pages_copy                  rows of pages
#pragma once
#include "common.hpp"
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
    bool fits;                                      // the table has entries for them
    __host__ __device__ constexpr Growth(const PageArgs &a, int b)
        : length(held(a.lengths[b], a.max_pages, a.page)), first(0), add(0), old_pages(0), new_pages(0), fits(false)
    {
        const int64_t from = a.starts[b] < 0 ? 0 : a.starts[b] > a.n ? a.n : a.starts[b], to = a.starts[b + 1] < 0 ? 0 : a.starts[b + 1] > a.n ? a.n : a.starts[b + 1];
        first = from;
        add = to > from ? to - from : 0;
        old_pages = (length + a.page - 1) / a.page;
        new_pages = (length + add + a.page - 1) / a.page;
        fits = new_pages <= a.max_pages;
    }
};

__global__ __launch_bounds__(kPageThreads) void k_pages_clear(unsigned *words, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * kPageThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kPageThreads) words[i] = 0u;
}

__global__ __launch_bounds__(kPageThreads) void k_pages_mark(const PageArgs a, unsigned *used, unsigned *shared)
{
    const int64_t all = (int64_t)a.B * a.max_pages;
    for (int64_t i = (int64_t)blockIdx.x * kPageThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kPageThreads) {
        const int b = (int)(i / a.max_pages), j = (int)(i - (int64_t)b * a.max_pages);
        if (j >= pages_of(held(a.lengths[b], a.max_pages, a.page), a.page)) continue;
        const int32_t p = a.tables[i];
        if (p < 0 || p >= a.n_pages) continue;
        const unsigned bit = 1u << (p & 31), old = atomicOr(&used[p >> 5], bit);
        if (old & bit) atomicOr(&shared[p >> 5], bit);
    }
}

// Inclusive sum over the block; *total: that of all.  sums: 17 words of LDS.
__device__ __forceinline__ unsigned block_scan(unsigned v, unsigned *sums, unsigned *total)
{
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    unsigned x = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const unsigned y = __shfl_up(x, o, kWave);
        if (lane >= o) x += y;
    }
    if (lane == kWave - 1) sums[wave] = x;
    __syncthreads();
    unsigned before = 0, all = 0;
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

// One block: how many pages the sequences up to each ask for, and that many free pages, the lowest first.
__global__ __launch_bounds__(kPlanThreads) void k_extend_plan(const PageArgs a, const ExtendScratch s)
{
    __shared__ unsigned sums[17];
    unsigned asked = 0;
    for (int64_t b0 = 0; b0 < a.B; b0 += kPlanThreads) {
        const int b = (int)(b0 + threadIdx.x);
        unsigned need = 0, all;
        if (b < a.B) {
            const Growth g(a, b);
            int32_t at;
            if (g.fits) need = (unsigned)(g.new_pages - g.old_pages) + (last_page_shared(a, b, g, s.shared, &at) ? 1u : 0u);
        }
        const unsigned upto = asked + block_scan(need, sums, &all);
        if (b < a.B) s.upto[b] = upto;
        asked += all;
    }
    unsigned found = 0;
    const int64_t words = words_of(a.n_pages);
    for (int64_t w0 = 0; w0 < words && found < asked; w0 += kPlanThreads) {
        const int64_t w = w0 + threadIdx.x;
        unsigned left = 0, all;
        if (w < words) {
            left = ~s.used[w];
            if (w == words - 1 && (a.n_pages & 31)) left &= (1u << (a.n_pages & 31)) - 1u;
        }
        const unsigned here = __popc(left);
        unsigned at = found + block_scan(here, sums, &all) - here;
        while (left && at < asked && at < s.room) {
            s.free[at++] = (unsigned)(w * 32 + (__ffs(left) - 1));
            left &= left - 1u;
        }
        found += all;
    }
    if (threadIdx.x == 0) *s.found = found;
}

// A block a sequence: its new entries, its rows' slots, its length; the rows that are of no sequence.
__global__ __launch_bounds__(kPageThreads) void k_extend_rows(const PageArgs a, const ExtendScratch s)
{
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        const Growth g(a, b);
        int32_t at = -1;
        const bool split = last_page_shared(a, b, g, s.shared, &at);
        const unsigned need = g.fits ? (unsigned)(g.new_pages - g.old_pages) + (split ? 1u : 0u) : 0u, begin = s.upto[b] - need;
        const bool served = g.add > 0 && g.fits && (need == 0 || s.upto[b] <= *s.found);
        int32_t *table = a.tables + (int64_t)b * a.max_pages;
        const int64_t last = g.length / a.page;         // entry of the row that is next
        const int32_t copy = served && split ? (int32_t)s.free[begin] : -1;
        const int32_t tail = copy >= 0 ? copy : g.length % a.page ? at : -1;    // page of that entry, if it holds rows already
        const unsigned *fresh = s.free + begin + (copy >= 0 ? 1 : 0);
        for (int64_t i = threadIdx.x; i < g.add; i += kPageThreads) {
            const int64_t pos = g.length + i, e = pos / a.page, off = pos - e * a.page;
            int64_t slot = -1;
            if (served) {
                const int32_t p = e < g.old_pages ? tail : (int32_t)fresh[e - g.old_pages];
                if (p >= 0 && p < a.n_pages) slot = (int64_t)p * a.page + off;
            }
            a.slots[g.first + i] = slot;
        }
        __syncthreads();                                // the entry of the next row has been read
        if (served)
            for (int64_t e = g.old_pages + threadIdx.x; e < g.new_pages; e += kPageThreads) table[e] = (int32_t)fresh[e - g.old_pages];
        if (threadIdx.x == 0) {
            if (copy >= 0) table[last] = copy;
            if (served) a.lengths[b] = (int32_t)(g.length + g.add);
            a.src[b] = copy >= 0 ? at : -1;
            a.dst[b] = copy;
            a.rows[b] = copy >= 0 ? (int32_t)(g.length % a.page) : 0;
        }
        __syncthreads();
    }
    const int64_t front = a.starts[0] < 0 ? 0 : a.starts[0] > a.n ? a.n : a.starts[0], back = a.starts[a.B] < 0 ? 0 : a.starts[a.B] > a.n ? a.n : a.starts[a.B];
    const int64_t at = (int64_t)blockIdx.x * kPageThreads + threadIdx.x, step = (int64_t)gridDim.x * kPageThreads;
    for (int64_t i = at; i < front; i += step) a.slots[i] = -1;
    for (int64_t i = back + at; i < a.n; i += step) a.slots[i] = -1;
}

struct CompactScratch {
    unsigned *used, *unused, *before;               // before: pages in use in earlier words
};

// One block: the pages in use are counted; the i-th hole below that number takes the i-th page from that number on.
__global__ __launch_bounds__(kPlanThreads) void k_compact_plan(const PageArgs a, const CompactScratch s)
{
    __shared__ unsigned sums[17];
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
    // pages in use before page n: as many are in front of it, and the others have to move
    const int64_t wn = n >> 5;
    __syncthreads();
    const unsigned low = wn < words ? s.before[wn] + (unsigned)__popc(s.used[wn] & ((1u << (n & 31)) - 1u)) : n;
    const unsigned moves = n - low;
    for (int64_t w = threadIdx.x; w < words; w += kPlanThreads) {
        const unsigned used = s.used[w], upto = s.before[w];
        const int64_t p0 = w * 32;
        const unsigned front = p0 + 32 <= n ? ~0u : p0 >= n ? 0u : (1u << (n - p0)) - 1u;     // pages below n
        for (unsigned left = ~used & front; left; left &= left - 1u) {
            const int bit = __ffs(left) - 1;
            const int64_t hole = p0 + bit - (upto + __popc(used & ((1u << bit) - 1u)));       // holes before this one
            a.dst[hole] = (int32_t)(p0 + bit);
        }
        for (unsigned left = used & ~front; left; left &= left - 1u) {
            const int bit = __ffs(left) - 1;
            a.src[upto + __popc(used & ((1u << bit) - 1u)) - low] = (int32_t)(p0 + bit);
        }
    }
    for (int64_t i = moves + threadIdx.x; i < a.n_pages / 2; i += kPlanThreads) a.src[i] = a.dst[i] = -1;
}

__global__ __launch_bounds__(kPageThreads) void k_compact_tables(const PageArgs a, const CompactScratch s)
{
    const int64_t words = words_of(a.n_pages);
    const unsigned n = s.before[words - 1] + (unsigned)__popc(s.used[words - 1]);
    const int64_t wn = n >> 5;
    const unsigned low = wn < words ? s.before[wn] + (unsigned)__popc(s.used[wn] & ((1u << (n & 31)) - 1u)) : n;
    const int64_t all = (int64_t)a.B * a.max_pages;
    for (int64_t i = (int64_t)blockIdx.x * kPageThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kPageThreads) {
        const int b = (int)(i / a.max_pages), j = (int)(i - (int64_t)b * a.max_pages);
        if (j >= pages_of(held(a.lengths[b], a.max_pages, a.page), a.page)) continue;
        const int32_t p = a.tables[i];
        if (p < (int64_t)n || p >= a.n_pages) continue;
        a.tables[i] = a.dst[s.before[p >> 5] + (unsigned)__popc(s.used[p >> 5] & ((1u << (p & 31)) - 1u)) - low];
    }
}

// V: bytes of a load.  Rows of a page lie side by side in both arrays, so that the rows of a copy are two stretches of memory.
template <typename V>
__device__ __forceinline__ void copy_stretch(char *to, const char *from, int64_t bytes)
{
    const int64_t whole = bytes / (int64_t)sizeof(V);
    for (int64_t i = threadIdx.x; i < whole; i += kPageThreads) reinterpret_cast<V *>(to)[i] = reinterpret_cast<const V *>(from)[i];
    for (int64_t i = whole * (int64_t)sizeof(V) + threadIdx.x; i < bytes; i += kPageThreads) to[i] = from[i];
}

// parts: blocks a page, each a part of its rows.
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
