// Gradient of a lookup of coded rows with respect to the dictionaries (hclae_lookup_grad):
//   dC[m][k] = factor * sum over the t with codes[rows[t]][m] == k of g_t,
// every sum in fp32 in an order that sizes alone decide, so that equal calls give equal bits.
#pragma once
#include "decode.hpp"

namespace hclae {

struct GradArgs {
    const void *g;                                  // [T][D]
    int64_t row_stride;                             // elements
    const uint8_t *codes;                           // [V][M]
    TableRows rows;
    float factor;
    int M, K, D;
    int64_t T;
    float *dC;                                      // [M][K][D]
};

// Eight coordinates of a 16-bit row or four of an fp32 one: 16 bytes a lane, the last of a row perhaps 8.
template <typename T>
struct Piece {
    static constexpr int dims = 16 / T::bytes;
    typedef unsigned raw4 __attribute__((ext_vector_type(4), aligned(8)));      // rows begin at 8 bytes where D is no multiple of 8
    typedef unsigned raw2 __attribute__((ext_vector_type(2), aligned(8)));
    float v[dims];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < dims; ++i) v[i] = 0.f;
    }
    __device__ static __forceinline__ uint4 load(const char *p, bool whole)
    {
        if (T::bytes == 4 || whole) {
            const raw4 q = *reinterpret_cast<const raw4 *>(p);
            return make_uint4(q.x, q.y, q.z, q.w);
        }
        const raw2 q = *reinterpret_cast<const raw2 *>(p);
        return make_uint4(q.x, q.y, 0u, 0u);
    }
    __device__ __forceinline__ void add(const uint4 &q)
    {
        const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (T::bytes == 4) {
                v[i] += __uint_as_float(w[i]);
            } else if constexpr (__is_same(T, Bf16)) {
                v[2 * i] += __uint_as_float(w[i] << 16);
                v[2 * i + 1] += __uint_as_float(w[i] & 0xffff0000u);
            } else {
                typedef _Float16 h2 __attribute__((ext_vector_type(2)));
                const h2 u = __builtin_bit_cast(h2, w[i]);
                v[2 * i] += (float)u.x;
                v[2 * i + 1] += (float)u.y;
            }
        }
    }
};

// Code of row t in dictionary m, -1 where the row number names no row.
__device__ __forceinline__ int grad_code(const GradArgs &a, int64_t t, int m)
{
    const int64_t r = a.rows.at(t);
    return r >= 0 ? min((int)a.codes[r * a.M + m], a.K - 1) : -1;
}

constexpr int kGradThreads = 256;
// Rows up to which one launch finds and sums them.  M = 8, K = 256, bf16, us in one launch and sorted: D = 128, T = 2048 13 and 18, T = 4096
// 20 and 19; D = 1024, 15 and 30, 26 and 31; D = 4096, 32 and 69, 57 and 72.
constexpr int kGradFew = 4096;

// Few rows: a block per codeword of a dictionary and part of the coordinates looks at the codes of all rows, lists those that have
// its codeword, in ascending order, and sums them: `lanes` (a power of two) lanes a row, kGradThreads / lanes rows at a
// time, which are added up in ascending order at the end.  One launch in place of five; the codes are read once per codeword, from L2, which
// is what grows with the rows.  T = 509, D = 960, M = 8, K = 256 in fp32: 12 us (2048 blocks; 7.9 MB are written in 1.2 us at the rate of a
// fill), the binding and the launch half of it.
template <typename T>
__global__ __launch_bounds__(kGradThreads) void k_grad_few(const GradArgs a, int lanes, int parts)
{
    using P = Piece<T>;
    __shared__ int list[kGradFew];
    __shared__ int counts[kGradThreads / kWave];
    __shared__ float sums[kGradThreads * P::dims];
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
    const int part = blockIdx.x % parts, mk = blockIdx.x / parts;
    const int m = mk / a.K, k = mk - m * a.K;
    int found = 0;
    for (int t0 = 0; t0 < (int)a.T; t0 += kGradThreads) {
        const int t = t0 + tid;
        const bool mine = t < (int)a.T && grad_code(a, t, m) == k;
        const unsigned long long who = __ballot(mine);
        if (lane == 0) counts[wave] = __popcll(who);
        __syncthreads();
        int at = found;
        for (int w = 0; w < wave; ++w) at += counts[w];
        for (int w = 0; w < kGradThreads / kWave; ++w) found += counts[w];
        if (mine) list[at + __popcll(who & ((1ull << lane) - 1ull))] = t;
        __syncthreads();
    }
    const int groups = kGradThreads / lanes, sub = tid / lanes, col0 = tid % lanes;
    const int pieces = (a.D + P::dims - 1) / P::dims, per = (pieces + parts - 1) / parts, end = min(pieces, (part + 1) * per);
    for (int c0 = part * per; c0 < end; c0 += lanes) {
        const int c = c0 + col0;
        const bool whole = (c + 1) * P::dims <= a.D;
        P s;
        s.zero();
        if (c < end) {
            const char *g = static_cast<const char *>(a.g) + (size_t)c * 16;
#pragma unroll 4
            for (int i = sub; i < found; i += groups) s.add(P::load(g + (size_t)list[i] * a.row_stride * T::bytes, whole));
        }
#pragma unroll
        for (int i = 0; i < P::dims; ++i) sums[tid * P::dims + i] = s.v[i];
        __syncthreads();
        for (int i = tid; i < lanes * P::dims; i += kGradThreads) {
            float t = 0.f;
            for (int j = 0; j < groups; ++j) t += sums[j * lanes * P::dims + i];
            const int d = c0 * P::dims + i;
            if (d < min(end * P::dims, a.D)) a.dC[((size_t)m * a.K + k) * a.D + d] = t * a.factor;
        }
        __syncthreads();
    }
}

// Many rows: sorted by code, dictionary by dictionary (a counting sort that keeps the order of equal codes), then summed in chunks.
// T = 16384, D = 4096, M = 8, K = 256 in bf16: 162 us, of which k_grad_count 4.7, k_grad_items 6.8, k_grad_place 6.3, k_grad_sums 135,
// k_grad_join 4.6.
// Rows of a block: the fewer, the more blocks there are, and the more ranges k_grad_items goes through (T = 16384: 1024 rows a block 13 us, 256 rows 6).
__host__ __device__ constexpr int sort_range(int64_t T) { return T <= 32768 ? 256 : T <= 131072 ? 512 : T <= 524288 ? 1024 : 2048; }
// What a sorted call of T rows needs of the scratch.  Rows of one item: 128, or so many that a dictionary's rows make at most 512 items (T / 512
// is rounded up, then to whole waves).  A codeword of n rows has at most max(1, n / chunk + 1) of them, so a dictionary K + T / chunk; where a
// codeword has several, at most 2 n / chunk, and their partial sums less than 2 T / chunk + 2 rows.
constexpr int kGradItems = 512;
struct GradPlan {
    int range, ranges, chunk, max_items, max_parts;
};
__host__ __device__ constexpr GradPlan grad_plan(int64_t T, int K)
{
    GradPlan p = {};
    p.range = sort_range(T);
    p.ranges = (int)((T + p.range - 1) / p.range);
    const int64_t most = (T + kGradItems - 1) / kGradItems, waves = (most + kWave - 1) / kWave;
    p.chunk = waves < 2 ? 2 * kWave : (int)(waves * kWave);
    p.max_items = K + (int)(T / p.chunk);
    p.max_parts = 2 * (int)(T / p.chunk) + 2;
    return p;
}
// The most that any call of N rows or fewer needs: one that takes a smaller range than N rows do has at most 512 of them.
__host__ __device__ constexpr GradPlan grad_room(int64_t N, int K)
{
    const int64_t own = N / sort_range(N);
    return {0, (int)(own > 512 ? own : 512) + 1, 0, K + kGradItems, 2 * kGradItems + 2};
}
__host__ __device__ constexpr bool fits(const GradPlan &p, const GradPlan &room)
{
    return p.ranges <= room.ranges && p.max_items <= room.max_items && p.max_parts <= room.max_parts;
}
constexpr int kSortGroup = 8;                       // dictionaries of a block, a wave each
constexpr int kSortThreads = kSortGroup * kWave;

struct GradItem {                                   // up to `chunk` rows of one codeword
    int k, first, count, part;                      // part < 0: all of its rows, else the row of partial sums
};
struct GradBucket {                                 // of a codeword with several items
    int part, items;                                // first row of its partial sums, how many
};

struct SortArgs : GradPlan {
    unsigned *counts;                               // [M][ranges][K], in the end where each range's rows begin
    int *list;                                      // [M][T]
    GradItem *items;                                // [M][max_items]
    GradBucket *buckets;                            // [M][K]
    float *partial;                                 // [M][max_parts][D]
};

// Rows of each code in each range.
__global__ __launch_bounds__(kSortThreads) void k_grad_count(const GradArgs a, const SortArgs s)
{
    __shared__ unsigned hist[kSortGroup][256];
    const int wave = threadIdx.x >> 6, lane = lane_id(), m = blockIdx.y * kSortGroup + wave;
    const int64_t t0 = (int64_t)blockIdx.x * s.range;
    for (int i = lane; i < 256; i += kWave) hist[wave][i] = 0u;
    __syncthreads();
    if (m < a.M) {
#pragma unroll 4
        for (int i = 0; i < s.range; i += kWave) {
            const int64_t t = t0 + i + lane;
            const int c = t < a.T ? grad_code(a, t, m) : -1;
            if (c >= 0) atomicAdd(&hist[wave][c], 1u);
        }
    }
    __syncthreads();
    if (m < a.M)
        for (int k = lane; k < a.K; k += kWave) s.counts[((size_t)m * s.ranges + blockIdx.x) * a.K + k] = hist[wave][k];
}

// A block per dictionary, four threads per codeword, each with a quarter of the ranges: where the rows of a range and codeword begin in
// the list, and the items.  Bound by the latency of the counts, which are read twice: sixteen on their way at a time.
constexpr int kItemParts = 4, kItemAhead = 16;
__global__ __launch_bounds__(256 * kItemParts) void k_grad_items(const GradArgs a, const SortArgs s)
{
    __shared__ int3 scan[256];
    __shared__ int quarter[kItemParts][256], begin[256];
    const int m = blockIdx.x, k = threadIdx.x & 255, part = threadIdx.x >> 8;
    const int r_first = (int)((int64_t)s.ranges * part / kItemParts), r_end = (int)((int64_t)s.ranges * (part + 1) / kItemParts);
    unsigned *counts = s.counts + (size_t)m * s.ranges * a.K;
    int mine = 0;
    if (k < a.K) {
        for (int r0 = r_first; r0 < r_end; r0 += kItemAhead) {
            unsigned c[kItemAhead];
#pragma unroll
            for (int i = 0; i < kItemAhead; ++i) c[i] = r0 + i < r_end ? counts[(size_t)(r0 + i) * a.K + k] : 0u;
#pragma unroll
            for (int i = 0; i < kItemAhead; ++i) mine += (int)c[i];
        }
    }
    quarter[part][k] = mine;
    __syncthreads();
    int total = 0, items = 0, parts = 0;
    int3 sum = make_int3(0, 0, 0);
    if (part == 0) {
#pragma unroll
        for (int q = 0; q < kItemParts; ++q) total += quarter[q][k];
        items = k < a.K ? max(1, (total + s.chunk - 1) / s.chunk) : 0;
        parts = items > 1 ? items : 0;
        sum = make_int3(total, items, parts);
        scan[k] = sum;
    }
    __syncthreads();
    for (int o = 1; o < 256; o <<= 1) {
        int3 v = make_int3(0, 0, 0);
        if (part == 0 && k >= o) v = scan[k - o];
        __syncthreads();
        sum = make_int3(sum.x + v.x, sum.y + v.y, sum.z + v.z);
        if (part == 0) scan[k] = sum;
        __syncthreads();
    }
    const int all = scan[255].y;
    if (part == 0) begin[k] = sum.x - total;
    __syncthreads();
    if (k < a.K) {
        unsigned at = (unsigned)begin[k];
        for (int q = 0; q < part; ++q) at += (unsigned)quarter[q][k];
        for (int r0 = r_first; r0 < r_end; r0 += kItemAhead) {
            unsigned c[kItemAhead];
#pragma unroll
            for (int i = 0; i < kItemAhead; ++i) c[i] = r0 + i < r_end ? counts[(size_t)(r0 + i) * a.K + k] : 0u;
#pragma unroll
            for (int i = 0; i < kItemAhead; ++i)
                if (r0 + i < r_end) {
                    counts[(size_t)(r0 + i) * a.K + k] = at;
                    at += c[i];
                }
        }
        if (part == 0) {
            const int first = sum.x - total, item0 = sum.y - items, part0 = sum.z - parts;
            GradItem *out = s.items + (size_t)m * s.max_items + item0;
            for (int i = 0; i < items; ++i)
                out[i] = {k, first + i * s.chunk, min(s.chunk, total - i * s.chunk), parts ? part0 + i : -1};
            s.buckets[(size_t)m * a.K + k] = {part0, items};
        }
    }
    for (int i = all + (int)threadIdx.x; i < s.max_items; i += 256 * kItemParts) s.items[(size_t)m * s.max_items + i] = {0, 0, -1, -1};
}

// The rows' places, a wave per dictionary and range: 64 rows at a time, equal codes ranked by lane.
__global__ __launch_bounds__(kSortThreads) void k_grad_place(const GradArgs a, const SortArgs s)
{
    __shared__ unsigned next[kSortGroup][256];
    const int wave = threadIdx.x >> 6, lane = lane_id(), m = blockIdx.y * kSortGroup + wave;
    const int64_t t0 = (int64_t)blockIdx.x * s.range;
    if (m < a.M)
        for (int k = lane; k < a.K; k += kWave) next[wave][k] = s.counts[((size_t)m * s.ranges + blockIdx.x) * a.K + k];
    __syncthreads();
    if (m >= a.M) return;
    int *list = s.list + (size_t)m * a.T;
    constexpr int AHEAD = 4;                        // codes on their way at a time; a range is 256 rows at least
    for (int i0 = 0; i0 < s.range; i0 += AHEAD * kWave) {
        int codes[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int64_t t = t0 + i0 + j * kWave + lane;
            codes[j] = t < a.T ? grad_code(a, t, m) : -1;
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int c = codes[j];
            unsigned long long same = __ballot(c >= 0);
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                const unsigned long long bit = __ballot((c >> b) & 1);
                same &= (c >> b) & 1 ? bit : ~bit;
            }
            if (c >= 0) {
                const unsigned at = next[wave][c], rank = (unsigned)__popcll(same & ((1ull << lane) - 1ull));
                list[at + rank] = (int)(t0 + i0 + j * kWave + lane);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // all lanes have read before the first of equals writes
                if (rank == 0) next[wave][c] = at + (unsigned)__popcll(same);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
}

// A wave per item and slice of 128 bytes of the rows: eight rows at a time, 64 in flight, lanes of a row's place summed at the end.
// Blocks go round the eight XCDs in order, and a slice belongs to one XCD, which works through its slices one after another:
// a slice of all rows (2 MB at T = 16384) then fits the L2 from which it is read once per dictionary.
// 133 us at the sizes above, 8 TB/s of rows read once per dictionary: rows of 8192 bytes put a slice of all of them into few of the L2's channels, and three reads
// of four miss it by its counters, a wave waits for 62 % of its life, and a SIMD executes vector instructions for 73 % of the time (rows 8320 bytes apart: 118 us
// for all five kernels in place of 165; slices in other orders: 167 to 185).
template <typename T>
__global__ __launch_bounds__(kGradThreads) void k_grad_sums(const GradArgs a, const SortArgs s, int slices, int blocks)
{
    using P = Piece<T>;
    constexpr int waves = kGradThreads / kWave;
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    // blocks: how many cover all items of a slice.  Fewer than eight slices: every XCD takes part in each.
    const unsigned side = min(slices, 8), b = blockIdx.x, round = b / (side * blocks), rest = b - round * side * blocks;
    const int slice = (int)(round * side + rest % side), at = (int)(rest / side) * waves + wave;
    if (slice >= slices || at >= a.M * s.max_items) return;
    const GradItem item = s.items[at];
    if (item.count < 0) return;
    const int m = at / s.max_items;
    const int sub = lane >> 3, c = slice * 8 + (lane & 7);
    const bool live = c * P::dims < a.D, whole = (c + 1) * P::dims <= a.D;
    const char *g = static_cast<const char *>(a.g) + (size_t)c * 16;
    const int *list = s.list + (size_t)m * a.T + item.first;
    P sum;
    sum.zero();
    for (int i0 = 0; i0 < item.count; i0 += kWave) {
        const int mine = i0 + lane < item.count ? list[i0 + lane] : 0;
        uint4 q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int t = __shfl(mine, 8 * j + sub, kWave);
            q[j] = make_uint4(0u, 0u, 0u, 0u);
            if (live && i0 + 8 * j + sub < item.count) q[j] = P::load(g + (size_t)t * a.row_stride * T::bytes, whole);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum.add(q[j]);
    }
    // Over the eight rows: the halves of the wave exchange half of the values each and add, then its quarters, then the eights within; lane
    // (bits 5, 4) ends with the totals of coordinates `mine` and on
    float t[P::dims / 2];
#pragma unroll
    for (int i = 0; i < P::dims / 2; ++i) {
        const auto e = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum.v[i]), __float_as_uint(sum.v[i + P::dims / 2]), false, false);
        t[i] = __uint_as_float(e[0]) + __uint_as_float(e[1]);
    }
    float r[P::dims / 4];
#pragma unroll
    for (int i = 0; i < P::dims / 4; ++i) {
        const auto e = __builtin_amdgcn_permlane16_swap(__float_as_uint(t[i]), __float_as_uint(t[i + P::dims / 4]), false, false);
        r[i] = __uint_as_float(e[0]) + __uint_as_float(e[1]);
        r[i] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(r[i]), 0x128, 0xf, 0xf, true));    // row_ror:8
    }
    const int d = c * P::dims + (lane >> 5) * (P::dims / 2) + ((lane >> 4) & 1) * (P::dims / 4);
    if (!(lane & 8) && d < a.D) {
        float *to = (item.part < 0 ? a.dC + ((size_t)m * a.K + item.k) * a.D : s.partial + ((size_t)m * s.max_parts + item.part) * a.D) + d;
        const float f = item.part < 0 ? a.factor : 1.f;
        if constexpr (P::dims == 8) *reinterpret_cast<float2 *>(to) = make_float2(r[0] * f, r[1] * f);
        else *to = r[0] * f;
    }
}

// Codewords of several items: their partial sums in ascending order.
__global__ __launch_bounds__(kGradThreads) void k_grad_join(const GradArgs a, const SortArgs s)
{
    const GradBucket b = s.buckets[blockIdx.x];
    if (b.items < 2) return;
    const int m = blockIdx.x / a.K, d = 4 * (blockIdx.y * kGradThreads + threadIdx.x);
    if (d >= a.D) return;
    const float *from = s.partial + ((size_t)m * s.max_parts + b.part) * a.D + d;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int i = 0; i < b.items; ++i) {
        const float4 v = *reinterpret_cast<const float4 *>(from + (size_t)i * a.D);
        t = make_float4(t.x + v.x, t.y + v.y, t.z + v.z, t.w + v.w);
    }
    *reinterpret_cast<float4 *>(a.dC + (size_t)blockIdx.x * a.D + d) = make_float4(t.x * a.factor, t.y * a.factor, t.z * a.factor, t.w * a.factor);
}

}  // namespace hclae
