// Reading codes back: rows of a paged cache (hclae_cache_read) and rows of a table kept as codes (hclae_lookup),
//   out[row] = scale * sum_m c_m(code_m)          (fp32 in the order of the comment at each kernel, rounded once at the end).
#pragma once
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include "common.hpp"

namespace hclae {

enum RowType { kRowF32 = 0, kRowF16 = 1, kRowBf16 = 2 };

struct F32 {
    static constexpr int bytes = 4;
    __device__ static __forceinline__ float4 load(const void *p, int64_t at) { return *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at); }
    __device__ static __forceinline__ void store(void *p, int64_t at, const float4 &v) { *reinterpret_cast<float4 *>(static_cast<float *>(p) + at) = v; }
};
struct F16 {
    static constexpr int bytes = 2;
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    __device__ static __forceinline__ float4 widen(const uint2 &q)
    {
        const h4 v = __builtin_bit_cast(h4, q);
        return make_float4((float)v.x, (float)v.y, (float)v.z, (float)v.w);
    }
    __device__ static __forceinline__ float4 load(const void *p, int64_t at) { return widen(*reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p) + at)); }
    __device__ static __forceinline__ void store(void *p, int64_t at, const float4 &v)
    {
        *reinterpret_cast<h4 *>(static_cast<_Float16 *>(p) + at) = (h4){(_Float16)v.x, (_Float16)v.y, (_Float16)v.z, (_Float16)v.w};
    }
};
struct Bf16 {
    static constexpr int bytes = 2;
    typedef __bf16 b4 __attribute__((ext_vector_type(4)));
    __device__ static __forceinline__ float4 widen(const uint2 &v)
    {
        return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
    }
    __device__ static __forceinline__ float4 load(const void *p, int64_t at) { return widen(*reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p) + at)); }
    __device__ static __forceinline__ void store(void *p, int64_t at, const float4 &v)
    {
        *reinterpret_cast<b4 *>(static_cast<uint16_t *>(p) + at) = (b4){(__bf16)v.x, (__bf16)v.y, (__bf16)v.z, (__bf16)v.w};
    }
};

// Where the codes of an output row are.  at(): the row of the code array, kNoRow: the output is zero, kSkip: it is left as it is.
constexpr int64_t kNoRow = -1, kSkip = -2;

struct TableRows {                                  // hclae_lookup
    const int64_t *rows;                            // or null: row t is row t
    int64_t V;
    __host__ __device__ constexpr int64_t at(int64_t t) const
    {
        const int64_t r = rows ? rows[t] : t;
        return r >= 0 && r < V ? r : kNoRow;
    }
    // The same in two steps, a load between them that need not be waited for.
    struct Probe {
        int64_t r;
    };
    __device__ __forceinline__ Probe look(int64_t t, int64_t) const { return {rows ? rows[t] : t}; }
    __device__ __forceinline__ int64_t at(const Probe &p) const { return p.r >= 0 && p.r < V ? p.r : kNoRow; }
};

// x / page of 0 <= x < 2^31 as x mul >> 31 + shift with 2^shift the power of two from page up and mul = 2^(31 + shift) / page rounded up:
// the product is too large by less than 2^31 / 2^(31 + shift) <= 1 / page, which a quotient of whole numbers does not notice.
__host__ __device__ constexpr int page_shift(int page)
{
    int s = 0;
    while (s < 31 && 1ll << s < page) ++s;
    return s;
}
__host__ __device__ constexpr unsigned page_mul(int page) { return (unsigned)(((1ull << (31 + page_shift(page))) + page - 1) / page); }

struct CacheRows {                                  // hclae_cache_read
    const int32_t *tables, *starts;
    int B, max_pages, page;
    int64_t pages;                                  // of the cache
    unsigned mul = page_mul(page);
    int shift = page_shift(page);
    unsigned named = pages < 1ll << 31 ? (unsigned)pages : 1u << 31;    // pages that a table can name
    // The sequence of row t is the last one that starts at or before it; whatever `starts` holds, the search ends inside [0, B).
    __host__ __device__ constexpr int sequence(int64_t t) const
    {
        int lo = 0, hi = B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (starts[mid] <= t) lo = mid;
            else hi = mid;
        }
        return lo;
    }
    // Where the row's page number is: its place in `tables`, or kNoRow or kSkip; off: its slot in the page.  lo: a sequence that the row is in or behind.
    __host__ __device__ constexpr int64_t entry(int64_t t, int lo, unsigned &off) const
    {
        if (t < starts[0] || t >= starts[B]) return kSkip;
        while (lo + 1 < B && starts[lo + 1] <= t) ++lo;
        const int64_t pos = t - starts[lo];
        if (pos < 0 || pos > 0x7fffffff) return kSkip;
        const unsigned p = page_of((unsigned)pos);
        off = (unsigned)pos - p * (unsigned)page;
        return p < (unsigned)max_pages ? (int64_t)lo * max_pages + p : kNoRow;
    }
    __host__ __device__ constexpr unsigned page_of(unsigned pos) const { return (unsigned)((uint64_t)pos * mul >> (31 + shift)); }
    __host__ __device__ constexpr int64_t slot(int32_t q, unsigned off) const { return (unsigned)q < named ? (int64_t)((uint64_t)(unsigned)q * (unsigned)page + off) : kNoRow; }
    __host__ __device__ constexpr int64_t at(int64_t t) const
    {
        unsigned off = 0;
        const int64_t e = entry(t, sequence(t), off);
        return e < 0 ? e : slot(tables[e], off);
    }
    // The same in two steps, a load between them that need not be waited for; first: the row of lane 0, the others' follow it.
    // Where all of a wave's rows are of one sequence (most often in long ones) little is done per lane.
    static constexpr unsigned kSkipOff = ~0u;       // no slot of a page
    struct Probe {
        int32_t q;
        unsigned off;
    };
    __device__ __forceinline__ Probe look(int64_t t, int64_t first) const
    {
        const int lo = __builtin_amdgcn_readfirstlane(sequence(first));
        const int begin = __builtin_amdgcn_readfirstlane(starts[lo]), end = __builtin_amdgcn_readfirstlane(starts[lo + 1]);
        Probe p = {-1, 0u};
        if (first >= begin && first + (kWave - 1) < end) {
            const unsigned pos = (unsigned)(first - begin) + (unsigned)(t - first), at = page_of(pos);
            p.off = pos - at * (unsigned)page;
            if (at < (unsigned)max_pages) p.q = (tables + (int64_t)lo * max_pages)[at];
            return p;
        }
        const int64_t e = entry(t, lo, p.off);
        if (e == kSkip) p.off = kSkipOff;
        if (e >= 0) p.q = tables[e];
        return p;
    }
    __device__ __forceinline__ int64_t at(const Probe &p) const { return p.off == kSkipOff ? kSkip : slot(p.q, p.off); }
};

struct DecodeArgs {
    const uint8_t *codes;                           // [rows][H][M]
    const float *scale;                             // [rows][H] or null
    float factor;                                   // of all rows
    const float *C;                                 // [H][M][K][D]
    int H, M, K, D;
    int64_t n;                                      // output rows
    void *out;
    int64_t row_stride, head_stride;                // elements
};

constexpr int kDecodeThreads = 256;

// Codewords straight from L2: a thread per four coordinates of a row, the dictionaries in ascending order, eight gathers in
// flight.  lanes: threads per row, the power of two from d4 up to 256; blockIdx.y: the 256 pieces of a longer row.
// Bound by L2, about 12 TB/s of codewords (32768 rows of 16 heads, D = 128, M = 8: 275 us), the smallest calls by the launch.
template <typename T, typename Rows>
__global__ __launch_bounds__(kDecodeThreads) void k_decode_rows(const DecodeArgs a, const Rows rows, int lanes)
{
    const int d4 = a.D >> 2, sub = threadIdx.x / lanes, p = blockIdx.y * kDecodeThreads + threadIdx.x % lanes;
    const int per = kDecodeThreads / lanes;
    if (p >= d4) return;
    const int64_t items = a.n * a.H;
    for (int64_t item = (int64_t)blockIdx.x * per + sub; item < items; item += (int64_t)gridDim.x * per) {
        const int64_t t = a.H == 1 ? item : item / a.H;
        const int h = (int)(item - t * a.H);
        const int64_t at = rows.at(t);
        if (at == kSkip) continue;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (at >= 0) {
            const uint8_t *code = a.codes + (at * a.H + h) * a.M;
            const float *C = a.C + (size_t)h * a.M * a.K * a.D + 4 * p;
            for (int m0 = 0; m0 < a.M; m0 += 8) {
                const int left = min(8, a.M - m0);
                float4 v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = i < left ? *reinterpret_cast<const float4 *>(C + ((size_t)(m0 + i) * a.K + min((int)code[m0 + i], a.K - 1)) * a.D)
                                    : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int i = 0; i < 8; ++i) s = make_float4(s.x + v[i].x, s.y + v[i].y, s.z + v[i].z, s.w + v[i].w);
            }
            const float f = a.scale ? a.scale[at * a.H + h] * a.factor : a.factor;
            s = make_float4(s.x * f, s.y * f, s.z * f, s.w * f);
        }
        T::store(a.out, t * a.row_stride + h * a.head_stride + 4 * p, s);
    }
}

// Many rows: a block keeps one slice of coordinates of all codewords of a head in LDS and takes rows through it.
//
// A half line of 128 bytes holds, for one k, the slice of S = 32 / G coordinates of G dictionaries, those of step i being i G .. i G + G - 1;
// a line, the K of a pair of steps, one step in each half.  Eight lanes read a row, each 16 bytes at a place of its own
// within the half lines; even rows read the two steps of a pair in one order, odd rows in the other.  Whatever the codes are, sixteen lanes so meet none
// of the 64 banks twice.  The lanes of one coordinate and different dictionaries add up at the end (DPP).  G is the least that lets
// all of it fit LDS (M = 8, K = 256: two).  A wave takes 64 rows at a time: it looks for them two rounds ahead, fetches their codes one round ahead and keeps
// them in LDS of its own, so that no barriers are needed once the slice is there.  32768 rows of 16 heads,
// D = 128, M = 8, bf16 in 70 to 85 us; 16384 rows of D = 4096 in 59 to 64 us (2.2 TB/s written); a million of D = 128 in fp32 in 180 us (2.8 TB/s).
// Nothing is saturated: in these three a SIMD executes vector instructions for 53, 67 and 33 % of the time, LDS works for 30, 37 and 23 %
// (4 % of that for bank conflicts), and a wave waits for 55, 32 and 29 % of its life on memory or LDS (in the last for 56 % on its turn to issue).
// 290 to 360 vector instructions a wave for 64 rows and a slice; those that find the rows and lay their codes out are among them, again for every slice.
// Threads of a block: half as many where a row's codes take more of LDS.
__host__ __device__ constexpr int slice_threads(int G) { return G <= 2 ? 1024 : 512; }
constexpr int kSliceMaxM = 32;                      // codes of a row travel in eight registers

struct SliceLds {
    int pairs;                                      // of steps, ceil(M / G) of which a code has
    int fours;                                      // of steps
    int zero, codes, factors, total;                // byte offsets: a line of zeros, [wave][64 rows][G][fours] four offsets, [wave][64]
};
__host__ __device__ constexpr SliceLds slice_lds(int M, int K, int G)
{
    SliceLds l = {};
    l.pairs = ((M + G - 1) / G + 1) / 2;
    l.fours = (l.pairs + 1) / 2;
    l.zero = l.pairs * K * 256;
    l.codes = l.zero + 256;
    l.factors = l.codes + slice_threads(G) * G * l.fours * 8;
    l.total = l.factors + slice_threads(G) * 4;
    return l;
}
// The G of a shape, 0 where nothing fits `budget` bytes.  No wider slices than the rows are.
__host__ __device__ constexpr int slice_dictionaries(int M, int K, int D, int budget)
{
    if (M > kSliceMaxM) return 0;
    int G = 1;
    while (G < 8 && 16 / G >= D) G *= 2;
    for (; G <= 8; G *= 2)
        if (slice_lds(M, K, G).total <= budget) return G;
    return 0;
}

template <int CTRL>
__device__ __forceinline__ float4 dpp_add(const float4 &v)
{
    auto from = [](float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true)); };
    return make_float4(v.x + from(v.x), v.y + from(v.y), v.z + from(v.z), v.w + from(v.w));
}

// splits: parts of the rows; blocks with neighbouring slices of one part, which write neighbouring pieces of its rows, are on one XCD
// (blocks go round the eight XCDs in order).  words_aligned: every row's codes are whole, aligned words.  ONE: four steps a code at most, in
// one go; else (M = 8 with K to 128 or so, M = 16 to 100) several, and 120 to 340 scalar registers go to lanes of vector ones, in fp32 with G = 1 or 2 also
// 8 to 31 vector registers to memory.  32768 rows of 8 heads, D = 128, us in bf16 and fp32: M = 8, K = 64 (several, G = 1) 40 and 42, K = 256 (one, G = 2) 39 and 40;
// M = 16, K = 64 and 100 (several, G = 2) 67 to 69 and 82 to 84, K = 256 (one, G = 4) 108 and 106.
template <typename T, typename Rows, int G, bool ONE>
__global__ __launch_bounds__(slice_threads(G)) void k_decode_slices(const DecodeArgs a, const Rows rows, int slices, int splits, bool words_aligned)
{
    extern __shared__ float4 smem4[];
    char *lds = reinterpret_cast<char *>(smem4);
    constexpr int LQ = 8 / G, S = 4 * LQ;           // lanes and coordinates of a codeword's slice
    constexpr int THREADS = slice_threads(G);
    constexpr int NW = ONE ? G : kSliceMaxM / 4;    // words of a row's codes
    const SliceLds L = slice_lds(a.M, a.K, G);
    const unsigned jobs = (unsigned)(a.H * slices * splits), per_xcd = (jobs + 7) / 8, job = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per_xcd || job >= jobs) return;
    const int slice = (int)(job % (unsigned)slices), part = (int)(job / (unsigned)slices), h = part % a.H, split = part / a.H;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // this wave's rows: 64 at a time
    const int64_t rounds = (a.n + kWave - 1) / kWave, first = rounds * split / splits, last = rounds * (split + 1) / splits;
    constexpr int waves = THREADS / kWave;
    int64_t round = first + wave;                   // the same for all lanes
    const int nw = (a.M + 3) >> 2;
    typedef typename Rows::Probe Probe;
    auto look = [&](int64_t r) {
        const int64_t t = r * kWave + lane;
        return r < last && t < a.n ? rows.look(t, r * kWave) : Probe{};
    };
    auto found = [&](int64_t r, const Probe &p) { return r < last && r * kWave + lane < a.n ? rows.at(p) : kSkip; };
    const uint8_t *codes_h = a.codes + h * a.M;
    const unsigned row_codes = (unsigned)(a.H * a.M);
    unsigned code[NW] = {};                         // of a row that is not there: any, as they are held below K and its sum is not kept
    float factor;
    auto fetch = [&](int64_t at) {
        factor = a.factor;
        if (at < 0) return;
        const uint8_t *p = codes_h + (uint64_t)at * row_codes;
        if (words_aligned) {
#pragma unroll
            for (int j = 0; j < NW; ++j) code[j] = reinterpret_cast<const unsigned *>(p)[min(j, nw - 1)];
        } else {
#pragma unroll
            for (int j = 0; j < NW; ++j) {
                unsigned b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) b[i] = p[min(4 * j + i, a.M - 1)];
                code[j] = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
            }
        }
        if (a.scale) factor = (a.scale + h)[(uint64_t)at * (unsigned)a.H] * a.factor;
    };
    int64_t at = found(round, look(round));
    Probe probe = look(round + waves);
    fetch(at);

    // the slice
    {
        const float *C = a.C + (size_t)h * a.M * a.K * a.D;
        const int total = (L.pairs * a.K + 1) * 16, pos = threadIdx.x & 7, odd = (threadIdx.x >> 3) & 1, g = pos / LQ, d = slice * S + 4 * (pos % LQ);
        for (int i0 = threadIdx.x; i0 < total; i0 += 8 * THREADS) {
            float4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int line = (i0 + u * THREADS) >> 4, i = line / a.K, k = line - i * a.K, m = (2 * i + odd) * G + g;
                v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (m < a.M && i < L.pairs && d < a.D) v[u] = *reinterpret_cast<const float4 *>(C + ((size_t)m * a.K + k) * a.D + d);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i0 + u * THREADS < total) smem4[i0 + u * THREADS] = v[u];
        }
    }
    __syncthreads();

    // a lane's place: the lanes 4..7 of a row run backwards, so that the half mirror adds equal coordinates
    const int l8 = lane & 7, lm = G > 1 && l8 >= 4 ? 7 - l8 : l8;
    const int q = lm % LQ, g = lm / LQ + (G > 1 && l8 >= 4 ? G / 2 : 0);
    const int my = (g * LQ + q) * 16 + (lane & 8) * 16, other = my ^ 128;      // in a line's half of the row's first and second step
    const int d = slice * S + 4 * q, fours = ONE ? 1 : L.fours, row_fours = G * fours;
    uint2 *offs = reinterpret_cast<uint2 *>(lds + L.codes) + wave * kWave * row_fours;
    float *factors = reinterpret_cast<float *>(lds + L.factors) + wave * kWave;
    const bool writes = d < a.D && (G == 1 || (l8 < 4 && l8 < LQ));
    auto off_of = [&](int m) {                      // of a codeword within its lines
        const unsigned c = (code[min(m >> 2, NW - 1)] >> (8 * (m & 3))) & 255u;
        return m < a.M ? min(c, (unsigned)a.K - 1u) * 256u : 0u;
    };
    // four steps, those beyond the last pair being zeros
    auto four = [&](const uint2 &c, int w, float4 (&v)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int pair = 2 * w + (i >> 1), base = (i & 1 ? other : my) + (pair < L.pairs ? pair * a.K * 256 : L.zero);
            const unsigned both = i < 2 ? c.x : c.y, off = i & 1 ? both >> 16 : both & 0xffffu;
            v[i] = *reinterpret_cast<const float4 *>(lds + (base + off));
        }
    };
    auto plus = [](const float4 &x, const float4 &y) { return make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w); };
    for (; round < last; round += waves) {
        // offsets and factors of these rows into LDS
#pragma unroll
        for (int w = 0; w < (ONE ? 1 : kSliceMaxM / 4); ++w)
            if (ONE || w < fours) {
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    const unsigned o0 = off_of(4 * w * G + i), o1 = off_of((4 * w + 1) * G + i), o2 = off_of((4 * w + 2) * G + i), o3 = off_of((4 * w + 3) * G + i);
                    offs[(lane * G + i) * fours + w] = lane & 1 ? make_uint2(o1 | o0 << 16, o3 | o2 << 16) : make_uint2(o0 | o1 << 16, o2 | o3 << 16);
                }
            }
        factors[lane] = factor;
        const unsigned long long kept = __ballot(at != kSkip), there = __ballot(at >= 0);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int64_t next = found(round + waves, probe);
        fetch(next);
        probe = look(round + 2 * waves);
        char *to = static_cast<char *>(a.out) + ((round * kWave + (lane >> 3)) * a.row_stride + h * a.head_stride + d) * T::bytes;
        const int64_t step = 8 * a.row_stride * T::bytes;
        const float *factor8 = factors + (lane >> 3);
        const uint2 *off8 = offs + (lane >> 3) * row_fours + g * fours;
        constexpr int U = 4;                        // rows in flight (two: 10 % slower)
#pragma unroll
        for (int j0 = 0; j0 < 8; j0 += U) {
            float f[U];
            uint2 c[U];
            float4 v[U][4], s[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                c[u] = off8[8 * (j0 + u) * row_fours];
                f[u] = factor8[8 * (j0 + u)];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) four(c[u], 0, v[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) s[u] = plus(plus(v[u][0], v[u][1]), plus(v[u][2], v[u][3]));
            if (!ONE)
                for (int w = 1; w < fours; ++w) {
#pragma unroll
                    for (int u = 0; u < U; ++u) four(off8[8 * (j0 + u) * row_fours + w], w, v[u]);
#pragma unroll
                    for (int u = 0; u < U; ++u) s[u] = plus(s[u], plus(plus(v[u][0], v[u][1]), plus(v[u][2], v[u][3])));
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (G == 8) s[u] = dpp_add<0xB1>(s[u]);     // quad_perm 1 0 3 2
                if (G >= 4) s[u] = dpp_add<0x4E>(s[u]);     // quad_perm 2 3 0 1
                if (G >= 2) s[u] = dpp_add<0x141>(s[u]);    // row_half_mirror
                s[u] = make_float4(s[u].x * f[u], s[u].y * f[u], s[u].z * f[u], s[u].w * f[u]);
            }
            if (there == ~0ull) {
                if (writes)
#pragma unroll
                    for (int u = 0; u < U; ++u) T::store(to + (j0 + u) * step, 0, s[u]);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int bit = 8 * (j0 + u) + (lane >> 3);     // rows that are not there are zero, whatever codeword 0 is
                    if (writes && (kept >> bit & 1ull)) T::store(to + (j0 + u) * step, 0, there >> bit & 1ull ? s[u] : make_float4(0.f, 0.f, 0.f, 0.f));
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        at = next;
    }
}

}  // namespace hclae
