// Attention of one new token of every sequence over its rows of a coded cache (hclae_cache_attend).
//   s_t = factor g_t q . (sum_m C[h][m][k_m(t)]),  p = softmax(s),  out = sum_t p_t g'_t sum_m C[G + h][m][v_m(t)]
// Scores are kept times log2(e) and exponentials taken to the base 2; softmax statistics, weights and sums are in 32 bits or more.
//   k_attend_rows, k_attend_join   rows decoded as they are needed: any shape, and few rows
//   k_attend_tables, k_attend_codes, k_attend_fold, k_attend_out   many rows, never decoded: q . C[h][m][k] is tabulated once for all codewords, a row's score is
//       the sum of M entries; the weights of the rows are summed by the codes of their values, and these sums meet the codewords at the end.
//       A row costs M reads and M adds a query head in place of M D, whatever D is, and is read as 2 (M + 4) bytes a head: 64 sequences of 8192 to 16384 rows,
//       8 key heads of 4 query heads, D = 128, M = 8, take 149 us of kernels, with rows decoded 5.7 ms.
#pragma once
#include <type_traits>

#include "decode.hpp"
#include "serve.hpp"

namespace hclae {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// The reference of scores before there is one: finite, so that a score of -infinity weighs exp(-infinity) = 0 whichever rows it shares a tile or a part with.
constexpr float kLowest = -3.402823466e38f;

// The rows of a sequence that take part, numbered from 0: those from `begin` to `end`, or those of the picked pages among them.
struct SeqRows {
    const int32_t *table, *picks;
    int max_pages;
    unsigned page, mul;
    int shift;
    unsigned named;                                 // pages that a table can name
    int64_t begin, end;
    int64_t count;                                  // numbers there are; of a number whose row takes no part slot() is kNoRow
    __host__ __device__ constexpr SeqRows(const AttendArgs &a, int b, int h)
        : table(a.rows.tables + (int64_t)b * a.rows.max_pages), picks(a.picked ? a.picked + ((int64_t)b * a.G + h) * a.n_picked : nullptr), max_pages(a.rows.max_pages),
          page((unsigned)a.rows.page), mul(page_mul(a.rows.page)), shift(page_shift(a.rows.page)), named(a.rows.pages < 1ll << 31 ? (unsigned)a.rows.pages : 1u << 31),
          begin(a.begins ? a.begins[b] : 0), end(a.rows.lengths[b]), count(0)
    {
        const int64_t most = (int64_t)max_pages * page;
        if (end > most) end = most;
        if (begin < 0) begin = 0;
        if (end > begin) count = picks ? (int64_t)a.n_picked * page : end - begin;
    }
    __host__ __device__ constexpr unsigned page_of(unsigned x) const { return (unsigned)((uint64_t)x * mul >> (31 + shift)); }
    // i in [0, count): the page and where in it, the page ~0u where the row takes no part
    __host__ __device__ constexpr unsigned where(unsigned i, unsigned &off) const
    {
        const bool power = page == 1u << shift;
        unsigned j = 0;
        if (picks) {
            const unsigned e = power ? i >> shift : page_of(i);
            off = power ? i & (page - 1u) : i - e * page;
            const int32_t at = picks[e];
            if (at < 0 || at >= max_pages) return ~0u;
            const int64_t t = (int64_t)at * page + off;
            if (t < begin || t >= end) return ~0u;
            j = (unsigned)at;
        } else {
            const unsigned t = (unsigned)begin + i;
            j = power ? t >> shift : page_of(t);
            off = power ? t & (page - 1u) : t - j * page;
        }
        const unsigned q = (unsigned)table[j];
        return q < named ? q : ~0u;
    }
    // The same for 64 rows from i on, a multiple of 64, in pages of multiples of 64 rows and with `begin` one too: they are in one page, from `off` on;
    // t: the place of the first in its sequence.  Whether a row is between begin and end is the caller's to look at.
    __host__ __device__ constexpr unsigned where_wave(unsigned i, unsigned &off, int64_t &t) const
    {
        unsigned j = 0;
        if (picks) {
            const unsigned e = page_of(i);
            off = i - e * page;
            const int32_t at = picks[e];
            if (at < 0 || at >= max_pages) return ~0u;
            j = (unsigned)at;
        } else {
            const unsigned at = (unsigned)begin + i;
            j = page_of(at);
            off = at - j * page;
        }
        t = (int64_t)j * page + off;
        const unsigned q = (unsigned)table[j];
        return q < named ? q : ~0u;
    }
    __host__ __device__ constexpr int64_t slot(unsigned i) const
    {
        unsigned off = 0;
        const unsigned q = where(i, off);
        return q != ~0u ? (int64_t)((uint64_t)q * page + off) : kNoRow;
    }
};

// Numbers of rows at most, over all sequences; lengths are below 2^31.
__host__ __device__ constexpr int64_t attend_capacity(const AttendArgs &a)
{
    const int64_t rows = (int64_t)(a.picked ? a.n_picked : a.rows.max_pages) * a.rows.page;
    return rows < 1ll << 31 ? rows : 1ll << 31;
}

constexpr int kDirectThreads = 256, kDirectSplits = 256, kDirectRows = 2, kDirectGroups = 32;

// Threads that share a row, a power of two; rows that a block decodes at once, in groups of those threads.
__host__ __device__ constexpr int direct_lanes(int D)
{
    int lanes = 1;
    while (lanes < D / 4) lanes *= 2;
    return lanes;
}
__host__ __device__ constexpr int direct_groups(int D) { return kDirectThreads / direct_lanes(D) < kDirectGroups ? kDirectThreads / direct_lanes(D) : kDirectGroups; }
__host__ __device__ constexpr int direct_tile(int D) { return direct_groups(D) * kDirectRows; }

// Query heads a block takes at once.
__host__ __device__ constexpr int heads_at_once(int R) { return R >= 3 ? 4 : R; }

// Parts of the rows of a sequence and head: four blocks a CU where there are rows enough.
__host__ __device__ constexpr int direct_splits(const AttendArgs &a, int cus)
{
    const int RB = heads_at_once(a.R);
    const int64_t jobs = (int64_t)a.rows.B * a.G * ((a.R + RB - 1) / RB), tiles = (attend_capacity(a) + direct_tile(a.D) - 1) / direct_tile(a.D);
    int64_t s = (4ll * cus + jobs - 1) / jobs;
    if (s > tiles) s = tiles;
    if (s > kDirectSplits) s = kDirectSplits;
    return (int)(s < 1 ? 1 : s);
}

// stats of a part and query head: the largest score and the sum of exponentials below it (negative: no rows, and no sums).
struct PartStat {
    float top, sum;
};

// Four coordinates of a row.
__device__ __forceinline__ float4 decode_piece(const float *C, const uint8_t *code, int M, int K, int D)
{
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int m0 = 0; m0 < M; m0 += 8) {
        const int left = min(8, M - m0);
        float4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = i < left ? *reinterpret_cast<const float4 *>(C + ((size_t)(m0 + i) * K + min((int)code[m0 + i], K - 1)) * D) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = make_float4(s.x + v[i].x, s.y + v[i].y, s.z + v[i].z, s.w + v[i].w);
    }
    return s;
}

// A block a part of the rows of one key head and RB of its query heads, in tiles of two rows a group of threads.  Keys and values are gathered
// at the same time: a tile costs one chain of loads (table, codes, codewords), which is what few rows are bound by.  One sequence of 150 rows, 8 key heads of 4
// query heads, D = 128, M = 8: 14 us in 80 blocks, and 4.7 us to join their parts (tiles of 32 rows, keys and values one after the other: 22 and 4.1).
template <typename T, int RB>
__global__ __launch_bounds__(kDirectThreads) void k_attend_rows(const AttendArgs a, int splits, PartStat *stats, float *sums)
{
    constexpr int MOST = kDirectGroups * kDirectRows;
    __shared__ float4 q[RB][64], red[RB][kDirectThreads];
    __shared__ float s[RB][MOST], w[RB][MOST], fade[RB], gv[MOST];
    __shared__ int64_t slots[MOST];
    const int RG = (a.R + RB - 1) / RB, d4 = a.D >> 2, H = 2 * a.G, lanes = direct_lanes(a.D), groups = direct_groups(a.D), tile = direct_tile(a.D);
    const int job = blockIdx.x, head = job / splits;
    const int split = job - head * splits, rg = head % RG, h = head / RG % a.G, b = head / RG / a.G;
    const SeqRows rows(a, b, h);
    const int64_t per = ((rows.count + splits - 1) / splits + tile - 1) / tile * tile, first = per * split, last = min(rows.count, first + per);
    const int lane = lane_id(), wave = threadIdx.x >> 6, g = threadIdx.x / lanes, p = threadIdx.x % lanes;
    if (first >= last) {
        if (threadIdx.x < RB) stats[(int64_t)job * RB + threadIdx.x] = {kLowest, -1.f};
        return;
    }
    for (int i = threadIdx.x; i < RB * d4; i += kDirectThreads) {
        const int r = i / d4, e = i - r * d4, hq = rg * RB + r;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (hq < a.R) v = T::load(a.Q, (int64_t)b * a.q_row + (int64_t)(h * a.R + hq) * a.q_head + 4 * e);
        const float f = a.factor * kLog2e;
        q[r][e] = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
    }
    const float *Ck = a.C + (size_t)h * a.M * a.K * a.D + 4 * p, *Cv = a.C + (size_t)(a.G + h) * a.M * a.K * a.D + 4 * p;
    float4 acc[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) acc[r] = make_float4(0.f, 0.f, 0.f, 0.f);
    float top = kLowest, sum = 0.f;                 // of head `wave`, in every lane of its wave
    for (int64_t t0 = first; t0 < last; t0 += tile) {
        if (threadIdx.x < (unsigned)tile) {
            slots[threadIdx.x] = t0 + threadIdx.x < last ? rows.slot((unsigned)(t0 + threadIdx.x)) : kNoRow;
        }
        __syncthreads();
        float4 v[kDirectRows];
        if (g < groups)
#pragma unroll
            for (int u = 0; u < kDirectRows; ++u) {
                const int i = g + u * groups;
                const int64_t at = slots[i];
                float4 k = make_float4(0.f, 0.f, 0.f, 0.f);
                float g_key = 1.f, g_value = 1.f;
                v[u] = k;
                if (at >= 0 && a.scale) {
                    g_key = a.scale[at * H + h];
                    g_value = a.scale[at * H + a.G + h];
                }
                if (at >= 0 && p < d4) {
                    const uint8_t *code = a.codes + at * H * a.M;
                    k = decode_piece(Ck, code + h * a.M, a.M, a.K, a.D);
                    v[u] = decode_piece(Cv, code + (a.G + h) * a.M, a.M, a.K, a.D);
                }
                float dot[RB];
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const float4 x = p < d4 ? q[r][p] : make_float4(0.f, 0.f, 0.f, 0.f);
                    dot[r] = k.x * x.x + k.y * x.y + k.z * x.z + k.w * x.w;
                }
                for (int o = lanes >> 1; o > 0; o >>= 1)
#pragma unroll
                    for (int r = 0; r < RB; ++r) dot[r] += __shfl_xor(dot[r], o, kWave);
                if (p == 0) {
                    gv[i] = g_value;
#pragma unroll
                    for (int r = 0; r < RB; ++r) s[r][i] = dot[r] * g_key;
                }
            }
        __syncthreads();
        if (wave < RB) {
            const bool there = lane < tile && slots[lane] >= 0;
            const float x = there ? s[wave][lane] : -INFINITY;
            float m = x;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
            const float now = fmaxf(top, m);
            float e = there ? exp2f(x - now) : 0.f;
            w[wave][lane] = there ? e * gv[lane] : 0.f;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) e += __shfl_xor(e, o, kWave);
            const float f = exp2f(top - now);
            sum = sum * f + e;
            top = now;
            if (lane == 0) fade[wave] = f;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const float f = fade[r];
            acc[r] = make_float4(acc[r].x * f, acc[r].y * f, acc[r].z * f, acc[r].w * f);
        }
        if (g < groups)
#pragma unroll
            for (int u = 0; u < kDirectRows; ++u) {
                const int i = g + u * groups;
                if (slots[i] < 0) continue;
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const float f = w[r][i];
                    acc[r] = make_float4(acc[r].x + f * v[u].x, acc[r].y + f * v[u].y, acc[r].z + f * v[u].z, acc[r].w + f * v[u].w);
                }
            }
        __syncthreads();
    }
    if (wave < RB && lane == 0) stats[(int64_t)job * RB + wave] = {top, sum};
#pragma unroll
    for (int r = 0; r < RB; ++r) red[r][threadIdx.x] = acc[r];
    __syncthreads();
    for (int i = threadIdx.x; i < RB * d4; i += kDirectThreads) {
        const int r = i / d4, e = i - r * d4;
        float4 v = red[r][e];
        for (int j = 1; j < groups; ++j) {
            const float4 o = red[r][j * lanes + e];
            v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
        }
        reinterpret_cast<float4 *>(sums)[((int64_t)job * RB + r) * d4 + e] = v;
    }
}

// A block a query head: its parts joined.
template <typename T, int RB>
__global__ __launch_bounds__(kWave) void k_attend_join(const AttendArgs a, int splits, const PartStat *stats, const float *sums)
{
    const int RG = (a.R + RB - 1) / RB, d4 = a.D >> 2, Hq = a.G * a.R;
    const int b = blockIdx.x / Hq, hq = blockIdx.x - b * Hq, h = hq / a.R, r = hq - h * a.R;
    const int64_t job = (((int64_t)b * a.G + h) * RG + r / RB) * splits;
    const PartStat *stat = stats + job * RB + r % RB;
    float top = kLowest;
    for (int i = 0; i < splits; ++i) top = fmaxf(top, stat[(int64_t)i * RB].top);
    float sum = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    const int p = threadIdx.x;
    bool any = false;
    for (int i0 = 0; i0 < splits; i0 += 8) {
        float4 o[8];
        PartStat st[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = min(i0 + j, splits - 1);
            st[j] = stat[(int64_t)i * RB];
            o[j] = reinterpret_cast<const float4 *>(sums)[((job + i) * RB + r % RB) * d4 + min(p, d4 - 1)];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (i0 + j >= splits || st[j].sum < 0.f) continue;
            any = true;
            const float f = exp2f(st[j].top - top);
            sum += f * st[j].sum;
            v = make_float4(v.x + f * o[j].x, v.y + f * o[j].y, v.z + f * o[j].z, v.w + f * o[j].w);
        }
    }
    if (any) {
        const float f = sum == 0.f ? 0.f : 1.f / sum;       // no row weighs anything
        v = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
    }
    if (p < d4) T::store(a.out, (int64_t)b * a.o_row + (int64_t)hq * a.o_head + 4 * p, v);
    if (p == 0 && a.lse) a.lse[(int64_t)b * Hq + hq] = any ? (top + log2f(sum)) * kLn2 : -INFINITY;
}

// ---- from tables --------------------------------------------------------------------------------

constexpr int kWindow = 2048;                       // rows between two flushes of the fixed-point sums
constexpr int kCodesMaxM = 32, kCodesSplits = 64;
constexpr int kCodesLds = 152 * 1024;               // tables and sums; the rest is for what the kernel declares

// Weights are summed in fixed point, by integer atomics on LDS, so that their order changes nothing.  wide: 64 bits a query head, else two query heads in
// 64 bits, 32 each.  Clocks of a CU for 64 additions at random words, measured with sixteen waves: u64 14.5 (4 of them for the additions, the rest because three or
// four lanes meet at a bank), u32 10.0, f64 26.6, f32 194; for 64 reads at random places 7.0 of 4 or 8 bytes and 12.7 of 16.
struct CodesPlan {
    int RB;                                         // query heads of a block; 0: the shape is not for tables
    bool wide;
    int words;                                      // of 64 bits
    int lds;
};
// Where in LDS the tables lie behind that many words of sums: they are filled sixteen bytes at a time.
__host__ __device__ constexpr int codes_lut(int words) { return (words + 1) / 2 * 16; }
__host__ __device__ constexpr CodesPlan codes_plan(int R, int M, int K, bool wide)
{
    if (M > kCodesMaxM) return {0, false, 0, 0};
    for (int RB = heads_at_once(R); RB >= 1; RB /= 2) {
        const bool w = wide || RB == 1;
        const int words = M * K * (w ? RB : RB / 2), lds = codes_lut(words) + M * K * RB * 4;
        if (lds <= kCodesLds) return {RB, w, words, lds};
    }
    return {0, false, 0, 0};
}
// Words of LDS at most for code rows of up to MW words; threads of a block, two blocks a CU where their LDS fits; words a thread looks after.
__host__ __device__ constexpr int codes_most(int RB, bool wide, int MW)
{
    const int all = MW * 4 * 256 * (wide ? RB : RB / 2), most = kCodesLds / (wide ? 12 : 16);
    return all < most ? all : most;
}
__host__ __device__ constexpr int codes_threads(int RB, bool wide, int MW) { return codes_most(RB, wide, MW) * (wide ? 12 : 16) <= 72 * 1024 ? 512 : 1024; }
// Steps of the fixed-point weights: 2^codes_bits of them at most are what the rows that a wave takes of a window (four a lane, or two) weigh together when the step is chosen,
// 7/4 of that before it is chosen anew: in 32 bits the rows of a window, all with one code, stay below 7/8 2^31 (and a step each for the rounding).
__host__ __device__ constexpr int codes_bits(int RB, bool wide, int MW) { return wide ? 48 : codes_threads(RB, wide, MW) == 512 ? 27 : 26; }
__host__ __device__ constexpr int codes_words(int RB, bool wide, int MW) { return (codes_most(RB, wide, MW) + codes_threads(RB, wide, MW) - 1) / codes_threads(RB, wide, MW); }
// Parts of a sequence's rows: as many blocks as the CUs hold at once, `blocks` each, with 2048 rows each at least, or 512 while there are fewer blocks than CUs.
__host__ __device__ constexpr int codes_splits(const AttendArgs &a, int RB, int blocks, int cus)
{
    const int64_t jobs = (int64_t)a.rows.B * a.G * ((a.R + RB - 1) / RB), rows = attend_capacity(a);
    int64_t s = (blocks * (int64_t)cus + jobs - 1) / jobs, most = (rows + 2047) / 2048;
    if (jobs * most < cus) {
        const int64_t more = (rows + 511) / 512, fill = (cus + jobs - 1) / jobs;
        most = more < fill ? more : fill;
    }
    if (s > most) s = most;
    if (s > kCodesSplits) s = kCodesSplits;
    return (int)(s < 1 ? 1 : s);
}
// Rows of sums, and of tables of RB query heads: whole fours.
__host__ __device__ constexpr int64_t sums_row(int M, int K) { return ((int64_t)M * K + 3) / 4 * 4; }
__host__ __device__ constexpr int64_t tab_row(int M, int K, int RB) { return ((int64_t)M * K * RB + 3) / 4 * 4; }

typedef float floatx4 __attribute__((ext_vector_type(4)));

// Products of floats on the bf16 matrix cores: a float is the sum of three bf16 numbers, rounded one after the other, up to 2^-27 of it;
// a bf16 number is one and a half number two.  Of the products of parts those beyond 2^-24 of the whole are left out: six for two floats, 96 cycles for
// 16 x 16 x 32 where the fp32 matrix cores take 256.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
template <int N>
__device__ __forceinline__ void split_floats(const float (&x)[8], bf16x8 (&part)[N])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float left = x[e];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            part[i][e] = (__bf16)left;
            if (i + 1 < N) left -= (float)part[i][e];
        }
    }
}
// s += a b, the small products first; NA parts of a and NB of b.
template <int NA, int NB>
__device__ __forceinline__ void mfma_parts(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], floatx4 &s)
{
    constexpr int last = (NA > NB ? NA : NB) - 1;
#pragma unroll
    for (int order = last; order >= 0; --order)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (order - i >= 0 && order - i < NB) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[order - i], s, 0, 0, 0);
}

constexpr int kTableThreads = 256;
// Queries that a block keeps in LDS at a time, for rows of 32 NJ coordinates in N parts.
__host__ __device__ constexpr int table_queries(int N, int NJ) { return N * NJ <= 4 ? 64 : N * NJ <= 12 ? 32 : 16; }

// tab[b][h][rg][codeword][RB] = factor log2(e) q . c.  A wave keeps 16 codewords in registers and takes tiles of 16 queries past them; queries of a head are numbered
// (b, rg, r).  Of a product's 32 coordinates a lane holds 8 side by side, 8 g .. 8 g + 7 of them in the wave's quarter g, for both operands alike.  Neighbouring
// lanes hold different rows, which the memory pipe takes one by one: the queries come through LDS.  N: parts of a query.  2048 query heads, 8 key heads, D = 128, M = 8,
// K = 256 (17 MB of tables, 1.1 G products): 13 us, with the fp32 matrix cores 20, with queries read by every wave 29; the least a call takes is 4 to 5.
template <typename T, int RB, int NJ, int N>
__global__ __launch_bounds__(kTableThreads) void k_attend_tables(const AttendArgs a, int stages, float *tab)
{
    constexpr int PITCH = 32 * NJ + 8, TQ = table_queries(N, NJ);
    __shared__ __attribute__((aligned(16))) __bf16 qs[N][TQ][PITCH];
    __shared__ int64_t q_at[TQ], tab_at[TQ];
    const int MK = a.M * a.K, RG = (a.R + RB - 1) / RB, groups = (MK + 63) / 64, d4 = a.D >> 2;
    const int h = blockIdx.x / groups, lane = lane_id(), i16 = lane & 15, g = lane >> 4;
    const int cw = (blockIdx.x - h * groups) * 64 + (threadIdx.x >> 6) * 16 + i16;
    const int all = a.rows.B * RG * RB;
    const float f = a.factor * kLog2e;
    const float *C = a.C + ((size_t)h * MK + min(cw, MK - 1)) * a.D;
    bf16x8 c[NJ][3];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int at = 32 * j + 8 * g;              // a row is at least four long, and whole fours
        const float4 u = *reinterpret_cast<const float4 *>(C + min(at, a.D - 4)), v = *reinterpret_cast<const float4 *>(C + min(at + 4, a.D - 4));
        const float fu = at < a.D ? 1.f : 0.f, fv = at + 4 < a.D ? 1.f : 0.f;
        const float w[8] = {u.x * fu, u.y * fu, u.z * fu, u.w * fu, v.x * fv, v.y * fv, v.z * fv, v.w * fv};
        split_floats<3>(w, c[j]);
    }
    for (int stage = blockIdx.y; stage < stages; stage += gridDim.y) {
        const int n0 = stage * TQ;
        if (threadIdx.x < TQ) {                     // where the stage's queries are, and where their tables go
            const int n = n0 + (int)threadIdx.x, u = n / RB, b = u / RG, rg = u - b * RG, hq = rg * RB + (n - u * RB);
            q_at[threadIdx.x] = n < all && hq < a.R ? (int64_t)b * a.q_row + (int64_t)(h * a.R + hq) * a.q_head : -1;
            tab_at[threadIdx.x] = n < all ? (((int64_t)b * a.G + h) * RG + rg) * tab_row(a.M, a.K, RB) + (n - u * RB) : -1;
        }
        __syncthreads();
        constexpr int PIECES = TQ * 8 * NJ, EACH = PIECES / kTableThreads;
        static_assert(PIECES % kTableThreads == 0, "whole rounds");
        float4 v[EACH];
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int i = threadIdx.x + j * kTableThreads, row = i / (8 * NJ), p = i - row * (8 * NJ);
            const int64_t at = q_at[row];
            v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (at >= 0 && p < d4) v[j] = T::load(a.Q, at + 4 * p);
        }
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int i = threadIdx.x + j * kTableThreads, row = i / (8 * NJ), p = i - row * (8 * NJ);
            float x[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
            for (int k = 0; k < N; ++k) {
                bf16x4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    o[e] = (__bf16)x[e];
                    x[e] -= (float)o[e];
                }
                *reinterpret_cast<bf16x4 *>(&qs[k][row][4 * p]) = o;
            }
        }
        __syncthreads();
#pragma unroll 2
        for (int tile = 0; tile < TQ / 16; ++tile) {
            if (n0 + 16 * tile >= all) break;
            floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                bf16x8 q[N];
#pragma unroll
                for (int k = 0; k < N; ++k) q[k] = *reinterpret_cast<const bf16x8 *>(&qs[k][16 * tile + i16][32 * j + 8 * g]);
                mfma_parts<N, 3>(q, c[j], s);
            }
            if (cw < MK)
#pragma unroll
                for (int e = 0; e < 4; e += RB) {   // queries n0 + 16 tile + 4 g + e of this lane's codeword
                    const int64_t at = tab_at[16 * tile + 4 * g + e];
                    if (at < 0) break;
                    float *to = tab + at + (int64_t)cw * RB;
                    if (RB == 4) *reinterpret_cast<float4 *>(to) = make_float4(s[0] * f, s[1] * f, s[2] * f, s[3] * f);
                    else if (RB == 2) *reinterpret_cast<float2 *>(to) = make_float2(s[e] * f, s[e + 1] * f);
                    else *to = s[e] * f;
                }
        }
        __syncthreads();
    }
}

// Floats as whole numbers in the same order, and back (no NaN); the largest over the wave (STEPS 6) or its first 16 lanes (4), in every lane.
__device__ __forceinline__ int float_key(float x)
{
    const int i = __float_as_int(x);
    return i ^ (int)((unsigned)(i >> 31) >> 1);
}
template <int STEPS>
__device__ __forceinline__ float key_max(int v)
{
    const int low = (int)0x80000000;
    v = max(v, __builtin_amdgcn_update_dpp(low, v, 0x111, 0xf, 0xf, false));   // row_shr:1
    v = max(v, __builtin_amdgcn_update_dpp(low, v, 0x112, 0xf, 0xf, false));   // row_shr:2
    v = max(v, __builtin_amdgcn_update_dpp(low, v, 0x114, 0xf, 0xf, false));   // row_shr:4
    v = max(v, __builtin_amdgcn_update_dpp(low, v, 0x118, 0xf, 0xf, false));   // row_shr:8
    if (STEPS == 6) {
        v = max(v, __builtin_amdgcn_update_dpp(low, v, 0x142, 0xa, 0xf, false));   // row_bcast:15 into rows 1 and 3
        v = max(v, __builtin_amdgcn_update_dpp(low, v, 0x143, 0xc, 0xf, false));   // row_bcast:31 into rows 2 and 3
    }
    const int i = __builtin_amdgcn_readlane(v, STEPS == 6 ? kWave - 1 : 15);
    return __int_as_float(i ^ (int)((unsigned)(i >> 31) >> 1));
}

// The sum over the wave, the same in every lane.
__device__ __forceinline__ float lanes_sum(float v)
{
#define LANES_PLUS(ctrl, rows) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xf, false))
    LANES_PLUS(0x111, 0xf);                         // row_shr:1, 2, 4, 8
    LANES_PLUS(0x112, 0xf);
    LANES_PLUS(0x114, 0xf);
    LANES_PLUS(0x118, 0xf);
    LANES_PLUS(0x142, 0xa);                         // row_bcast:15 into rows 1 and 3
    LANES_PLUS(0x143, 0xc);                         // row_bcast:31 into rows 2 and 3
#undef LANES_PLUS
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), kWave - 1));
}

struct CodesStat {
    float top, sum, bad, unused;                    // bad: NaN where a value that takes part has no finite scale, else 0
};

// What the launch knows beside the arguments.
struct CodesArgs {
    int splits;
    bool grouped;                                   // blocks go round the eight XCDs: those that read the same rows to one of them
    bool words;                                     // every row's codes are whole, aligned words
    bool small;                                     // offsets within a page fit 32 bits, and its rows 24
    const float *tab;
    CodesStat *stats;
    float *sums;
};

// A block a part of the rows of a key head and RB of its query heads.  Windows of 2048 rows, two or four a thread:
//   scores from the tables in LDS; weights p g' to fixed point, added up by code in LDS; these sums, times what a step stands for, to the running sums,
//   which threads keep in registers.
// Two query heads share a word where outputs are of 16 bits, 32 bits each: a step is under 2^-24 of the most that a wave's rows of a window have weighed together so far (codes_bits),
// and so of all weights' sum, as a float's last place.  Weights are rounded to the step below or above by a fraction that goes round with the row (the golden
// ratio's multiples), so that many small weights add up to what they are.  float outputs and single query heads take 64 bits, steps of 2^-46.  A block looks for the
// largest score and sum of a window only if one of them is beyond what the last ones allow for; a wave adds its weights up to know (less than 1 us of the calls below).
// What bounds it: 64 sequences of 8192 to 16384 rows, 8 key heads, 4 query heads each, M = 8, take 114 us (1.3 TB/s of codes and scales): LDS works for 45 % of it,
// 61 % of that because lanes meet at banks, a SIMD executes vector instructions for 34 %, the memory pipe takes a row's four pieces (two codes, two
// scales, lines of their own) one by one for 37 %; 13 us of a block are its first loads, the tables' 32 KB and its sums' way out, a window of two blocks on a
// CU 12 us.  On the way there, us: 1024 threads with two rows each 184, 512 with one, two and four rows 221, 165 and 148; with offsets in the instructions and the
// largest looked for only when it grows 117; with the next window's codes on their way 114.
// FULL: K = 256 and 4 MW dictionaries, whole aligned words: the offsets in LDS are in the instructions.  BY_WAVE: pages of multiples of 64 rows: the rows of a wave are
// in one page, found in scalar registers.
template <int RB, bool WIDE, int MW, bool FULL, bool BY_WAVE>
__global__ __launch_bounds__(codes_threads(RB, WIDE, MW), 4) void k_attend_codes(const AttendArgs a, const CodesArgs x)
{
    constexpr int kCodesThreads = codes_threads(RB, WIDE, MW), kCodesRows = kWindow / kCodesThreads, kCodesWaves = kCodesThreads / kWave;
    extern __shared__ __attribute__((aligned(16))) char codes_lds[];
    __shared__ float2 red[RB][16];
    __shared__ int any_bad, grow[2];
    constexpr int P = WIDE ? RB : RB / 2, NW = codes_words(RB, WIDE, MW);
    constexpr float kRoom = 8.f;                    // a score may be so far above the reference
    const int M = FULL ? 4 * MW : a.M, K = FULL ? 256 : a.K, MK = M * K, RG = (a.R + RB - 1) / RB, H = 2 * a.G, heads = a.G * RG;
    unsigned u;                                     // part of a sequence; at most 64 each of 16384
    int hr;                                         // key head and group of its query heads
    if (x.grouped) {
        const unsigned at = blockIdx.x >> 3;
        u = at / (unsigned)heads * 8 + (blockIdx.x & 7);
        hr = (int)(at % (unsigned)heads);
    } else {
        u = blockIdx.x / (unsigned)heads;
        hr = (int)(blockIdx.x - u * (unsigned)heads);
    }
    if (u >= (unsigned)a.rows.B * (unsigned)x.splits) return;
    const int b = (int)(u / (unsigned)x.splits), split = (int)(u - (unsigned)b * (unsigned)x.splits), h = hr / RG;
    const int64_t seq = (int64_t)b * heads + hr, job = seq * x.splits + split;
    const SeqRows rows(a, b, h);
    // rows are numbered below 2^31
    const unsigned count = (unsigned)rows.count, per = ((count + (unsigned)x.splits - 1u) / (unsigned)x.splits + 255u) / 256u * 256u;
    const uint64_t first64 = (uint64_t)per * (unsigned)split;
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    if (first64 >= count) {
        if (threadIdx.x < RB) x.stats[job * RB + threadIdx.x] = {kLowest, 0.f, 0.f, 0.f};
        return;
    }
    const unsigned first = (unsigned)first64, last = (unsigned)(first64 + per < count ? first64 + per : count);
    const int words = MK * P;
    unsigned long long *hist = reinterpret_cast<unsigned long long *>(codes_lds);
    float *lut = reinterpret_cast<float *>(codes_lds + codes_lut(words));
    {
        const float4 *from = reinterpret_cast<const float4 *>(x.tab + seq * tab_row(M, K, RB));
        const int fours = (int)(tab_row(M, K, RB) / 4), whole = MK * RB / 4;
        constexpr int EACH = 4;
        for (int i0 = threadIdx.x; i0 < fours; i0 += EACH * kCodesThreads) {
            float4 f[EACH];
#pragma unroll
            for (int j = 0; j < EACH; ++j) f[j] = from[min(i0 + j * kCodesThreads, fours - 1)];
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const int i = i0 + j * kCodesThreads;
                if (i < whole) *reinterpret_cast<float4 *>(lut + 4 * i) = f[j];
                else if (i < fours) {               // a last one that is not whole
                    const float e[4] = {f[j].x, f[j].y, f[j].z, f[j].w};
                    for (int k = 4 * i; k < MK * RB; ++k) lut[k] = e[k - 4 * i];
                }
            }
        }
        for (int i = threadIdx.x; i < words; i += kCodesThreads) hist[i] = 0;
        if (threadIdx.x == 0) any_bad = grow[0] = grow[1] = 0;
    }
    // which pair of query heads a word of this thread's is for, two bits each
    uint64_t pairs = 0;
#pragma unroll
    for (int j = 0; j < NW; ++j) pairs |= (uint64_t)((threadIdx.x + j * kCodesThreads) / K % P) << (2 * j);
    float acc[NW][WIDE ? 1 : 2] = {};
    constexpr int kBits = codes_bits(RB, WIDE, MW);
    // WIDE: of a weight, 2048 of which stay far below 2^63; else of a wave's sum
    constexpr float top_steps = WIDE ? 0x1p51f : 1.75f * (float)(1 << (WIDE ? 0 : kBits));
    static_assert(WIDE || (int64_t)kCodesWaves << kBits == 1 << 30, "7/4 of it and 2048 steps are below 2^31");
    float ref[RB], unit[RB], back[RB], largest[RB], sum[RB];   // reference of the scores, steps in 1 and their size, log2 of the largest sum of a wave's weights so far
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        ref[r] = kLowest;
        largest[r] = -INFINITY;
        unit[r] = back[r] = 1.f;
        sum[r] = 0.f;
    }
    bool bad = false;
    const unsigned page_codes = (unsigned)a.rows.page * (unsigned)(H * M), page_scales = (unsigned)a.rows.page * (unsigned)H;   // used where they fit
    const unsigned lane_codes = (unsigned)(lane * H * M), lane_scales = (unsigned)(lane * H);
    // Where the rows of a window are; their codes and scales, sent for while the window before is added up.
    bool there[kCodesRows], there_next[kCodesRows];
    unsigned page_next[kCodesRows], off_next[kCodesRows];
    unsigned kc[kCodesRows][MW], vc[kCodesRows][MW];
    float gk[kCodesRows], gv[kCodesRows];
    auto locate = [&](unsigned w) {
#pragma unroll
        for (int i = 0; i < kCodesRows; ++i) {
            unsigned off = 0, q = ~0u;
            if (BY_WAVE) {
                const unsigned t = __builtin_amdgcn_readfirstlane(w + i * kCodesThreads + wave * kWave);
                int64_t at = 0;
                if (t < last) q = __builtin_amdgcn_readfirstlane(rows.where_wave(t, off, at));
                there_next[i] = q != ~0u && t + lane < last && at + lane >= rows.begin && at + lane < rows.end;
            } else {
                const unsigned t = w + i * kCodesThreads + threadIdx.x;
                if (t < last) q = rows.where(t, off);
                there_next[i] = q != ~0u;
            }
            page_next[i] = q;
            off_next[i] = off;
        }
    };
    auto fetch = [&](unsigned (&kc)[kCodesRows][MW], unsigned (&vc)[kCodesRows][MW], float (&gk)[kCodesRows], float (&gv)[kCodesRows]) {
#pragma unroll
        for (int i = 0; i < kCodesRows; ++i) {
            gk[i] = gv[i] = 1.f;
#pragma unroll
            for (int j = 0; j < MW; ++j) kc[i][j] = vc[i][j] = 0u;
            if (!there_next[i]) continue;
            const uint8_t *kp = a.codes + h * M;
            const float *gp = a.scale;
            if (BY_WAVE) {
                const uint64_t row = (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane(page_next[i]) * (unsigned)a.rows.page + (unsigned)__builtin_amdgcn_readfirstlane(off_next[i]);
                kp += row * (unsigned)(H * M) + lane_codes;
                gp += row * (unsigned)H + lane_scales;
            } else if (x.small) {
                kp += (uint64_t)page_next[i] * page_codes + __umul24(off_next[i], (unsigned)(H * M));
                gp += (uint64_t)page_next[i] * page_scales + __umul24(off_next[i], (unsigned)H);
            } else {
                const uint64_t row = (uint64_t)page_next[i] * (unsigned)a.rows.page + off_next[i];
                kp += row * (unsigned)(H * M);
                gp += row * (unsigned)H;
            }
            const uint8_t *vp = kp + a.G * M;
            if (FULL) {
                typedef unsigned row_words __attribute__((ext_vector_type(MW < 4 ? MW : 4), aligned(4)));
#pragma unroll
                for (int j = 0; j < MW; j += 4) {
                    const row_words k4 = *reinterpret_cast<const row_words *>(kp + 4 * j), v4 = *reinterpret_cast<const row_words *>(vp + 4 * j);
#pragma unroll
                    for (int e = 0; e < (MW < 4 ? MW : 4); ++e) {
                        kc[i][j + e] = k4[e];
                        vc[i][j + e] = v4[e];
                    }
                }
            } else if (x.words) {
#pragma unroll
                for (int j = 0; j < MW; ++j)
                    if (4 * j < M) {
                        kc[i][j] = reinterpret_cast<const unsigned *>(kp)[j];
                        vc[i][j] = reinterpret_cast<const unsigned *>(vp)[j];
                    }
            } else {
#pragma unroll
                for (int m = 0; m < 4 * MW; ++m)
                    if (m < M) {
                        kc[i][m >> 2] |= (unsigned)kp[m] << (8 * (m & 3));
                        vc[i][m >> 2] |= (unsigned)vp[m] << (8 * (m & 3));
                    }
            }
            if (a.scale) {
                gk[i] = gp[h];
                gv[i] = gp[a.G + h];
            }
        }
    };
    locate(first);
    fetch(kc, vc, gk, gv);
    __syncthreads();
    int turn_of = 0;
    for (unsigned w0 = first; w0 < last; w0 += kWindow, turn_of ^= 1) {
#pragma unroll
        for (int i = 0; i < kCodesRows; ++i) there[i] = there_next[i];
        float s[kCodesRows][RB], v[kCodesRows][RB];
        locate(w0 + kWindow);
        float here[RB];                             // the window's sums of exponentials
        float highest = 0.f, heaviest = 0.f;        // score above its reference, weight in steps (WIDE); NaN are passed over
        float heavy[RB];                            // the weights' sum in steps (not WIDE)
        // weights in steps (WIDE: as they are), with the fraction that decides which way they are rounded
        auto weigh = [&](int i) {
            const float turn = (float)(((w0 + i * kCodesThreads + threadIdx.x) * 0x9E3779B9u) >> 8) * 0x1p-24f;
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const float e = s[i][r] - ref[r], p = __builtin_amdgcn_exp2f(e), w = p * gv[i];
                here[r] += p;
                v[i][r] = WIDE ? w : w * unit[r] + turn;
                highest = fmaxf(highest, e);
                if (WIDE) heaviest = fmaxf(heaviest, fabsf(w * unit[r]));
                else heavy[r] += fabsf(v[i][r]);
            }
        };
#pragma unroll
        for (int r = 0; r < RB; ++r) here[r] = heavy[r] = 0.f;
#pragma unroll
        for (int i = 0; i < kCodesRows; ++i) {
#pragma unroll
            for (int r = 0; r < RB; ++r) s[i][r] = 0.f;
            if (!there[i]) continue;
#pragma unroll
            for (int m = 0; m < 4 * MW; ++m)
                if (m < M) {
                    unsigned k = kc[i][m >> 2] >> (8 * (m & 3)) & 255u;
                    if (!FULL) k = min(k, (unsigned)K - 1u);
                    const float *e = lut + m * K * RB + k * RB;
                    if (RB == 4) {
                        const float4 f = *reinterpret_cast<const float4 *>(e);
                        s[i][0] += f.x;
                        s[i][RB > 1 ? 1 : 0] += f.y;
                        s[i][RB > 2 ? 2 : 0] += f.z;
                        s[i][RB > 3 ? 3 : 0] += f.w;
                    } else if (RB == 2) {
                        const float2 f = *reinterpret_cast<const float2 *>(e);
                        s[i][0] += f.x;
                        s[i][RB > 1 ? 1 : 0] += f.y;
                    } else s[i][0] += *e;
                }
#pragma unroll
            for (int r = 0; r < RB; ++r) s[i][r] *= gk[i];
            bad |= !(fabsf(gv[i]) < INFINITY);
            weigh(i);
        }
        bool more = highest > kRoom || heaviest > top_steps;
        if (!WIDE)
#pragma unroll
            for (int r = 0; r < RB; ++r) more |= !(lanes_sum(heavy[r]) <= top_steps);    // a NaN too: it would hide what is beside it
        if (more) grow[turn_of] = 1;                // the same value from whoever writes
        __syncthreads();
        if (grow[turn_of]) {                        // the largest score of the window over the block, then the largest sum of a wave's weights
            float now[RB], fade[RB];
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < kCodesRows; ++i)
                    if (there[i]) top = fmaxf(top, s[i][r]);
                top = key_max<6>(float_key(top));
                if (lane == 0) red[r][wave].x = top;
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                now[r] = fmaxf(ref[r], key_max<4>(float_key(red[r][min(lane, kCodesWaves - 1)].x)));
                float l[kCodesRows], most = -INFINITY;  // log2 of the weights that the reference makes
#pragma unroll
                for (int i = 0; i < kCodesRows; ++i) {
                    l[i] = there[i] ? (s[i][r] - now[r]) + __builtin_amdgcn_logf(fabsf(gv[i])) : -INFINITY;
                    most = fmaxf(most, l[i]);
                }
                most = key_max<6>(float_key(most));
                float all = 0.f;                    // in parts of the largest; what is no number counts nothing
#pragma unroll
                for (int i = 0; i < kCodesRows; ++i) all += fmaxf(__builtin_amdgcn_exp2f(l[i] - most), 0.f);
                all = lanes_sum(all);
                if (lane == 0) red[r][wave].y = most + fmaxf(__builtin_amdgcn_logf(all), 0.f);
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const float move = ref[r] - now[r];
                fade[r] = __builtin_amdgcn_exp2f(move);
                largest[r] = fmaxf(largest[r] == -INFINITY ? largest[r] : largest[r] + move, key_max<4>(float_key(red[r][min(lane, kCodesWaves - 1)].y)));
                ref[r] = now[r];
                // a wave's weights are 2^e together; only zeros: any step
                const float e = largest[r] == -INFINITY ? 0.f : fminf(fmaxf(ceilf(largest[r] + 0.01f), -100.f), 140.f);
                const int n = min(kBits - (int)e, 120);
                unit[r] = ldexpf(1.f, n);
                back[r] = ldexpf(1.f, -n);
                sum[r] *= fade[r];
                here[r] = heavy[r] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < NW; ++j) {
                const int q = (int)(pairs >> (2 * j) & 3);
                if (WIDE) {
                    float f = fade[0];
#pragma unroll
                    for (int r = 1; r < RB; ++r)
                        if (q == r) f = fade[r];
                    acc[j][0] *= f;
                } else {
                    const bool second = RB == 4 && q == 1;
                    acc[j][0] *= second ? fade[RB == 4 ? 2 : 0] : fade[0];
                    acc[j][WIDE ? 0 : 1] *= second ? fade[RB - 1] : fade[RB >= 2 ? 1 : 0];
                }
            }
#pragma unroll
            for (int i = 0; i < kCodesRows; ++i)
                if (there[i]) weigh(i);
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) sum[r] += here[r];
        if (threadIdx.x == 0) grow[turn_of ^ 1] = 0;
        unsigned kn[kCodesRows][MW], vn[kCodesRows][MW];
        float gkn[kCodesRows], gvn[kCodesRows];
        fetch(kn, vn, gkn, gvn);
#pragma unroll
        for (int i = 0; i < kCodesRows; ++i) {
            if (!there[i]) continue;
            unsigned long long add[P];
#pragma unroll
            for (int q = 0; q < P; ++q) {
                if (WIDE) {
                    const double d = (double)v[i][q] * (double)unit[q];
                    add[q] = (unsigned long long)(d == d ? (long long)rint(d) : 0ll);
                } else {
                    const int lo = (int)floorf(v[i][(2 * q) % RB]), hi = (int)floorf(v[i][(2 * q + 1) % RB]);
                    add[q] = (unsigned long long)(unsigned)(hi + (lo >> 31)) << 32 | (unsigned)lo;
                }
            }
            unsigned long long any = add[0];
#pragma unroll
            for (int q = 1; q < P; ++q) any |= add[q];
            if (any == 0) continue;                 // weights that are no step: rows that hardly count do not meet at banks
#pragma unroll
            for (int m = 0; m < 4 * MW; ++m)
                if (m < M) {
                    unsigned k = vc[i][m >> 2] >> (8 * (m & 3)) & 255u;
                    if (!FULL) k = min(k, (unsigned)K - 1u);
#pragma unroll
                    for (int q = 0; q < P; ++q)
                        __hip_atomic_fetch_add(hist + (m * P + q) * K + k, add[q], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NW; ++j) {
            const int i = threadIdx.x + j * kCodesThreads, q = (int)(pairs >> (2 * j) & 3);
            if (i >= words) break;
            const unsigned long long w = hist[i];
            hist[i] = 0;
            if (WIDE) {
                float o = back[0];
#pragma unroll
                for (int r = 1; r < RB; ++r)
                    if (q == r) o = back[r];
                acc[j][0] += (float)((double)(long long)w * (double)o);
            } else {
                const int lo = (int)(unsigned)w, hi = (int)((unsigned)(w >> 32) + ((unsigned)w >> 31));
                const bool second = RB == 4 && q == 1;
                acc[j][0] += (float)lo * (second ? back[RB == 4 ? 2 : 0] : back[0]);
                acc[j][WIDE ? 0 : 1] += (float)hi * (second ? back[RB - 1] : back[RB >= 2 ? 1 : 0]);
            }
        }
#pragma unroll
        for (int i = 0; i < kCodesRows; ++i) {
            gk[i] = gkn[i];
            gv[i] = gvn[i];
#pragma unroll
            for (int j = 0; j < MW; ++j) {
                kc[i][j] = kn[i][j];
                vc[i][j] = vn[i][j];
            }
        }
    }
    if (bad) any_bad = 1;                           // the same value from whoever writes
    // the exponentials' sums, in a fixed order
    float *sums16 = reinterpret_cast<float *>(red);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        float v = sum[r];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
        if (lane == 0) sums16[r * 16 + wave] = v;
    }
    __syncthreads();
    if (threadIdx.x < RB) {
        float v = 0.f, t = 0.f;
        for (int w = 0; w < kCodesWaves; ++w) v += sums16[threadIdx.x * 16 + w];
#pragma unroll
        for (int r = 0; r < RB; ++r)
            if ((int)threadIdx.x == r) t = ref[r];
        x.stats[job * RB + threadIdx.x] = {t, v, any_bad ? NAN : 0.f, 0.f};
    }
    const int64_t row = sums_row(M, K);
    float *to = x.sums + job * RB * row;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
        const int i = threadIdx.x + j * kCodesThreads, q = (int)(pairs >> (2 * j) & 3);
        if (i >= words) break;
        const int e = i / K, mk = e / P * K + (i - e * K);
        if (WIDE) to[q * row + mk] = acc[j][0];
        else {
            to[2 * q * row + mk] = acc[j][0];
            to[(2 * q + 1) * row + mk] = acc[j][WIDE ? 0 : 1];
        }
    }
    if (threadIdx.x < RB)
        for (int64_t i = MK; i < row; ++i) to[threadIdx.x * row + i] = 0.f;     // up to whole fours
}

constexpr int kFoldThreads = 256, kFoldFrom = 5;   // parts from which they are added up by a kernel of their own

// What the parts of a query head amount to: their common reference, its sum, NaN where a value is; f: what each counts.  By one wave.
__device__ __forceinline__ CodesStat join_parts(const CodesStat *st, int64_t stride, int splits, float *f)
{
    static_assert(kCodesSplits <= kWave, "a part a lane");
    const int lane = lane_id();
    CodesStat x = {kLowest, 0.f, 0.f, 0.f};
    if (lane < splits) x = st[lane * stride];
    float top = x.top, bad = x.bad;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        top = fmaxf(top, __shfl_xor(top, o, kWave));
        bad += __shfl_xor(bad, o, kWave);
    }
    const float e = x.sum != 0.f ? __builtin_amdgcn_exp2f(x.top - top) : 0.f;       // a part without rows has no sums; nor need one whose rows weigh nothing be read
    float sum = x.sum != 0.f ? e * x.sum : 0.f;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
    if (lane < splits) f[lane] = e;
    return {top, sum, bad, 0.f};
}

// The parts' sums by code added up, a block 1024 of a query head's; they take the place of the first part's.  32 parts of 64 query heads, M = 8, K = 256 (17 MB): 7 us;
// the product below took 207 us where it added 32 parts up by itself, with 1 to 4 it is faster than two launches.
template <int RB>
__global__ __launch_bounds__(kFoldThreads) void k_attend_fold(const AttendArgs a, int splits, const CodesStat *stats, float *sums, CodesStat *joined)
{
    __shared__ float f[kCodesSplits];
    const int64_t n = blockIdx.x, seq = n / RB, row = sums_row(a.M, a.K);
    const int r = (int)(n - seq * RB);
    if (threadIdx.x < kWave) {
        const CodesStat x = join_parts(stats + seq * splits * RB + r, RB, splits, f);
        if (threadIdx.x == 0 && blockIdx.y == 0) joined[n] = x;
    }
    __syncthreads();
    const int64_t i = (int64_t)(blockIdx.y * kFoldThreads + threadIdx.x) * 4;
    if (i >= row) return;
    float *to = sums + (seq * splits * RB + r) * row + i;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < splits; s0 += 8) {
        float4 w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const float4 *>(to + (int64_t)min(s0 + j, splits - 1) * RB * row);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = s0 + j < splits ? f[s0 + j] : 0.f;
            if (e != 0.f) v = make_float4(v.x + e * w[j].x, v.y + e * w[j].y, v.z + e * w[j].z, v.w + e * w[j].w);
        }
    }
    *reinterpret_cast<float4 *>(to) = v;
}

constexpr int kOutThreads = 1024, kOutWaves = kOutThreads / kWave, kOutChunk = 64, kOutPitch = kOutChunk + 8, kOutParts = 3;
__host__ __device__ constexpr int out_lds(int CW)
{
    const int rows = kOutWaves * kOutParts * 16 * kOutPitch * 2, sums = kOutWaves * 16 * (16 * CW + 1) * 4;
    return rows > sums ? rows : sums;
}

// out = the sums by code times the codewords, over the exponentials' sum: a block 16 query heads and 16 CW coordinates (a lane CW side by side), its waves
// every sixteenth 64 codewords each.  A wave lays the 64 sums of 16 query heads out in LDS of its own, the parts added up on the way.
// Blocks of one XCD (they go round the eight) have neighbouring numbers, which is the same head most often: its codewords stay in that L2.
// Sums and codewords are three bf16 parts each, as in the tables, which is what a float holds (with two, 17 bits, calls of many rows take 1 to 7 % less).
// 2048 query heads, D = 128, M = 8, K = 256: 21 us, with two parts 16 (with those: fp32 matrix cores 28; eight waves a block 17; the next 64 codewords on their way 19): a chain of loads, LDS and products
// for every 64 codewords of a wave; the sums are read once for each 64 coordinates.
// span: parts between one sequence's sums and the next; splits: parts to add up, the first of those.
template <typename T, int RB, int CW>
__global__ __launch_bounds__(kOutThreads, 4) void k_attend_out(const AttendArgs a, int splits, int span, int tiles, const CodesStat *stats, const float *sums)
{
    constexpr int N = kOutParts;
    extern __shared__ __attribute__((aligned(16))) float out_room[];
    __shared__ float part[16][kCodesSplits];
    const int RG = (a.R + RB - 1) / RB, MK = a.M * a.K, slices = (a.D + 16 * CW - 1) / (16 * CW), all = a.rows.B * RG * RB;
    const int total = tiles * a.G * slices, per_xcd = (total + 7) / 8, job = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || job >= total) return;
    const int h = job / (tiles * slices), rest = job - h * tiles * slices, tile = rest / slices, slice = rest - tile * slices;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, g = lane >> 4;
    auto seq_of = [&](int n) {
        const int u = n / RB, b = u / RG;
        return ((int64_t)b * a.G + h) * RG + (u - b * RG);
    };
    const int d = (slice * 16 + i16) * CW;
    const float *C = a.C + (size_t)(a.G + h) * MK * a.D + min(d, a.D - CW);
    auto codewords = [&](int k0, float (&c)[8][CW]) {   // k0 + 8 g .. + 7
        const bool whole = k0 + 32 <= MK;
        const float *from = C + (size_t)(whole ? k0 + 8 * g : 0) * a.D;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float *at = whole ? from + e * a.D : C + (size_t)min(k0 + 8 * g + e, MK - 1) * a.D;
            if (CW == 4) {
                const float4 q = *reinterpret_cast<const float4 *>(at);
                c[e][0] = q.x;
                c[e][CW > 1 ? 1 : 0] = q.y;
                c[e][CW > 2 ? 2 : 0] = q.z;
                c[e][CW > 3 ? 3 : 0] = q.w;
            } else c[e][0] = *at;
        }
    };
    const int64_t row = sums_row(a.M, a.K);
    const float *from[4];                           // a lane's four rows of sums
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = min(tile * 16 + 4 * j + g, all - 1);
        from[j] = sums + (seq_of(n) * span * RB + n % RB) * row;
    }
#pragma unroll
    for (int j = 0; j < 16 / kOutWaves; ++j) {      // what a part counts, a wave a query head
        const int i = wave * (16 / kOutWaves) + j, n = tile * 16 + i, u = n / RB, b = u / RG, hq = (u - b * RG) * RB + (n - u * RB);
        if (n < all && hq < a.R) {
            const CodesStat x = join_parts(stats + seq_of(n) * splits * RB + n % RB, RB, splits, part[i]);
            if (lane < splits) part[i][lane] = (x.sum != 0.f ? part[i][lane] / x.sum : 0.f) + x.bad;
            if (slice == 0 && lane == 0 && a.lse) a.lse[(int64_t)b * a.G * a.R + h * a.R + hq] = x.sum != 0.f ? (x.top + log2f(x.sum)) * kLn2 : -INFINITY;
        } else if (lane < splits) part[i][lane] = 0.f;
    }
    __syncthreads();
    __bf16 *mine = reinterpret_cast<__bf16 *>(out_room) + wave * N * 16 * kOutPitch;
    floatx4 s[CW];
#pragma unroll
    for (int q = 0; q < CW; ++q) s[q] = (floatx4){0.f, 0.f, 0.f, 0.f};
    auto products = [&](int j, const float (&c)[8][CW]) {
        bf16x8 v[N];
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = *reinterpret_cast<const bf16x8 *>(mine + (k * 16 + i16) * kOutPitch + j + 8 * g);
#pragma unroll
        for (int q = 0; q < CW; ++q) {
            float x[8];
            bf16x8 o[N];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = c[e][q];
            split_floats<N>(x, o);
            mfma_parts<N, N>(v, o, s[q]);
        }
    };
    for (int k0 = wave * kOutChunk; k0 < MK; k0 += kOutWaves * kOutChunk) {
        float c0[8][CW], c1[8][CW];
        codewords(k0, c0);
        // four rows at a time, a quarter of the wave each
        float4 w[4];
        const int at = k0 + 4 * i16;
        const int64_t near = min((int64_t)at, row - 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p = 0; p < splits; ++p) {
            float4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const float4 *>(from[j] + (int64_t)p * RB * row + near);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float f = part[4 * j + g][p];
                if (f != 0.f && at < row) w[j] = make_float4(w[j].x + f * x[j].x, w[j].y + f * x[j].y, w[j].z + f * x[j].z, w[j].w + f * x[j].w);
            }
        }
        codewords(min(k0 + 32, MK - 1), c1);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float x[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
            for (int k = 0; k < N; ++k) {
                bf16x4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    o[e] = (__bf16)x[e];
                    x[e] -= (float)o[e];
                }
                *reinterpret_cast<bf16x4 *>(mine + (k * 16 + 4 * j + g) * kOutPitch + 4 * i16) = o;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        products(0, c0);
        products(32, c1);
    }
    // A codeword that is not finite, or no sum of finite bf16 parts, is a NaN in every row of its column, whether its sum is zero or not.  Where a NaN is none of its query head's
    // the wave multiplies again, one by one, and leaves out what no row has: 115 to 290 us more a call; the look costs nothing that shows.
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int q = 0; q < CW; ++q) odd |= s[q][e] != s[q][e];
    if (__ballot(odd)) {
        odd = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            bool number = true;
            for (int p = 0; p < splits; ++p) number &= part[4 * g + e][p] == part[4 * g + e][p];
#pragma unroll
            for (int q = 0; q < CW; ++q) odd |= number && s[q][e] != s[q][e];
        }
    }
    if (__ballot(odd)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int n = min(tile * 16 + 4 * g + e, all - 1);
            const float *sum = sums + (seq_of(n) * span * RB + n % RB) * row;
            float v[CW] = {};
            for (int k0 = wave * kOutChunk; k0 < MK; k0 += kOutWaves * kOutChunk)
                for (int k = k0; k < min(k0 + kOutChunk, MK); ++k) {
                    float w = 0.f;
                    for (int p = 0; p < splits; ++p)
                        if (part[4 * g + e][p] != 0.f) w += part[4 * g + e][p] * sum[(int64_t)p * RB * row + k];
                    if (w != 0.f)
#pragma unroll
                        for (int q = 0; q < CW; ++q) v[q] += w * C[(size_t)k * a.D + q];
                }
#pragma unroll
            for (int q = 0; q < CW; ++q) s[q][e] = v[q];
        }
    }
    __syncthreads();                                // the sums' places are free
    constexpr int OP = 16 * CW + 1;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int q = 0; q < CW; ++q) out_room[(wave * 16 + 4 * g + e) * OP + i16 * CW + q] = s[q][e];
    __syncthreads();
    for (int t = threadIdx.x; t < 64 * CW; t += kOutThreads) {
        const int i = t / (4 * CW), p = t - i * 4 * CW, m = tile * 16 + i, u = m / RB, b = u / RG, hq = (u - b * RG) * RB + (m - u * RB), at = slice * 16 * CW + 4 * p;
        if (m < all && hq < a.R && at < a.D) {
            float v[4] = {};
            for (int w = 0; w < kOutWaves; ++w)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += out_room[(w * 16 + i) * OP + 4 * p + e];
            T::store(a.out, (int64_t)b * a.o_row + (int64_t)(h * a.R + hq) * a.o_head + at, make_float4(v[0], v[1], v[2], v[3]));
        }
    }
}

}  // namespace hclae
