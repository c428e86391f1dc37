// Attention of one new token of every sequence over its rows of a coded cache (hclae_cache_attend).
//   s_t = factor g_t q . (sum_m C[h][m][k_m(t)]),  p = softmax(s),  out = sum_t p_t g'_t sum_m C[G + h][m][v_m(t)]
// Scores are kept times log2(e) and exponentials taken to the base 2; softmax statistics, weights and sums are in 32 bits or more.
//   k_attend_rows, k_attend_join   rows decoded as they are needed: any shape, and few rows
//   k_attend_tables, k_attend_codes, k_attend_out   many rows, never decoded: q . C[h][m][k] is tabulated once for all codewords, a row's score is
//       the sum of M entries; the weights of the rows are summed by the codes of their values, and these sums meet the codewords at the end.
//       A row costs M reads and M adds a query head in place of M D, whatever D is.
#pragma once
#include <type_traits>

#include "decode.hpp"
#include "serve.hpp"

namespace hclae {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

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
    // i in [0, count)
    __host__ __device__ constexpr int64_t slot(unsigned i) const
    {
        unsigned j = 0, off = 0;
        if (picks) {
            const unsigned e = page_of(i);
            off = i - e * page;
            const int32_t at = picks[e];
            if (at < 0 || at >= max_pages) return kNoRow;
            const int64_t t = (int64_t)at * page + off;
            if (t < begin || t >= end) return kNoRow;
            j = (unsigned)at;
        } else {
            const unsigned t = (unsigned)begin + i;
            j = page_of(t);
            off = t - j * page;
        }
        const int32_t q = table[j];
        return (unsigned)q < named ? (int64_t)((uint64_t)(unsigned)q * page + off) : kNoRow;
    }
};

// Numbers of rows at most, over all sequences.
__host__ __device__ constexpr int64_t attend_capacity(const AttendArgs &a) { return (int64_t)(a.picked ? a.n_picked : a.rows.max_pages) * a.rows.page; }

constexpr int kDirectThreads = 256, kDirectTile = 32, kDirectSplits = 256;

// Query heads a block takes at once.
__host__ __device__ constexpr int heads_at_once(int R) { return R >= 3 ? 4 : R; }

// Parts of the rows of a sequence and head: four blocks a CU where there are rows enough.
__host__ __device__ constexpr int direct_splits(const AttendArgs &a, int cus)
{
    const int RB = heads_at_once(a.R);
    const int64_t jobs = (int64_t)a.rows.B * a.G * ((a.R + RB - 1) / RB), tiles = (attend_capacity(a) + kDirectTile - 1) / kDirectTile;
    int64_t s = (4ll * cus + jobs - 1) / jobs;
    if (s > tiles) s = tiles;
    if (s > kDirectSplits) s = kDirectSplits;
    return (int)(s < 1 ? 1 : s);
}

// stats of a part and query head: the largest score (-inf: no rows) and the sum of exponentials below it.
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

// A block a part of the rows of one key head and RB of its query heads; `lanes` threads a row, the power of two from D / 4 up.
template <typename T, int RB>
__global__ __launch_bounds__(kDirectThreads) void k_attend_rows(const AttendArgs a, int splits, int lanes, PartStat *stats, float *sums)
{
    __shared__ float4 q[RB][64], red[kDirectThreads];
    __shared__ float s[RB][kDirectTile], w[RB][kDirectTile], fade[RB];
    __shared__ int64_t slots[kDirectTile];
    const int RG = (a.R + RB - 1) / RB, d4 = a.D >> 2, H = 2 * a.G;
    const int64_t job = blockIdx.x, head = job / splits;
    const int split = (int)(job - head * splits), rg = (int)(head % RG), h = (int)(head / RG % a.G), b = (int)(head / RG / a.G);
    const SeqRows rows(a, b, h);
    const int64_t per = ((rows.count + splits - 1) / splits + kDirectTile - 1) / kDirectTile * kDirectTile, first = per * split, last = min(rows.count, first + per);
    const int lane = lane_id(), wave = threadIdx.x >> 6, g = threadIdx.x / lanes, p = threadIdx.x % lanes, groups = kDirectThreads / lanes;
    if (first >= last) {
        if (threadIdx.x < RB) stats[job * RB + threadIdx.x] = {-INFINITY, 0.f};
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
    float top = -INFINITY, sum = 0.f;               // of head `wave`, in every lane of its wave
    for (int64_t t0 = first; t0 < last; t0 += kDirectTile) {
        if (threadIdx.x < kDirectTile) slots[threadIdx.x] = t0 + threadIdx.x < last ? rows.slot((unsigned)(t0 + threadIdx.x)) : kNoRow;
        __syncthreads();
        for (int i = g; i < kDirectTile; i += groups) {
            const int64_t at = slots[i];
            float dot[RB] = {};
            if (at >= 0 && p < d4) {
                const float4 k = decode_piece(Ck, a.codes + (at * H + h) * a.M, a.M, a.K, a.D);
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const float4 v = q[r][p];
                    dot[r] = k.x * v.x + k.y * v.y + k.z * v.z + k.w * v.w;
                }
            }
            for (int o = lanes >> 1; o > 0; o >>= 1)
#pragma unroll
                for (int r = 0; r < RB; ++r) dot[r] += __shfl_xor(dot[r], o, kWave);
            if (p == 0) {
                const float f = at >= 0 && a.scale ? a.scale[at * H + h] : 1.f;
#pragma unroll
                for (int r = 0; r < RB; ++r) s[r][i] = dot[r] * f;
            }
        }
        __syncthreads();
        if (wave < RB) {
            const bool there = lane < kDirectTile && slots[lane & (kDirectTile - 1)] >= 0;
            const float x = there ? s[wave][lane] : -INFINITY;
            float m = x;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
            const float now = fmaxf(top, m);
            float e = there ? exp2f(x - now) : 0.f;
            if (lane < kDirectTile) {
                const int64_t at = slots[lane];
                w[wave][lane] = there ? (a.scale ? e * a.scale[at * H + a.G + h] : e) : 0.f;
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) e += __shfl_xor(e, o, kWave);
            const float f = top == -INFINITY ? 0.f : exp2f(top - now);
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
        for (int i = g; i < kDirectTile; i += groups) {
            const int64_t at = slots[i];
            if (at < 0 || p >= d4) continue;
            const float4 v = decode_piece(Cv, a.codes + (at * H + a.G + h) * a.M, a.M, a.K, a.D);
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const float f = w[r][i];
                acc[r] = make_float4(acc[r].x + f * v.x, acc[r].y + f * v.y, acc[r].z + f * v.z, acc[r].w + f * v.w);
            }
        }
        __syncthreads();
    }
    if (wave < RB && lane == 0) stats[job * RB + wave] = {top, sum};
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        red[threadIdx.x] = acc[r];
        __syncthreads();
        if (threadIdx.x < d4) {
            float4 v = red[threadIdx.x];
            for (int i = 1; i < groups; ++i) {
                const float4 o = red[i * lanes + threadIdx.x];
                v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
            }
            reinterpret_cast<float4 *>(sums)[(job * RB + r) * d4 + threadIdx.x] = v;
        }
        __syncthreads();
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
    float top = -INFINITY;
    for (int i = 0; i < splits; ++i) top = fmaxf(top, stat[(int64_t)i * RB].top);
    float sum = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    const int p = threadIdx.x;
    bool any = false;
    for (int i = 0; i < splits; ++i) {
        const PartStat st = stat[(int64_t)i * RB];
        if (st.sum == 0.f) continue;                // no rows
        any = true;
        const float f = exp2f(st.top - top);
        sum += f * st.sum;
        if (p < d4) {
            const float4 o = reinterpret_cast<const float4 *>(sums)[((job + i) * RB + r % RB) * d4 + p];
            v = make_float4(v.x + f * o.x, v.y + f * o.y, v.z + f * o.z, v.w + f * o.w);
        }
    }
    if (any) {
        const float f = 1.f / sum;
        v = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
    }
    if (p < d4) T::store(a.out, (int64_t)b * a.o_row + (int64_t)hq * a.o_head + 4 * p, v);
    if (p == 0 && a.lse) a.lse[(int64_t)b * Hq + hq] = any ? (top + log2f(sum)) * kLn2 : -INFINITY;
}

// ---- from tables --------------------------------------------------------------------------------

constexpr int kCodesThreads = 1024, kCodesRows = 2, kWindow = kCodesThreads * kCodesRows, kCodesWaves = kCodesThreads / kWave;
constexpr int kCodesMaxM = 32, kCodesSplits = 64;
constexpr int kCodesLds = 152 * 1024;               // tables and sums; the rest is for what the kernel declares
constexpr int kWideBits = 40, kPairBits = 19;       // steps of a fixed-point weight, as powers of two below the largest of its window

// Weights are summed in fixed point, by integer atomics on LDS, so that their order changes nothing.  wide: 64 bits a query head, else two query heads in
// 64 bits, 32 each.
struct CodesPlan {
    int RB;                                         // query heads of a block; 0: the shape is not for tables
    bool wide;
    int words;                                      // of 64 bits
    int lds;
};
__host__ __device__ constexpr CodesPlan codes_plan(int R, int M, int K, bool wide)
{
    if (M > kCodesMaxM) return {0, false, 0, 0};
    for (int RB = heads_at_once(R); RB >= 1; RB /= 2) {
        const bool w = wide || RB == 1;
        const int words = M * K * (w ? RB : RB / 2), lds = M * K * RB * 4 + words * 8;
        if (lds <= kCodesLds) return {RB, w, words, lds};
    }
    return {0, false, 0, 0};
}
// Words a thread looks after, for code rows of up to MW words.
__host__ __device__ constexpr int codes_words(int RB, bool wide, int MW)
{
    const int each = wide ? RB : RB / 2, most = (kCodesLds / (wide ? 12 : 16) + kCodesThreads - 1) / kCodesThreads;
    return MW * each < most ? MW * each : most;
}
__host__ __device__ constexpr int codes_splits(const AttendArgs &a, int RB, int cus)
{
    const int64_t jobs = (int64_t)a.rows.B * a.G * ((a.R + RB - 1) / RB);
    int64_t s = (2ll * cus + jobs - 1) / jobs, most = (attend_capacity(a) + 1023) / 1024;
    if (s > most) s = most;
    if (s > kCodesSplits) s = kCodesSplits;
    return (int)(s < 1 ? 1 : s);
}
// Rows of sums: whole fours.
__host__ __device__ constexpr int64_t sums_row(int M, int K) { return ((int64_t)M * K + 3) / 4 * 4; }

typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kTableThreads = 256;

// tab[b][h][rg][codeword][RB] = factor log2(e) q . c on the fp32 matrix cores.  A wave keeps 16 codewords in registers and takes tiles of 16 queries past
// them; queries of a head are numbered (b, rg, r).  The 4 x 4 blocks of an instruction take coordinates 16 j + 4 g + e, g the quarter of the wave: a lane so
// loads four side by side, for both operands alike.
template <typename T, int RB, int NJ>
__global__ __launch_bounds__(kTableThreads) void k_attend_tables(const AttendArgs a, int tiles, float *tab)
{
    const int MK = a.M * a.K, RG = (a.R + RB - 1) / RB, groups = (MK + 63) / 64;
    const int h = blockIdx.x / groups, lane = lane_id(), i16 = lane & 15, g = lane >> 4;
    const int cw = (blockIdx.x - h * groups) * 64 + (threadIdx.x >> 6) * 16 + i16;
    const float *C = a.C + ((size_t)h * MK + min(cw, MK - 1)) * a.D + 4 * g;
    float4 c[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) c[j] = 16 * j + 4 * g < a.D ? *reinterpret_cast<const float4 *>(C + 16 * j) : make_float4(0.f, 0.f, 0.f, 0.f);
    const int all = a.rows.B * RG * RB;
    const float f = a.factor * kLog2e;
    for (int tile = blockIdx.y; tile < tiles; tile += gridDim.y) {
        const int n = tile * 16 + i16, u = n / RB, b = u / RG, hq = (u - b * RG) * RB + (n - u * RB);
        const bool there = n < all && hq < a.R;
        float4 q[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            q[j] = there && 16 * j + 4 * g < a.D ? T::load(a.Q, (int64_t)b * a.q_row + (int64_t)(h * a.R + hq) * a.q_head + 16 * j + 4 * g) : make_float4(0.f, 0.f, 0.f, 0.f);
        floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(q[j].x, c[j].x, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(q[j].y, c[j].y, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(q[j].z, c[j].z, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(q[j].w, c[j].w, s, 0, 0, 0);
        }
        if (cw >= MK) continue;
#pragma unroll
        for (int e = 0; e < 4; e += RB) {           // queries tile * 16 + 4 g + e of this lane's codeword
            const int m = tile * 16 + 4 * g + e, v = m / RB, bb = v / RG;
            if (m >= all) break;
            float *to = tab + ((((int64_t)bb * a.G + h) * RG + (v - bb * RG)) * MK + cw) * RB;
            if (RB == 4) *reinterpret_cast<float4 *>(to) = make_float4(s[0] * f, s[1] * f, s[2] * f, s[3] * f);
            else if (RB == 2) *reinterpret_cast<float2 *>(to) = make_float2(s[e] * f, s[e + 1] * f);
            else *to = s[e] * f;
        }
    }
}

// The largest of v over the wave, in every lane (NaN are passed over).
__device__ __forceinline__ float wave_max(float v)
{
    auto from = [](float x, auto ctrl, auto rows) {
        return __int_as_float(__builtin_amdgcn_update_dpp((int)0xff800000, __float_as_int(x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
    };
    v = fmaxf(v, from(v, std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>()));   // row_shr:1
    v = fmaxf(v, from(v, std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>()));
    v = fmaxf(v, from(v, std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>()));
    v = fmaxf(v, from(v, std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>()));
    v = fmaxf(v, from(v, std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>()));   // row_bcast:15
    v = fmaxf(v, from(v, std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>()));   // row_bcast:31
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), kWave - 1));
}

struct CodesStat {
    float top, sum, bad, unused;                    // bad: NaN where a value that takes part has no finite scale, else 0
};

template <int RB>
struct Heads {
    float v[RB];
};

// A block a part of the rows of a key head and RB of its query heads.  Windows of 2048 rows, two a thread:
//   scores from the tables in LDS; the largest score and the largest weight |p g'| of the window over the block; weights to fixed point below that weight,
//   added up by code in LDS; these sums, times what the window's fixed point stands for, to the running sums, which threads keep in registers.
// Where two query heads share a word, a weight is in steps of 2^-19 of the window's largest, rounded to the step below or above by a fraction that goes round
// with the row (the golden ratio's multiples), so that many small ones add up to what they are: the error of a sum of n weights is about sqrt(n) / 4
// steps.  bf16 and fp16 outputs have steps of 2^-8 and 2^-11.  float outputs take 64 bits a query head, steps of 2^-40.
template <int RB, bool WIDE, int MW>
__global__ __launch_bounds__(kCodesThreads) void k_attend_codes(const AttendArgs a, int splits, bool grouped, bool words_aligned, const float *tab, CodesStat *stats, float *sums)
{
    extern __shared__ __attribute__((aligned(16))) char codes_lds[];
    __shared__ float red[kCodesWaves][2 * RB];
    __shared__ int any_bad;
    constexpr int P = WIDE ? RB : RB / 2, NW = codes_words(RB, WIDE, MW);
    const int MK = a.M * a.K, K = a.K, RG = (a.R + RB - 1) / RB, H = 2 * a.G, heads = a.G * RG;
    int64_t u;                                      // part of a sequence
    int hr;                                         // key head and group of its query heads
    if (grouped) {                                  // blocks go round the eight XCDs: those that read the same rows to one of them
        const int64_t at = blockIdx.x >> 3;
        u = at / heads * 8 + (blockIdx.x & 7);
        hr = (int)(at % heads);
    } else {
        u = blockIdx.x / heads;
        hr = (int)(blockIdx.x - u * heads);
    }
    if (u >= (int64_t)a.rows.B * splits) return;
    const int b = (int)(u / splits), split = (int)(u - (int64_t)b * splits), h = hr / RG;
    const int64_t seq = (int64_t)b * heads + hr, job = seq * splits + split;
    const SeqRows rows(a, b, h);
    const int64_t per = ((rows.count + splits - 1) / splits + 255) / 256 * 256, first = per * split, last = min(rows.count, first + per);
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    if (first >= last) {
        if (threadIdx.x < RB) stats[job * RB + threadIdx.x] = {-INFINITY, 0.f, 0.f, 0.f};
        return;
    }
    float *lut = reinterpret_cast<float *>(codes_lds);
    unsigned long long *hist = reinterpret_cast<unsigned long long *>(codes_lds + (size_t)MK * RB * 4);
    const int words = MK * P;
    {
        const float *t = tab + seq * MK * RB;
        for (int i = threadIdx.x; i < MK * RB; i += kCodesThreads) lut[i] = t[i];
        for (int i = threadIdx.x; i < words; i += kCodesThreads) hist[i] = 0;
        if (threadIdx.x == 0) any_bad = 0;
    }
    // which pair of query heads a word of this thread's is for, two bits each
    unsigned pairs = 0;
#pragma unroll
    for (int j = 0; j < NW; ++j) pairs |= (unsigned)((threadIdx.x + j * kCodesThreads) / K % P) << (2 * j);
    float acc[NW][WIDE ? 1 : 2] = {};
    Heads<RB> ref, sum;
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        ref.v[r] = -INFINITY;
        sum.v[r] = 0.f;
    }
    bool bad = false;
    __syncthreads();
    for (int64_t w0 = first; w0 < last; w0 += kWindow) {
        bool there[kCodesRows];
        unsigned vc[kCodesRows][MW];
        float gv[kCodesRows], s[kCodesRows][RB], top[RB], most[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) top[r] = most[r] = -INFINITY;
#pragma unroll
        for (int i = 0; i < kCodesRows; ++i) {
            const int64_t t = w0 + i * kCodesThreads + threadIdx.x;
            const int64_t at = t < last ? rows.slot((unsigned)t) : kNoRow;
            there[i] = at >= 0;
            gv[i] = 0.f;
#pragma unroll
            for (int r = 0; r < RB; ++r) s[i][r] = -INFINITY;
            if (at < 0) continue;
            unsigned kc[MW];
            float gk = 1.f;
            auto fetch = [&](unsigned (&c)[MW], const uint8_t *p) {
                if (words_aligned) {
#pragma unroll
                    for (int j = 0; j < MW; ++j) c[j] = 4 * j < a.M ? reinterpret_cast<const unsigned *>(p)[j] : 0u;
                } else {
#pragma unroll
                    for (int j = 0; j < MW; ++j) {
                        c[j] = 0u;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (4 * j + e < a.M) c[j] |= (unsigned)p[4 * j + e] << (8 * e);
                    }
                }
                if (K < 256) {
#pragma unroll
                    for (int j = 0; j < MW; ++j) {
                        unsigned o = 0u;
#pragma unroll
                        for (int e = 0; e < 4; ++e) o |= min(c[j] >> (8 * e) & 255u, (unsigned)K - 1u) << (8 * e);
                        c[j] = o;
                    }
                }
            };
            const uint8_t *row = a.codes + at * (int64_t)(H * a.M);
            fetch(kc, row + h * a.M);
            fetch(vc[i], row + (a.G + h) * a.M);
            if (a.scale) {
                const float *g = a.scale + at * H;
                gk = g[h];
                gv[i] = g[a.G + h];
            } else gv[i] = 1.f;
            bad |= !(fabsf(gv[i]) < INFINITY);
            float x[RB] = {};
#pragma unroll
            for (int m = 0; m < 4 * MW; ++m)
                if (m < a.M) {
                    const unsigned k = kc[m >> 2] >> (8 * (m & 3)) & 255u;
                    const float *e = lut + (m * K + (int)k) * RB;
                    if (RB == 4) {
                        const float4 v = *reinterpret_cast<const float4 *>(e);
                        x[0] += v.x;
                        x[1] += v.y;
                        x[RB - 2] += v.z;
                        x[RB - 1] += v.w;
                    } else if (RB == 2) {
                        const float2 v = *reinterpret_cast<const float2 *>(e);
                        x[0] += v.x;
                        x[RB - 1] += v.y;
                    } else x[0] += *e;
                }
            const float lg = log2f(fabsf(gv[i]));
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                s[i][r] = x[r] * gk;
                top[r] = fmaxf(top[r], s[i][r]);
                most[r] = fmaxf(most[r], s[i][r] + lg);
            }
        }
        // the largest of the window, over the block
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const float x = wave_max(top[r]), y = wave_max(most[r]);
            if (lane == 0) {
                red[wave][2 * r] = x;
                red[wave][2 * r + 1] = y;
            }
        }
        __syncthreads();
        float fade[RB], unit[RB], back[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const float2 v = lane < kCodesWaves ? *reinterpret_cast<const float2 *>(&red[lane][2 * r]) : make_float2(-INFINITY, -INFINITY);
            const float x = wave_max(v.x), y = wave_max(v.y), now = fmaxf(ref.v[r], x);
            fade[r] = ref.v[r] == -INFINITY ? 0.f : exp2f(ref.v[r] - now);
            ref.v[r] = now;
            // weights below 2^e; none or only zeros: any step
            const float e = y == -INFINITY ? 0.f : ceilf(y - now + 0.01f);
            const int n = (WIDE ? kWideBits : kPairBits) - (int)fminf(fmaxf(e, -80.f), 140.f);
            unit[r] = ldexpf(1.f, n > 120 ? 120 : n);
            back[r] = ldexpf(1.f, -(n > 120 ? 120 : n));
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) sum.v[r] *= fade[r];
#pragma unroll
        for (int i = 0; i < kCodesRows; ++i) {
            if (!there[i]) continue;
            const float turn = (float)(((unsigned)(w0 + i * kCodesThreads + threadIdx.x) * 0x9E3779B9u) >> 8) * 0x1p-24f;
            unsigned long long add[P];
            long long fixed[RB];
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const float p = exp2f(s[i][r] - ref.v[r]);
                sum.v[r] += p;
                const float w = p * gv[i];
                if (WIDE) {
                    const double d = (double)w * (double)unit[r];
                    fixed[r] = d == d ? (long long)rint(d) : 0;
                } else fixed[r] = (int)floorf(w * unit[r] + turn);
            }
#pragma unroll
            for (int q = 0; q < P; ++q)
                add[q] = WIDE ? (unsigned long long)fixed[q] : ((unsigned long long)fixed[(2 * q + 1) % RB] << 32) + (unsigned long long)fixed[(2 * q) % RB];
#pragma unroll
            for (int m = 0; m < 4 * MW; ++m)
                if (m < a.M) {
                    const unsigned k = vc[i][m >> 2] >> (8 * (m & 3)) & 255u;
#pragma unroll
                    for (int q = 0; q < P; ++q)
                        __hip_atomic_fetch_add(hist + (m * P + q) * K + (int)k, add[q], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NW; ++j) {
            const int i = threadIdx.x + j * kCodesThreads, q = pairs >> (2 * j) & 3;
            if (i >= words) break;
            const unsigned long long v = hist[i];
            hist[i] = 0;
            if (WIDE) {
                float f = fade[0], o = back[0];
#pragma unroll
                for (int r = 1; r < RB; ++r)
                    if (q == r) {
                        f = fade[r];
                        o = back[r];
                    }
                acc[j][0] = acc[j][0] * f + (float)((double)(long long)v * (double)o);
            } else {
                const int lo = (int)(unsigned)v, hi = (int)(unsigned)((v - (unsigned long long)(long long)lo) >> 32);
                const bool second = RB == 4 && q == 1;
                acc[j][0] = acc[j][0] * (second ? fade[RB == 4 ? 2 : 0] : fade[0]) + (float)lo * (second ? back[RB == 4 ? 2 : 0] : back[0]);
                acc[j][WIDE ? 0 : 1] = acc[j][WIDE ? 0 : 1] * (second ? fade[RB - 1] : fade[RB >= 2 ? 1 : 0]) + (float)hi * (second ? back[RB - 1] : back[RB >= 2 ? 1 : 0]);
            }
        }
    }
    if (bad) any_bad = 1;                           // the same value from whoever writes
    __syncthreads();
    // the exponentials' sums, in a fixed order
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        float x = sum.v[r];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
        if (lane == 0) red[wave][r] = x;
    }
    __syncthreads();
    if (threadIdx.x < RB) {
        float x = 0.f, t = 0.f;
        for (int w = 0; w < kCodesWaves; ++w) x += red[w][threadIdx.x];
#pragma unroll
        for (int r = 0; r < RB; ++r)
            if ((int)threadIdx.x == r) t = ref.v[r];
        stats[job * RB + threadIdx.x] = {t, x, any_bad ? NAN : 0.f, 0.f};
    }
    const int64_t row = sums_row(a.M, K);
    float *to = sums + job * RB * row;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
        const int i = threadIdx.x + j * kCodesThreads, q = pairs >> (2 * j) & 3;
        if (i >= words) break;
        const int e = i / K, mk = e / P * K + (i - e * K);
        if (WIDE) to[q * row + mk] = acc[j][0];
        else {
            to[2 * q * row + mk] = acc[j][0];
            to[(2 * q + 1) * row + mk] = acc[j][WIDE ? 0 : 1];
        }
    }
    if (threadIdx.x < RB * (int)(row - MK)) to[threadIdx.x / (int)(row - MK) * row + MK + threadIdx.x % (int)(row - MK)] = 0.f;
}

constexpr int kOutThreads = 512, kOutWaves = kOutThreads / kWave;

// out = sum over the parts and codewords of the sums by code, times the codewords, over the exponentials' sum: a block 16 query heads and 16 coordinates, its waves
// a share of the codewords each, on the fp32 matrix cores.
template <typename T, int RB>
__global__ __launch_bounds__(kOutThreads) void k_attend_out(const AttendArgs a, int splits, int tiles, const CodesStat *stats, const float *sums)
{
    __shared__ float part[16][kCodesSplits], out[kOutWaves][16][17];
    const int RG = (a.R + RB - 1) / RB, MK = a.M * a.K, slices = (a.D + 15) / 16, all = a.rows.B * RG * RB;
    const int at = blockIdx.x >> 3, th = at / slices * 8 + (blockIdx.x & 7), slice = at % slices;    // slices of a tile on one XCD
    if (th >= tiles * a.G) return;
    const int tile = th / a.G, h = th - tile * a.G, lane = lane_id(), wave = threadIdx.x >> 6, i16 = lane & 15, g = lane >> 4;
    auto job_of = [&](int n) {                      // its first part
        const int u = n / RB, b = u / RG;
        return (((int64_t)b * a.G + h) * RG + (u - b * RG)) * splits;
    };
    // what a part counts: four lanes... one thread a query head
    if (threadIdx.x < 16) {
        const int n = tile * 16 + (int)threadIdx.x, u = n / RB, b = u / RG, hq = (u - b * RG) * RB + n % RB;
        const bool there = n < all && hq < a.R;
        const CodesStat *st = there ? stats + job_of(n) * RB + n % RB : stats;
        float top = -INFINITY, sum = 0.f, bad = 0.f;
        if (there) {
            for (int i = 0; i < splits; ++i) top = fmaxf(top, st[(int64_t)i * RB].top);
            for (int i = 0; i < splits; ++i) {
                const CodesStat x = st[(int64_t)i * RB];
                bad += x.bad;
                float f = 0.f;
                if (x.sum != 0.f) {
                    f = exp2f(x.top - top);
                    sum += f * x.sum;
                }
                part[threadIdx.x][i] = f;
            }
        } else
            for (int i = 0; i < splits; ++i) part[threadIdx.x][i] = 0.f;
        if (sum != 0.f)
            for (int i = 0; i < splits; ++i) part[threadIdx.x][i] = part[threadIdx.x][i] / sum + bad;
        if (there && slice == 0 && a.lse) a.lse[(int64_t)b * a.G * a.R + h * a.R + hq] = sum != 0.f ? (top + log2f(sum)) * kLn2 : -INFINITY;
    }
    __syncthreads();
    const int n = tile * 16 + i16, d = slice * 16 + i16;
    const int64_t row = sums_row(a.M, a.K);
    const float *W = sums + (n < all ? job_of(n) * RB + n % RB : 0) * row + 4 * g;
    const float *C = a.C + (size_t)(a.G + h) * MK * a.D + min(d, a.D - 1);
    floatx4 s = {0.f, 0.f, 0.f, 0.f};
    for (int j = 16 * wave; j < MK; j += 16 * kOutWaves) {
        float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
        if (j + 4 * g < MK)
            for (int i = 0; i < splits; ++i) {
                const float f = part[i16][i];
                if (f == 0.f) continue;             // a part without rows has no sums
                const float4 v = *reinterpret_cast<const float4 *>(W + (int64_t)i * RB * row + j);
                w = make_float4(w.x + f * v.x, w.y + f * v.y, w.z + f * v.z, w.w + f * v.w);
            }
        float c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = C[(size_t)min(j + 4 * g + e, MK - 1) * a.D];
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(w.x, c[0], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(w.y, c[1], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(w.z, c[2], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(w.w, c[3], s, 0, 0, 0);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) out[wave][4 * g + e][i16] = s[e];
    __syncthreads();
    if (threadIdx.x < 64) {
        const int i = threadIdx.x >> 2, p = threadIdx.x & 3, m = tile * 16 + i, u = m / RB, b = u / RG, hq = (u - b * RG) * RB + m % RB;
        if (m < all && hq < a.R && slice * 16 + 4 * p < a.D) {
            float v[4] = {};
            for (int w = 0; w < kOutWaves; ++w)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += out[w][i][4 * p + e];
            T::store(a.out, (int64_t)b * a.o_row + (int64_t)(h * a.R + hq) * a.o_head + slice * 16 + 4 * p, make_float4(v[0], v[1], v[2], v[3]));
        }
    }
}

}  // namespace hclae
