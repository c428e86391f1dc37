// Attention of one new token of every sequence over its rows of a coded cache (hclae_cache_attend).
//   s_t = factor g_t q . (sum_m C[h][m][k_m(t)]),  p = softmax(s),  out = sum_t p_t g'_t sum_m C[G + h][m][v_m(t)]
// Scores are kept times log2(e) and exponentials taken to the base 2; softmax statistics, weights and sums are in 32 bits or more.
//   k_attend_rows, k_attend_join   rows decoded as they are needed: any shape
#pragma once
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

}  // namespace hclae
