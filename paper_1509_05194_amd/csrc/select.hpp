// The pages of a sequence whose stand-ins score highest against its new token's queries (hclae_cache_select):
//   score(b, h, j) = scale[p][h] * sum_m t[m][codes[p][h][m]],  t[m][k] = (sum over the R queries of the head) . C[h][m][k],  p = tables[b][j]
// in 64 bits throughout: which of two pages is better is a decision.
//   k_select_tables   t of every sequence and head, for all codewords once: from then on a page costs M additions whatever D is
//   k_select_pages    scores as sortable whole numbers, the k-th largest by digits, the pages above it in order
#pragma once
#include "../../include/hclae.h"
#include "decode.hpp"
#include "serve.hpp"

namespace hclae {

constexpr int kSelectThreads = 256, kSelectSeqs = 8, kPickThreads = 1024;

// A block a dictionary of a head and eight sequences, a thread a codeword; codewords in pieces of four coordinates, so that neighbouring
// threads read neighbouring bytes.
template <typename T>
__global__ __launch_bounds__(kSelectThreads) void k_select_tables(const SelectArgs a, double *tab)
{
    __shared__ double q[kSelectSeqs][HCLAE_CACHE_MAX_D];
    const int hm = blockIdx.x, h = hm / a.M, b0 = blockIdx.y * kSelectSeqs, n = min(kSelectSeqs, a.rows.B - b0), d4 = a.D >> 2;
    for (int i = threadIdx.x; i < n * d4; i += kSelectThreads) {
        const int j = i / d4, p = i - j * d4;
        double s[4] = {};
        for (int r = 0; r < a.R; ++r) {
            const float4 v = T::load(a.Q, (int64_t)(b0 + j) * a.q_row + (int64_t)(h * a.R + r) * a.q_head + 4 * p);
            s[0] += v.x;
            s[1] += v.y;
            s[2] += v.z;
            s[3] += v.w;
        }
        for (int e = 0; e < 4; ++e) q[j][4 * p + e] = s[e];
    }
    __syncthreads();
    const int k = threadIdx.x;
    if (k >= a.K) return;
    const float4 *C = a.T + (size_t)hm * a.pieces * a.columns + k;
    double s[kSelectSeqs] = {};
    for (int p = 0; p < d4; ++p) {
        const float4 c = C[(size_t)p * a.columns];
#pragma unroll
        for (int j = 0; j < kSelectSeqs; ++j) {
            s[j] = fma(q[j][4 * p], (double)c.x, s[j]);
            s[j] = fma(q[j][4 * p + 1], (double)c.y, s[j]);
            s[j] = fma(q[j][4 * p + 2], (double)c.z, s[j]);
            s[j] = fma(q[j][4 * p + 3], (double)c.w, s[j]);
        }
    }
    for (int j = 0; j < n; ++j) tab[(((int64_t)(b0 + j) * a.G * a.M) + hm) * a.K + k] = s[j];
}

// Greater numbers are greater keys; a NaN is the least number, 0 is no page, and all ones a page that is taken whatever its score.
__host__ __device__ inline uint64_t score_key(double x)
{
    if (x != x) x = -__builtin_inf();
    x += 0.0;                                       // both zeros are one
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return u >> 63 ? ~u : u | 1ull << 63;
}

// A block a sequence and head.  IN_LDS: the tables and keys fit there.
template <bool IN_LDS>
__global__ __launch_bounds__(kPickThreads) void k_select_pages(const SelectArgs a, const double *tab, uint64_t *key_room)
{
    extern __shared__ __attribute__((aligned(16))) char select_lds[];
    __shared__ unsigned hist[256], counts[2][17];
    __shared__ uint64_t s_prefix;
    __shared__ unsigned s_need, s_all;
    const int job = blockIdx.x, b = job / a.G, h = job - b * a.G, lane = lane_id(), wave = threadIdx.x >> 6;
    const int64_t length = a.rows.lengths[b];
    const int64_t most = length <= 0 ? 0 : (length + a.rows.page - 1) / a.rows.page;
    const int P = (int)(most < a.rows.max_pages ? most : a.rows.max_pages);
    const int32_t *table = a.rows.tables + (int64_t)b * a.rows.max_pages;
    const double *t = tab + (int64_t)job * a.M * a.K;
    uint64_t *keys = key_room + (int64_t)job * a.rows.max_pages;
    if (IN_LDS) {
        double *to = reinterpret_cast<double *>(select_lds);
        for (int i = threadIdx.x; i < a.M * a.K; i += kPickThreads) to[i] = t[i];
        t = to;
        keys = reinterpret_cast<uint64_t *>(to + a.M * a.K);
    }
    if (threadIdx.x == 0) s_all = 0;
    __syncthreads();
    unsigned there = 0;
    for (int j = threadIdx.x; j < P; j += kPickThreads) {
        const int32_t p = table[j];
        uint64_t key = 0;
        if (p >= 0 && p < a.rows.pages) {
            if (j < a.first || j >= P - a.recent) key = ~0ull;
            else {
                const int64_t row = (int64_t)p * a.G + h;
                const uint8_t *code = a.codes + row * a.M;
                double x = 0.0;
                for (int m = 0; m < a.M; ++m) x += t[m * a.K + min((int)code[m], a.K - 1)];
                key = score_key(a.scale ? x * (double)a.scale[row] : x);
            }
            ++there;
        }
        keys[j] = key;
    }
    if (there) atomicAdd(&s_all, there);
    __syncthreads();
    // the k-th largest key, a digit at a time: keys whose leading digits are `prefix` are undecided, those above it are taken
    uint64_t prefix = 0, mask = 0;
    unsigned need = (unsigned)a.k;
    if (s_all <= need) need = s_all;                // all there are
    else
        for (int shift = 56; shift >= 0; shift -= 8) {
            if (threadIdx.x < 256) hist[threadIdx.x] = 0;
            __syncthreads();
            for (int j = threadIdx.x; j < P; j += kPickThreads) {
                const uint64_t key = keys[j];
                if (key && (key & mask) == prefix) atomicAdd(&hist[(key >> shift) & 255], 1u);
            }
            __syncthreads();
            if (wave == 0) {                        // lane i: digits 255 - 4 i down to 252 - 4 i
                unsigned c[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += c[i] = hist[255 - 4 * lane - i];
                unsigned upto = sum;
#pragma unroll
                for (int o = 1; o < kWave; o <<= 1) {
                    const unsigned y = __shfl_up(upto, o, kWave);
                    if (lane >= o) upto += y;
                }
                unsigned above = upto - sum;
                if (above < need && upto >= need) {
                    for (int i = 0; i < 4; ++i) {
                        if (above + c[i] >= need) {
                            s_prefix = prefix | (uint64_t)(255 - 4 * lane - i) << shift;
                            s_need = need - above;
                            s_all = c[i];
                            break;
                        }
                        above += c[i];
                    }
                }
            }
            __syncthreads();
            prefix = s_prefix;
            mask |= 255ull << shift;
            need = s_need;
            if (s_all == need) break;               // all the undecided are taken
        }
    // in the order of the pages; of equal keys the first
    int32_t *out = a.picked + (int64_t)job * a.k;
    unsigned taken = 0, equal = 0;
    for (int j0 = 0; j0 < P; j0 += kPickThreads) {
        const int j = j0 + (int)threadIdx.x;
        const uint64_t key = j < P ? keys[j] : 0, lead = key & mask;
        const bool above = key && lead > prefix, same = key && lead == prefix;
        const unsigned long long eq = __ballot(same);
        if (lane == 0) counts[0][wave] = __popcll(eq);
        __syncthreads();
        unsigned rank = equal + __popcll(eq & ((1ull << lane) - 1ull));
        for (int w = 0; w < kPickThreads / kWave; ++w) {
            if (w < wave) rank += counts[0][w];
            equal += counts[0][w];
        }
        const bool take = above || (same && rank < need);
        const unsigned long long sel = __ballot(take);
        if (lane == 0) counts[1][wave] = __popcll(sel);
        __syncthreads();
        unsigned at = taken + __popcll(sel & ((1ull << lane) - 1ull));
        for (int w = 0; w < kPickThreads / kWave; ++w) {
            if (w < wave) at += counts[1][w];
            taken += counts[1][w];
        }
        if (take && at < (unsigned)a.k) out[at] = j;
        __syncthreads();
    }
    for (int i = (int)taken + (int)threadIdx.x; i < a.k; i += kPickThreads) out[i] = -1;
}

}  // namespace hclae
