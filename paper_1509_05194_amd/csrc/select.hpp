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

constexpr int kSelectThreads = 256, kSelectSeqs = 16, kPickThreads = 1024, kPickWaves = kPickThreads / kWave;

typedef double doublex4 __attribute__((ext_vector_type(4)));

// t on the fp64 matrix cores, a wave 16 codewords of a head and 16 sequences.  The 4 x 4 blocks of an instruction take coordinates 16 j + 4 g + e, g the
// quarter of the wave: a lane so loads four of its codeword side by side; the queries' sums come through LDS.  Of the result a lane holds codewords
// g, 4 + g, 8 + g and 12 + g of one sequence.  8 key heads, D = 128, M = 8, K = 256: 5.8 us for one sequence, 9.8 for 32 (134 M products; a codeword a thread, eight
// sequences at a time: 12.4 and 17).
template <typename T>
__global__ __launch_bounds__(kSelectThreads) void k_select_tables(const SelectArgs a, double *tab)
{
    constexpr int PITCH = HCLAE_CACHE_MAX_D + 2;
    __shared__ __attribute__((aligned(16))) double q[kSelectSeqs][PITCH];
    const int MK = a.M * a.K, groups = (MK + 63) / 64, h = blockIdx.x / groups % a.G, b0 = blockIdx.x / groups / a.G * kSelectSeqs, n = min(kSelectSeqs, a.rows.B - b0), d4 = a.D >> 2;
    const int lane = lane_id(), i16 = lane & 15, g = lane >> 4, d16 = (a.D + 15) / 16 * 16;
    const int first = blockIdx.x % groups * 64 + (threadIdx.x >> 6) * 16;
    const float *C = a.C + ((size_t)h * MK + min(first + i16, MK - 1)) * a.D;
    constexpr int AHEAD = 4;
    float4 c[AHEAD];
    auto load = [&](int j) { return 16 * j + 4 * g < a.D ? *reinterpret_cast<const float4 *>(C + 16 * j + 4 * g) : make_float4(0.f, 0.f, 0.f, 0.f); };
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) c[j] = load(j);
    for (int i = threadIdx.x; i < kSelectSeqs * d16 / 4; i += kSelectThreads) {
        const int s = i / (d16 / 4), p = i - s * (d16 / 4);
        double x[4] = {};
        if (s < n && p < d4)
            for (int r = 0; r < a.R; ++r) {
                const float4 v = T::load(a.Q, (int64_t)(b0 + s) * a.q_row + (int64_t)(h * a.R + r) * a.q_head + 4 * p);
                x[0] += v.x;
                x[1] += v.y;
                x[2] += v.z;
                x[3] += v.w;
            }
#pragma unroll
        for (int e = 0; e < 4; ++e) q[s][4 * p + e] = x[e];
    }
    __syncthreads();
    doublex4 s = {0., 0., 0., 0.};
    for (int j0 = 0; 16 * j0 < a.D; j0 += AHEAD)
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (16 * (j0 + j) >= a.D) break;
            const float4 v = c[j];
            c[j] = load(j0 + j + AHEAD);
            const double2 lo = *reinterpret_cast<const double2 *>(&q[i16][16 * (j0 + j) + 4 * g]), hi = *reinterpret_cast<const double2 *>(&q[i16][16 * (j0 + j) + 4 * g + 2]);
            s = __builtin_amdgcn_mfma_f64_16x16x4f64((double)v.x, lo.x, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f64_16x16x4f64((double)v.y, lo.y, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f64_16x16x4f64((double)v.z, hi.x, s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f64_16x16x4f64((double)v.w, hi.y, s, 0, 0, 0);
        }
    if (i16 < n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int cw = first + 4 * e + g;
            if (cw < MK) tab[((int64_t)(b0 + i16) * a.G + h) * MK + cw] = s[e];
        }
}

// Greater numbers are greater keys; a NaN is the least number, 0 is no page, and all ones a page that is taken whatever its score.
__host__ __device__ inline uint64_t score_key(double x)
{
    if (x != x) x = -__builtin_inf();
    x += 0.0;                                       // both zeros are one
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return u >> 63 ? ~u : u | 1ull << 63;
}

constexpr int kDigitBits = 12, kDigits = 1 << kDigitBits, kFew = 64;

__host__ __device__ constexpr size_t pick_lds(int M, int K, int max_pages) { return 8 * ((size_t)M * K + max_pages); }

// A block a sequence and head.  IN_LDS: the tables and keys fit there.  The k-th largest key is found by digits of 12 bits (scores of one query differ in
// their exponents and a few bits more: two digits leave a handful), the last 64 undecided are ranked one against all.  Eight lists of 125 pages 10 us, 256
// lists of 1024 to 2048 pages 24 us, 8 of it codes and scales that lie anywhere, 3 the first digit's counts (few exponents: many lanes at one word), 3 a second digit, 2 the
// order of the pages.  Digits of 8 bits took 20 us with less spread scores and five rounds; ranking up to 256 undecided through LDS took 37.
template <bool IN_LDS>
__global__ __launch_bounds__(kPickThreads) void k_select_pages(const SelectArgs a, const double *tab, uint64_t *key_room)
{
    extern __shared__ __attribute__((aligned(16))) char select_lds[];
    __shared__ unsigned hist[kDigits], sums[kPickWaves], taken_before[kPickWaves];
    __shared__ uint64_t few[kFew], s_prefix;
    __shared__ int few_at[kFew];
    __shared__ unsigned s_need, s_left, s_count;
    const int job = blockIdx.x, b = job / a.G, h = job - b * a.G, lane = lane_id(), wave = threadIdx.x >> 6;
    const int64_t length = a.rows.lengths[b];
    const int64_t most = length <= 0 ? 0 : (length + a.rows.page - 1) / a.rows.page;
    const int P = (int)(most < a.rows.max_pages ? most : a.rows.max_pages);
    const int32_t *table = a.rows.tables + (int64_t)b * a.rows.max_pages;
    const double *t = tab + (int64_t)job * a.M * a.K;
    uint64_t *keys = key_room + (int64_t)job * a.rows.max_pages;
    if (IN_LDS) {
        double2 *to = reinterpret_cast<double2 *>(select_lds);
        const double2 *from = reinterpret_cast<const double2 *>(t);
        const int n = a.M * a.K;
        if (n % 2 == 0) {                           // every job's tables begin at whole pairs
            for (int i = threadIdx.x; i < n / 2; i += kPickThreads) to[i] = from[i];
        } else
            for (int i = threadIdx.x; i < n; i += kPickThreads) reinterpret_cast<double *>(select_lds)[i] = t[i];
        t = reinterpret_cast<const double *>(select_lds);
        keys = reinterpret_cast<uint64_t *>(select_lds) + n;
    }
    for (int i = threadIdx.x; i < kDigits; i += kPickThreads) hist[i] = 0;
    if (threadIdx.x == 0) s_left = s_count = 0;
    __syncthreads();
    const bool words = a.M % 4 == 0 && reinterpret_cast<uintptr_t>(a.codes) % 4 == 0;
    unsigned there = 0;
    constexpr int U = 4;                            // pages of a thread whose codes are sent for at once
    for (int j0 = threadIdx.x; j0 < P; j0 += U * kPickThreads) {
        int32_t p[U];
#pragma unroll
        for (int i = 0; i < U; ++i) p[i] = j0 + i * kPickThreads < P ? table[j0 + i * kPickThreads] : -1;
        unsigned w[U][2];
        float g[U];
        bool read[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int j = j0 + i * kPickThreads;
            read[i] = p[i] >= 0 && p[i] < a.rows.pages && j >= a.first && j < P - a.recent;
            w[i][0] = w[i][1] = 0u;
            g[i] = 1.f;
            if (!read[i]) continue;
            const int64_t row = (int64_t)p[i] * a.G + h;
            if (words) {
                const unsigned *code = reinterpret_cast<const unsigned *>(a.codes + row * a.M);
                w[i][0] = code[0];
                if (a.M > 4) w[i][1] = code[1];
            }
            if (a.scale) g[i] = a.scale[row];
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int j = j0 + i * kPickThreads;
            if (j >= P) break;
            uint64_t key = 0;
            if (p[i] >= 0 && p[i] < a.rows.pages) {
                key = ~0ull;
                if (read[i]) {
                    const uint8_t *code = a.codes + ((int64_t)p[i] * a.G + h) * a.M;
                    double x = 0.0;
                    if (words) {
#pragma unroll
                        for (int m = 0; m < 8; ++m)
                            if (m < a.M) x += t[m * a.K + min((int)(w[i][m >> 2] >> (8 * (m & 3)) & 255u), a.K - 1)];
                        for (int m0 = 8; m0 < a.M; m0 += 4) {
                            const unsigned c = *reinterpret_cast<const unsigned *>(code + m0);
#pragma unroll
                            for (int m = 0; m < 4; ++m) x += t[(m0 + m) * a.K + min((int)(c >> (8 * m) & 255u), a.K - 1)];
                        }
                    } else
                        for (int m = 0; m < a.M; ++m) x += t[m * a.K + min((int)code[m], a.K - 1)];
                    key = score_key(a.scale ? x * (double)g[i] : x);
                }
                ++there;
                atomicAdd(&hist[key >> (64 - kDigitBits)], 1u);
            }
            keys[j] = key;
        }
    }
    if (there) atomicAdd(&s_left, there);
    __syncthreads();
    // keys whose leading digits are `prefix` are undecided, those above it are taken
    uint64_t prefix = 0, mask = 0;
    unsigned need = (unsigned)a.k, left = s_left;
    bool ranked = false;
    if (left <= need) need = left;                  // all there are
    else
        for (int shift = 64 - kDigitBits;; shift -= kDigitBits) {
            const int low = shift < 0 ? 0 : shift;
            if (mask) {
                for (int i = threadIdx.x; i < kDigits; i += kPickThreads) hist[i] = 0;
                __syncthreads();
                for (int j = threadIdx.x; j < P; j += kPickThreads) {
                    const uint64_t key = keys[j];
                    if (key && (key & mask) == prefix) atomicAdd(&hist[(unsigned)(key >> low) & (kDigits - 1) & (unsigned)(~mask >> low)], 1u);
                }
                __syncthreads();
            }
            // thread i: digits 4095 - 4 i down to 4092 - 4 i
            unsigned c[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += c[i] = hist[kDigits - 1 - 4 * threadIdx.x - i];
            unsigned upto = sum;
#pragma unroll
            for (int o = 1; o < kWave; o <<= 1) {
                const unsigned y = __shfl_up(upto, o, kWave);
                if (lane >= o) upto += y;
            }
            if (lane == kWave - 1) sums[wave] = upto;
            __syncthreads();
            unsigned above = upto - sum;
            for (int w = 0; w < wave; ++w) above += sums[w];
            if (above < need && above + sum >= need) {
                for (int i = 0; i < 4; ++i) {
                    if (above + c[i] >= need) {
                        s_prefix = prefix | (uint64_t)(kDigits - 1 - 4 * threadIdx.x - i) << low;
                        s_need = need - above;
                        s_left = c[i];
                        break;
                    }
                    above += c[i];
                }
            }
            __syncthreads();
            prefix = s_prefix;
            need = s_need;
            left = s_left;
            mask |= (uint64_t)(kDigits - 1) << low;
            if (left == need || low == 0) break;    // all the undecided are taken, or equal
            if (left <= kFew) {
                ranked = true;
                break;
            }
        }
    if (ranked) {                                   // of the undecided those which fewer than `need` are ahead of
        for (int j = threadIdx.x; j < P; j += kPickThreads) {
            const uint64_t key = keys[j];
            if (key && (key & mask) == prefix) {
                const unsigned i = atomicAdd(&s_count, 1u);
                few[i] = key;
                few_at[i] = j;
            }
        }
        __syncthreads();
        static_assert(kFew <= kWave, "one wave ranks them");
        if (wave == 0) {
            const uint64_t key = few[lane];
            const int at = few_at[lane];
            unsigned ahead = 0;
            for (int i = 0; i < (int)left; ++i) {
                const unsigned hi = __builtin_amdgcn_readlane((int)(key >> 32), i), lo = __builtin_amdgcn_readlane((int)key, i);
                const uint64_t other = (uint64_t)hi << 32 | lo;
                ahead += other > key || (other == key && __builtin_amdgcn_readlane(at, i) < at) ? 1u : 0u;
            }
            // taken, or not; where infinite scores share the prefix of pages that are taken whatever theirs, these `need` keys are all that have it
            if (lane < (int)left) keys[at] = ahead < need ? ~0ull : 0ull;
        }
        __syncthreads();
    }
    // in the order of the pages; of equal keys the first
    int32_t *out = a.picked + (int64_t)job * a.k;
    unsigned taken = 0, equal = 0;
    for (int j0 = 0; j0 < P; j0 += kPickThreads) {
        const int j = j0 + (int)threadIdx.x;
        const uint64_t key = j < P ? keys[j] : 0, lead = key & mask;
        const bool above = key && lead > prefix, same = key && lead == prefix && need > 0;
        const unsigned long long eq = __ballot(same);
        if (lane == 0) sums[wave] = __popcll(eq);
        __syncthreads();
        unsigned rank = equal + __popcll(eq & ((1ull << lane) - 1ull));
        for (int w = 0; w < kPickWaves; ++w) {
            if (w < wave) rank += sums[w];
            equal += sums[w];
        }
        const bool take = above || (same && rank < need);
        const unsigned long long sel = __ballot(take);
        if (lane == 0) taken_before[wave] = __popcll(sel);
        __syncthreads();
        unsigned at = taken + __popcll(sel & ((1ull << lane) - 1ull));
        for (int w = 0; w < kPickWaves; ++w) {
            if (w < wave) at += taken_before[w];
            taken += taken_before[w];
        }
        if (take && at < (unsigned)a.k) out[at] = j;
    }
    for (int i = (int)taken + (int)threadIdx.x; i < a.k; i += kPickThreads) out[i] = -1;
}

}  // namespace hclae
