// Quantising the rows of a cache as they are written (hclae_cache_write): rows of H heads, each head with M dictionaries of its
// own, into slots of a paged cache.  Per row x and head
//   g = max |x|,  u = x / g  (u = x where no scales are kept),  r = u;
//   for m = 0..M-1:  i_m = argmin_k ||r - c_m(k)||^2 (the direct form in 64 bits, the lowest index of equals),  r = r - c_m(i_m) in 32 bits,
// which is the greedy encoding of Eq. 3 with one path on a row brought to a largest magnitude of one.
#pragma once
#include "assign_half.hpp"
#include "decode.hpp"
#include "encode.hpp"
#include "encode_wave.hpp"

namespace hclae {

constexpr int kCacheMaxD = 256;
constexpr int kFewThreads = 1024;

// Codewords that a block's threads cover side by side: 64, 128 or 256.
__host__ __device__ constexpr int few_columns(int K) { return K <= 64 ? 64 : K <= 128 ? 128 : 256; }

struct CacheRowsIn {
    const void *X;
    int type;
    int64_t row_stride, head_stride;                // elements
    const int64_t *slots;
    int64_t n, n_slots;
    uint8_t *codes;                                 // [n_slots][H][M]
    float *scale;                                   // [n_slots][H] or null
    int H, M, K, D;
};

__device__ __forceinline__ float4 load_in(const CacheRowsIn &a, int64_t at)
{
    return a.type == kRowF32 ? F32::load(a.X, at) : a.type == kRowF16 ? F16::load(a.X, at) : Bf16::load(a.X, at);
}

// The dictionaries as k_cache_write_one and k_cache_write_some read them: T[dictionary][piece of four coordinates][codeword], so that neighbouring lanes
// read neighbouring codewords, padded with zeros to `pieces`; and a copy as they are.  A block per dictionary and 16 pieces.
__global__ __launch_bounds__(256) void k_cache_lay(const float *__restrict__ C, int K, int D, int columns, int pieces, float *__restrict__ copy, float4 *__restrict__ T)
{
    const int d4 = D >> 2;
    const float4 *from = reinterpret_cast<const float4 *>(C + (size_t)blockIdx.x * K * D);
    float4 *to = T + (size_t)blockIdx.x * pieces * columns;
    float4 *same = reinterpret_cast<float4 *>(copy + (size_t)blockIdx.x * K * D);
    __shared__ float4 tile[16][17];
    const int i = threadIdx.x & 15, j = threadIdx.x >> 4;
    const int p0 = 16 * blockIdx.y;
    for (int k0 = 0; k0 < columns; k0 += 16) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k0 + j < K && p0 + i < d4) {
            v = from[(size_t)(k0 + j) * d4 + p0 + i];
            same[(size_t)(k0 + j) * d4 + p0 + i] = v;
        }
        tile[i][j] = v;
        __syncthreads();
        to[(size_t)(p0 + j) * columns + k0 + i] = tile[j][i];
        __syncthreads();
    }
}

typedef float floatv4 __attribute__((ext_vector_type(4)));

template <int CTRL>
__device__ __forceinline__ float dpp_plus(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// The sum over the sixteen lanes of a row, the same in all of them.
__device__ __forceinline__ float sum16(float v)
{
    return dpp_plus<0x140>(dpp_plus<0x141>(dpp_plus<0x4E>(dpp_plus<0xB1>(v))));     // quad_perm 1 0 3 2, 2 3 0 1, row_half_mirror, row_mirror
}

// The least of 64 numbers that order as unsigned integers, the same in every lane (see wave_max_int).
__device__ __forceinline__ unsigned wave_min_bits(unsigned v)
{
    v = min(v, (unsigned)__builtin_amdgcn_update_dpp(-1, (int)v, 0x111, 0xf, 0xf, false));   // row_shr:1
    v = min(v, (unsigned)__builtin_amdgcn_update_dpp(-1, (int)v, 0x112, 0xf, 0xf, false));   // row_shr:2
    v = min(v, (unsigned)__builtin_amdgcn_update_dpp(-1, (int)v, 0x114, 0xf, 0xf, false));   // row_shr:4
    v = min(v, (unsigned)__builtin_amdgcn_update_dpp(-1, (int)v, 0x118, 0xf, 0xf, false));   // row_shr:8
    v = min(v, (unsigned)__builtin_amdgcn_update_dpp(-1, (int)v, 0x142, 0xa, 0xf, false));   // row_bcast:15
    v = min(v, (unsigned)__builtin_amdgcn_update_dpp(-1, (int)v, 0x143, 0xc, 0xf, false));   // row_bcast:31
    return (unsigned)__builtin_amdgcn_readlane((int)v, kWave - 1);
}

// One row of the input into LDS, by a wave: divided by its largest magnitude where scales are kept, zero beyond D up to `padded`.
__device__ __forceinline__ int64_t take_row(const CacheRowsIn &a, int64_t n, int h, float4 *row, int padded, int lane)
{
    const int64_t s = n < a.n ? a.slots[n] : -1;
    const bool live = s >= 0 && s < a.n_slots;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (live && 4 * lane < a.D) v = load_in(a, n * a.row_stride + h * a.head_stride + 4 * lane);
    // magnitudes order as integers do, NaN above infinity
    int top = max(max(__float_as_int(fabsf(v.x)), __float_as_int(fabsf(v.y))), max(__float_as_int(fabsf(v.z)), __float_as_int(fabsf(v.w))));
    top = wave_max_int(top);
    float g = __int_as_float(top);
    if (top >= 0x7f800000) {                        // not a number: kept as a row of zeros whose scale says so
        v = make_float4(0.f, 0.f, 0.f, 0.f);
        g = __builtin_nanf("");
    } else if (a.scale && top) {
        v = make_float4(v.x / g, v.y / g, v.z / g, v.w / g);
    }
    if (4 * lane < padded) row[lane] = v;
    if (lane == 0 && live && a.scale) a.scale[s * a.H + h] = g;
    return live ? s : -1;
}

// A row or few in all: a block takes one row of one head through all dictionaries.  Every thread keeps a share of one codeword (its
// pieces q, q + Q, ...) in registers, the next dictionary's on their way meanwhile; the row is in LDS, where all lanes read the
// same piece.  The threads that hold the chosen codeword subtract it: no gather, a dictionary is read once.
// A dictionary takes about 2 us: its share from L2, three barriers and the reductions between them, one after another (16 rows, D = 128,
// M = 8, K = 256: 21 us, of which 4 are the call's).
template <int COLS, int P>
__global__ __launch_bounds__(kFewThreads) void k_cache_write_one(const CacheRowsIn a, const float4 *__restrict__ T)
{
    constexpr int Q = kFewThreads / COLS;           // threads that share a codeword
    constexpr bool AHEAD = P <= 8;                  // room for the next dictionary's share
    __shared__ float4 row[kCacheMaxD / 4];
    __shared__ float part[Q][COLS];
    __shared__ int chosen;
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
    const int k = tid % COLS, q = tid / COLS, d4 = a.D >> 2;
    constexpr size_t SET = (size_t)P * Q * COLS;    // of a dictionary
    const int64_t jobs = a.n * a.H;
    for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
        const int h = (int)(job % a.H);
        const float4 *Th = T + (size_t)h * a.M * SET;
        float4 c[P], ahead[AHEAD ? P : 1];
        auto fetch = [&](int m, float4 (&to)[P]) {
#pragma unroll
            for (int i = 0; i < P; ++i) to[i] = (Th + m * SET + i * kFewThreads)[tid];       // piece q + i Q of codeword k
        };
        fetch(0, c);
        int64_t slot = -1;
        if (wave == 0) slot = take_row(a, job / a.H, h, row, kCacheMaxD, lane);
        __syncthreads();
        for (int m = 0; m < a.M; ++m) {
            if constexpr (AHEAD) fetch(min(m + 1, a.M - 1), ahead);
            float d = 0.f;
#pragma unroll
            for (int i = 0; i < P; ++i) {           // beyond D both are zero
                const float4 x = row[q + i * Q];
                const float e0 = x.x - c[i].x, e1 = x.y - c[i].y, e2 = x.z - c[i].z, e3 = x.w - c[i].w;
                d = fmaf(e3, e3, fmaf(e2, e2, fmaf(e1, e1, fmaf(e0, e0, d))));
            }
            part[q][k] = d;
            __syncthreads();
            if (wave == 0) {
                constexpr int N = COLS / kWave;
                float s[N];
                unsigned best = ~0u, next = ~0u;    // distances are not negative: they order as integers, NaN last
                int at = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    s[i] = 0.f;
#pragma unroll
                    for (int j = 0; j < Q; ++j) s[i] += part[j][lane + kWave * i];
                    const unsigned u = lane + kWave * i < a.K ? __float_as_uint(s[i]) & 0x7fffffffu : ~0u;
                    next = min(next, max(best, u));
                    at = u < best ? lane + kWave * i : at;
                    best = min(best, u);
                }
                const unsigned least = wave_min_bits(best);
                const int winner = __ffsll(__ballot(best == least)) - 1;
                const float b0 = __uint_as_float(least), b1 = __uint_as_float(wave_min_bits(lane == winner ? next : best));
                at = __builtin_amdgcn_readlane(at, winner);
                // 4 P additions of squares with one rounding in the difference and two in the square, and Q more
                constexpr float eta = (float)(4 * P + Q + 6) * 6.1e-8f;
                if (a.K > 1 && !(b0 * (1.f + eta) < b1 * (1.f - eta) && b1 > 1e-25f && b1 < __builtin_inff())) {
                    // every codeword that may be the nearest, in 64 bits
                    const float limit = b0 * (1.f + 4.f * eta) + 1e-30f;
                    const bool all = !(limit < __builtin_inff());
                    double db = __builtin_inf();
                    int kb = 0x7fffffff;
#pragma unroll 1
                    for (int i = 0; i < N; ++i) {
                        const int k0 = lane + kWave * i;
                        float si = s[0];
#pragma unroll
                        for (int j = 1; j < N; ++j) si = i == j ? s[j] : si;
                        if (k0 >= a.K || !(all || si <= limit)) continue;
                        double t = 0.0;
#pragma unroll 2
                        for (int p = 0; p < d4; ++p) {
                            const float4 u = Th[m * SET + (size_t)p * COLS + k0], w = row[p];
                            const double t0 = (double)w.x - (double)u.x, t1 = (double)w.y - (double)u.y, t2 = (double)w.z - (double)u.z, t3 = (double)w.w - (double)u.w;
                            t = fma(t3, t3, fma(t2, t2, fma(t1, t1, fma(t0, t0, t))));
                        }
                        if (t < db) {
                            db = t;
                            kb = k0;
                        }
                    }
#pragma unroll
                    for (int o = 32; o > 0; o >>= 1) {
                        const double od = __shfl_xor(db, o, kWave);
                        const int ok = __shfl_xor(kb, o, kWave);
                        if (od < db || (od == db && ok < kb)) { db = od; kb = ok; }
                    }
                    at = kb < a.K ? kb : 0;         // beyond only where a dictionary holds no numbers
                }
                if (lane == 0) {
                    chosen = at;
                    if (slot >= 0) a.codes[(slot * a.H + h) * a.M + m] = (uint8_t)at;
                }
            }
            __syncthreads();
            if (chosen == k) {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float4 x = row[q + i * Q];
                    row[q + i * Q] = make_float4(x.x - c[i].x, x.y - c[i].y, x.z - c[i].z, x.w - c[i].w);
                }
            }
            if constexpr (AHEAD) {
#pragma unroll
                for (int i = 0; i < P; ++i) c[i] = ahead[i];
            } else {
                fetch(min(m + 1, a.M - 1), c);
            }
            __syncthreads();
        }
    }
}

// Some rows a head: a block takes sixteen rows of one head through all dictionaries, a wave sixteen codewords, its share in registers
// as before (D > 64: 10 to 17 of its registers go to memory), as operands of the fp32 matrix cores (v_mfma_f32_16x16x4_f32: lane 16 g + i holds of codeword or row i the dimension
// that is the g-th of four).  Scores x.c - ||c||^2 / 2; a row whose two best are within what rounding can do to them,
//   (D + 8) 2^-22 (||x|| max||c|| + max||c||^2 / 2)                 (each of D products and additions loses at most a unit or two of 2^-23),
// is decided from the distances of the codewords within that margin by one wave (some 2 in 1000).
// A dictionary takes about 12000 cycles: 4096 are the matrix cores', the rest the three barriers and what is between them
// (1024 rows, D = 128, M = 16, K = 256: 92 us).
constexpr int kSomeRows = 16;
template <int COLS, int P>
__global__ __launch_bounds__(kFewThreads) void k_cache_write_some(const CacheRowsIn a, const float4 *__restrict__ T, const float *__restrict__ halves)
{
    constexpr bool AHEAD = P <= 8;
    constexpr int PITCH = 4 * P + 1;                // float4 of a row in LDS: an odd number, so that sixteen rows spread over the banks
    __shared__ float4 rows[kSomeRows][PITCH];
    __shared__ float4 found[kSomeRows][kWave];      // best, second, which of four; of each wave's four groups
    __shared__ int chosen[kSomeRows];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, g = lane >> 4;
    const int64_t per_head = (a.n + kSomeRows - 1) / kSomeRows, jobs = per_head * a.H;
    const bool mine = 16 * wave < COLS;             // the wave has codewords
    const int at = g * COLS + (mine ? 16 * wave : 0) + i16;
    for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
        const int h = (int)(job / per_head);
        const int64_t n0 = (job - h * per_head) * kSomeRows;
        constexpr size_t SET = (size_t)4 * P * COLS;
        const float4 *Th = T + (size_t)h * a.M * SET;
        const float *half = halves + (size_t)h * a.M * 256;
        float4 c[P], ahead[AHEAD ? P : 1], hc, hahead;
        float cmax, cmax_ahead;
        auto piece = [&](int m, int j) { return (Th + m * SET + j * 4 * COLS)[at]; };       // 4 j + g of codeword 16 wave + i16
        auto fetch_half = [&](int m, float4 &hm, float &most) {
            hm = *reinterpret_cast<const float4 *>(half + (size_t)m * 256 + (mine ? 16 * wave : 0) + 4 * g);
            most = halves[(size_t)a.H * a.M * 256 + h * a.M + m];
        };
#pragma unroll
        for (int j = 0; j < P; ++j) c[j] = piece(0, j);
        fetch_half(0, hc, cmax);
        const int64_t slot = take_row(a, n0 + wave, h, rows[wave], 16 * P, lane);       // a wave per row
        __syncthreads();
        for (int m = 0; m < a.M; ++m) {
            const int then_m = min(m + 1, a.M - 1);
            if (mine) {
                typedef float floatx4 __attribute__((ext_vector_type(4)));
                floatx4 acc = {hc.x, hc.y, hc.z, hc.w};
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const float4 x = rows[i16][4 * j + g];
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(c[j].x, x.x, acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(c[j].y, x.y, acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(c[j].z, x.z, acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(c[j].w, x.w, acc, 0, 0, 0);
                    // (all loads at once would wait for each other at the head: 128 KB at 64 bytes a cycle)
                    if constexpr (AHEAD) ahead[j] = piece(then_m, j);
                }
                fetch_half(then_m, hahead, cmax_ahead);
                // lane 16 g + i: codewords 16 wave + 4 g + v of row i
                float best = acc[0], second = -__builtin_inff();
                int v = 0;
#pragma unroll
                for (int w = 1; w < 4; ++w) {
                    second = acc[w] > best ? best : fmaxf(second, acc[w]);
                    if (acc[w] > best) {
                        best = acc[w];
                        v = w;
                    }
                }
                found[i16][4 * wave + g] = make_float4(best, second, __int_as_float(v), 0.f);
            } else if (fetch_half(then_m, hahead, cmax_ahead); lane < kSomeRows) {
#pragma unroll
                for (int w = 0; w < 4; ++w) found[lane][4 * wave + w] = make_float4(-__builtin_inff(), -__builtin_inff(), 0.f, 0.f);
            }
            __syncthreads();
            {
                const float4 f = found[wave][lane];
                const float4 x = 4 * lane < 16 * P ? rows[wave][lane] : make_float4(0.f, 0.f, 0.f, 0.f);
                float xx = fmaf(x.x, x.x, fmaf(x.y, x.y, fmaf(x.z, x.z, x.w * x.w)));
                // descending floats as ascending unsigned integers
                auto key = [](float s) { const unsigned u = __float_as_uint(s); return (int)u < 0 ? u : ~(u | 0x80000000u); };
                auto value = [](unsigned u) { return __uint_as_float((int)u < 0 ? u : ~u & 0x7fffffffu); };
                const unsigned most = wave_min_bits(key(f.x));
                const unsigned long long who = __ballot(key(f.x) == most);
                const int winner = __ffsll(who) - 1;
                const unsigned then = wave_min_bits(lane == winner ? key(f.y) : key(f.x));
                xx = sum16(xx);
                xx = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(xx), 0)) + __int_as_float(__builtin_amdgcn_readlane(__float_as_int(xx), 16)) +
                     __int_as_float(__builtin_amdgcn_readlane(__float_as_int(xx), 32)) + __int_as_float(__builtin_amdgcn_readlane(__float_as_int(xx), 48));
                const float err = (float)(16 * P + 8) * 2.4e-7f * (sqrtf(xx) * cmax + 0.5f * cmax * cmax) + 1e-36f;
                int nearest = 4 * winner + __builtin_amdgcn_readlane(__float_as_int(f.z), winner);
                const float top = value(most);
                if (!(top - value(then) > 2.f * err)) {
                    // the fours of codewords whose best is within the margin, sixteen lanes a codeword, in fp32
                    const unsigned long long near = __ballot(!(f.x < top - 2.f * err));
                    unsigned long long fours = near;
                    float least = __builtin_inff(), next = __builtin_inff();
                    int at = 0;
                    while (fours) {
                        const int k = 4 * (__ffsll(fours) - 1) + g;
                        fours &= fours - 1ull;
                        float d = 0.f;
#pragma unroll
                        for (int i = 0; i < P / 4; ++i) {
                            const int p = i16 + 16 * i;
                            const float4 u = Th[m * SET + (size_t)p * COLS + min(k, COLS - 1)], w = rows[wave][p];
                            const float e0 = w.x - u.x, e1 = w.y - u.y, e2 = w.z - u.z, e3 = w.w - u.w;
                            d = fmaf(e3, e3, fmaf(e2, e2, fmaf(e1, e1, fmaf(e0, e0, d))));
                        }
                        d = sum16(d);
                        if (k >= a.K) d = __builtin_inff();
                        next = d < least ? least : fminf(next, d);
                        if (d < least) {
                            least = d;
                            at = k;
                        }
                    }
                    float b0 = __builtin_inff(), b1 = __builtin_inff();
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float l = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(least), 16 * j)), t = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(next), 16 * j));
                        b1 = l < b0 ? fminf(b0, t) : fminf(b1, l);
                        if (l < b0) {
                            b0 = l;
                            nearest = __builtin_amdgcn_readlane(at, 16 * j);
                        }
                    }
                    constexpr float eta = (float)(P + 10) * 6.1e-8f;
                    if (a.K > 1 && !(b0 * (1.f + eta) < b1 * (1.f - eta) && b1 > 1e-25f)) {
                        // the same in 64 bits, the lowest index of equals
                        double db = __builtin_inf();
                        int kb = 0x7fffffff;
                        fours = near;
#pragma unroll 1
                        while (fours) {
                            const int k = 4 * (__ffsll(fours) - 1) + g;
                            fours &= fours - 1ull;
                            double t = 0.0;
#pragma unroll 1
                            for (int p = i16; p < 4 * P; p += 16) {
                                const float4 u = Th[m * SET + (size_t)p * COLS + min(k, COLS - 1)], w = rows[wave][p];
                                const double t0 = (double)w.x - (double)u.x, t1 = (double)w.y - (double)u.y, t2 = (double)w.z - (double)u.z, t3 = (double)w.w - (double)u.w;
                                t = fma(t3, t3, fma(t2, t2, fma(t1, t1, fma(t0, t0, t))));
                            }
#pragma unroll
                            for (int o = 1; o < 16; o <<= 1) t += __shfl_xor(t, o, kWave);
                            if (k < a.K && t < db) {                // ascending k
                                db = t;
                                kb = k;
                            }
                        }
#pragma unroll
                        for (int o = 16; o < kWave; o <<= 1) {
                            const double od = __shfl_xor(db, o, kWave);
                            const int ok = __shfl_xor(kb, o, kWave);
                            if (od < db || (od == db && ok < kb)) { db = od; kb = ok; }
                        }
                        nearest = __builtin_amdgcn_readfirstlane(kb < a.K ? kb : 0);
                    }
                }
                if (lane == 0) {
                    chosen[wave] = nearest;
                    if (slot >= 0) a.codes[(slot * a.H + h) * a.M + m] = (uint8_t)nearest;
                }
            }
            __syncthreads();
            {
                const int all = chosen[i16];
                unsigned hit = (unsigned)__ballot(lane < kSomeRows && (all >> 4) == wave);      // rows that leave one of the wave's codewords
                while (hit) {
                    const int r = __ffs(hit) - 1, k = __builtin_amdgcn_readlane(all, r);
                    hit &= hit - 1u;
                    if (i16 == (k & 15)) {
#pragma unroll
                        for (int j0 = 0; j0 < P; j0 += 4) {
                            float4 x[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) x[j] = rows[r][4 * (j0 + j) + g];
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                rows[r][4 * (j0 + j) + g] = make_float4(x[j].x - c[j0 + j].x, x[j].y - c[j0 + j].y, x[j].z - c[j0 + j].z, x[j].w - c[j0 + j].w);
                        }
                    }
                }
            }
            if constexpr (AHEAD) {
#pragma unroll
                for (int j = 0; j < P; ++j) c[j] = ahead[j];
            } else {
#pragma unroll
                for (int j = 0; j < P; ++j) c[j] = piece(then_m, j);
            }
            hc = hahead;
            cmax = cmax_ahead;
            __syncthreads();
        }
    }
}

// Many rows a head: scores from the fp16 matrix cores, a wave per tile of 32 rows of one head, through all its dictionaries, the
// rows staying in registers.  Scores, their bounds and the margins are those of assign_half.hpp: score k is off by at most
// e w_k + margin, so that with L the largest of (score - e w) a codeword is a candidate while score + e w_k >= L - 2 margin.
// For L the largest w of a block of 32 codewords stands for each one's: the codewords are laid out by ascending norm (k_cache_sort), so that
// it nearly is.  L runs along with the blocks: the candidates of two blocks are those that reach the L of that time, and blocks whose
// best does not reach the last L drop out at the end, so that no score is kept beyond its blocks (64 registers less than keeping
// all of them).  One candidate is the nearest codeword; two or more are decided in fp32 in their direct form, or in 64 bits.
// 131072 rows, D = 128, M = 8, K = 256: 160 us, 430 TFLOP/s of scores.  A dictionary takes a block 20000 to 28000 cycles, the products 5000 of them, the
// rows' fp16 images 2500; the rest are the loads of candidates (2.2 rows of 32 have more than one) and of the codewords to subtract, which wait on L2
// together in all waves of a block, as the dictionary in LDS holds them in step.  (K <= 64, D from 65 to 128, eight waves: 19 vector registers go to memory.)  Two blocks of half the waves a CU, waves out of step by half a
// dictionary and pairs of tiles a wave (registers spill) were no faster.
//
// Coordinates are laid out so that a lane's eight of a matrix instruction lie side by side in memory: position 16 t + 4 i .. + 3
// holds the coordinates 16 t + 4 j .. + 3 with j = 0, 2, 1, 3 for i = 0, 1, 2, 3.
struct CacheTables {
    const char *parts;                              // [H M][UNITS]: what passes through LDS, as TilePart says
    const float *C;                                 // [H M][K][Dp] sorted, positions in place of coordinates, zero beyond D
    const uint8_t *order;                           // [H M][256]: the codeword at a place
    const float *halves;                            // of k_cache_write_some (k_cache_sort)
};

// A part of a dictionary (all of it, or half of its blocks): the fp16 image, -||C||^2/2, fp16 {2^-10, w_k}, -mu, the largest w of each
// block, the constants; whole kilobytes.
struct TilePart {
    int image, hn, pairs, mu, w, consts, bytes;     // byte offsets, but for the first and the last
};
__host__ __device__ constexpr TilePart tile_part(int kbu, int nc)
{
    TilePart p = {};
    p.image = kbu * nc * 4096;
    p.hn = p.image;
    p.pairs = p.hn + 128 * kbu;
    p.mu = p.pairs + 128 * kbu;
    p.w = p.mu + 256 * nc;
    p.consts = p.w + 32;
    p.bytes = (p.consts + 4 * kEncodeConsts + 1023) / 1024 * 1024;
    return p;
}
__host__ __device__ constexpr int tile_units(int kb, int nc) { return kb * nc > 16 ? 2 : 1; }
// 64-position chunks of a row: 1, 2 or 4.
__host__ __device__ constexpr int cache_chunks(int D) { return D <= 64 ? 1 : D <= 128 ? 2 : 4; }
__host__ __device__ constexpr int cache_padded(int D) { return 64 * cache_chunks(D); }

// Codewords in ascending order of their distance from the mean of a few, equal ones by index.  A block per dictionary.
// halves: [dictionaries][256] -||c||^2 / 2 of codewords as they are, unscaled, and so -inf beyond K (a score may be any finite number); then
// [dictionaries] the largest ||c|| (rounded up).
__global__ __launch_bounds__(256) void k_cache_sort(const float *__restrict__ C, int K, int D, float *__restrict__ sorted, uint8_t *__restrict__ order,
                                                    float *__restrict__ halves)
{
    __shared__ float size[256];
    __shared__ float norm[256];
    __shared__ uint8_t at[256];
    const float *Cm = C + (size_t)blockIdx.x * K * D;
    const int lane = lane_id(), wave = threadIdx.x >> 6, tid = threadIdx.x;
    float4 mu = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < kMuRows; ++i) {
        const float4 v = load_row_piece(Cm, (int)((unsigned)(i * K) / kMuRows), 4 * lane, K, D, D);
        mu = make_float4(mu.x + v.x / kMuRows, mu.y + v.y / kMuRows, mu.z + v.z / kMuRows, mu.w + v.w / kMuRows);
    }
    at[tid] = 0;
    for (int k = wave; k < K; k += 4) {
        const float4 v = load_row_piece(Cm, k, 4 * lane, K, D, D);
        const float a = v.x - mu.x, b = v.y - mu.y, c = v.z - mu.z, d = v.w - mu.w;
        float s = 4 * lane < D ? a * a + b * b + c * c + d * d : 0.f;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
        const double n = wave_sum((double)v.x * v.x + (double)v.y * v.y + (double)v.z * v.z + (double)v.w * v.w);
        if (lane == 0) {
            norm[k] = s;
            size[k] = (float)(0.5 * n);
        }
    }
    __syncthreads();
    halves[(size_t)blockIdx.x * 256 + tid] = tid < K ? -size[tid] : -__builtin_inff();
    if (wave == 0) {
        float most = 0.f;
        for (int k = lane; k < K; k += kWave) most = fmaxf(most, size[k]);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o, kWave));
        if (lane == 0) halves[(size_t)gridDim.x * 256 + blockIdx.x] = sqrtf(2.f * most) * 1.00001f;
    }
    if (tid < K) {
        const float mine = norm[tid];
        int rank = 0;
        for (int k = 0; k < K; ++k) rank += norm[k] < mine || (!(norm[k] > mine) && k < tid) ? 1 : 0;
        at[min(rank, K - 1)] = (uint8_t)tid;        // the minimum for codewords that are no numbers
    }
    __syncthreads();
    order[(size_t)blockIdx.x * 256 + tid] = at[tid];
    const int Dp = cache_padded(D), d4 = Dp >> 2;
    for (int i = tid; i < K * d4; i += 256) {
        const int k = i / d4, p = i - k * d4, piece = (p & ~3) | (p & 1) << 1 | (p & 2) >> 1;
        reinterpret_cast<float4 *>(sorted + (size_t)blockIdx.x * K * Dp)[i] = load_row_piece(Cm, at[k], 4 * piece, K, D, D);
    }
}

// The parts, from what k_encode_prep leaves.  A block per part.
__global__ __launch_bounds__(256) void k_cache_pack(
    const char *__restrict__ img, const float *__restrict__ hn, const float *__restrict__ wtab, const float *__restrict__ negmu,
    const float *__restrict__ consts, int kb, int nc, int units, char *__restrict__ parts)
{
    const int set = blockIdx.x / units, u = blockIdx.x - set * units, kbu = kb / units, tid = threadIdx.x;
    const TilePart p = tile_part(kbu, nc);
    char *to = parts + (size_t)blockIdx.x * p.bytes;
    for (int i = tid; i < p.image / 16; i += 256) {
        const int at = i >> 6, t = at / kbu, b = at - t * kbu;      // kilobyte (t, b)
        reinterpret_cast<uint4 *>(to)[i] = reinterpret_cast<const uint4 *>(img + ((size_t)set * 4 * nc * kb + t * kb + u * kbu + b) * 1024)[i & 63];
    }
    const size_t first = (size_t)set * 32 * kb + u * 32 * kbu;
    if (tid < 32 * kbu) {
        const float w = wtab[first + tid];
        reinterpret_cast<float *>(to + p.hn)[tid] = hn[first + tid];
        reinterpret_cast<unsigned *>(to + p.pairs)[tid] = __builtin_bit_cast(unsigned, (halfx2){(_Float16)0.0009765625f, (_Float16)w});
        float most = w;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o, kWave));
        if ((tid & 31) == 0) reinterpret_cast<float *>(to + p.w)[tid >> 5] = most;
    }
    if (tid < 64 * nc) reinterpret_cast<float *>(to + p.mu)[tid] = negmu[(size_t)set * 64 * nc + tid];
    if (tid < kEncodeConsts) reinterpret_cast<float *>(to + p.consts)[tid] = consts[(size_t)set * kEncodeConsts + tid];
}

// LDS of k_cache_write_tiles: a part and the next, and a stretch for every wave: four undecided rows, or a piece of 16 positions of the
// codewords to subtract.
constexpr int kTileBatch = 4;                       // undecided rows of a wave at a time, sixteen lanes each
__host__ __device__ constexpr int tile_stretch(int nc) { return nc == 4 ? 4096 : 2048; }
__host__ __device__ constexpr int tile_lds(int kbu, int nc, int waves) { return 2 * tile_part(kbu, nc).bytes + waves * tile_stretch(nc); }

// Waves of a block: what LDS and registers allow.  Half of them where those are enough for all tiles at once.
__host__ __device__ constexpr int tile_waves(int nc) { return nc == 4 ? 4 : 8; }

// KB: blocks of 32 codewords.  NC: 64-position chunks (1, 2 or 4).  UNITS: parts in which a dictionary passes through LDS.
template <int KB, int NC, int UNITS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4) void k_cache_write_tiles(const CacheRowsIn a, const CacheTables tab, int groups)
{
    extern __shared__ float4 smem4[];
    char *lds = reinterpret_cast<char *>(smem4);
    constexpr int KBU = KB / UNITS, T = 4 * NC, S = 8 * NC, W = (KB + 1) / 2;
    constexpr TilePart L = tile_part(KBU, NC);
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hh = lane >> 5, r = lane & 31;
    const float inf = __builtin_inff();
    const int D = a.D;
    constexpr int Dp = 64 * NC;
    // blocks go round the XCDs: neighbouring groups of tiles, of one head, to one of them
    const int jobs = groups * a.H, per_xcd = (jobs + 7) / 8;
    const int stride = gridDim.x >> 3, mine0 = blockIdx.x >> 3;
    auto job_of = [&](int i) {                      // -1: none
        const int j = mine0 + i * stride;
        const int job = (int)(blockIdx.x & 7) * per_xcd + j;
        return j < per_xcd && job < jobs ? job : -1;
    };
    // part u of dictionary `set` into a half of LDS, a share for every wave
    auto stage = [&](int set, int u, int half) {
        const char *from = tab.parts + ((size_t)set * UNITS + u) * L.bytes + 16 * lane;
        char *to = lds + half * L.bytes;
#pragma unroll 1
        for (int at = wave * 1024; at < L.bytes; at += WAVES * 1024) load_to_lds(from + at, to + at);
    };
    auto landed = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0f70);         // vmcnt(0)
        __syncthreads();
    };
    char *stretch = lds + 2 * L.bytes + wave * tile_stretch(NC);
    int job = job_of(0), half = 1;
    if (job < 0) return;                            // the whole block
    stage(job / groups * a.M, 0, 0);
    for (int turn = 0; job >= 0; ++turn) {
        const int h = job / groups, after = job_of(turn + 1);
        const int64_t n0 = ((int64_t)(job - h * groups) * WAVES + wave) * kTileVec, n = n0 + r;
        const bool active = n0 < a.n;
        const int64_t slot = n < a.n ? a.slots[n] : -1;
        const bool live = slot >= 0 && slot < a.n_slots;
        float4 x[S];                                // x[2 t], x[2 t + 1]: coordinates 16 t + 8 hh .. + 7
        {
            int end = D - 8 * hh;                   // coordinates of the lane's first eight on
            asm volatile("" : "+v"(end));           // (what it decides is cheaper found again than kept: sixteen masks)
            const int64_t at = (live ? n * a.row_stride + h * a.head_stride : 0) + 8 * hh;
            auto from = [&](int s) { return at + min(16 * (s >> 1) + 4 * (s & 1), max(end - 4, -8 * hh)); };
            // all loads are on their way before the first is used; rows that are not kept read the first one
            if (a.type == kRowF32) {
#pragma unroll
                for (int s = 0; s < S; ++s) x[s] = F32::load(a.X, from(s));
            } else {
                uint2 raw[S];
#pragma unroll
                for (int s = 0; s < S; ++s) raw[s] = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(a.X) + from(s));
                const bool half = a.type == kRowF16;
#pragma unroll
                for (int s = 0; s < S; ++s) x[s] = half ? F16::widen(raw[s]) : Bf16::widen(raw[s]);
            }
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (!live || 16 * (s >> 1) + 4 * (s & 1) >= end) x[s] = make_float4(0.f, 0.f, 0.f, 0.f);
            int top = 0;                            // magnitudes order as integers do, NaN above infinity
#pragma unroll
            for (int s = 0; s < S; ++s)
                top = max(max(max(__float_as_int(fabsf(x[s].x)), __float_as_int(fabsf(x[s].y))), max(__float_as_int(fabsf(x[s].z)), __float_as_int(fabsf(x[s].w)))), top);
            const uint2 both = both_halves((unsigned)top);
            top = (int)max(both.x, both.y);
            float g = __int_as_float(top);
            if (top >= 0x7f800000) {
                g = __builtin_nanf("");
#pragma unroll
                for (int s = 0; s < S; ++s) x[s] = make_float4(0.f, 0.f, 0.f, 0.f);
            } else if (a.scale && top) {
                // x / g in fp32 by a product.  f is above 1 / g by 2^-53 to 2^-50 of it, the product's own rounding included, and a number of 50 bits is cut off:
                // a quotient that is a number of 50 bits comes out as it is, so one halfway between two fp32 numbers, which there is only among the
                // subnormal ones, is rounded as a tie; any other is 2^-49 of it away from there at least, as a quotient of two numbers of 24 bits, and stays on its side.
                const double f = 1.0 / (double)g * (1.0 + 0x1p-51);
                auto over = [&](float v) { return (float)__longlong_as_double(__double_as_longlong(v * f) & ~7ll); };
#pragma unroll
                for (int s = 0; s < S; ++s) x[s] = make_float4(over(x[s].x), over(x[s].y), over(x[s].z), over(x[s].w));
            }
            if (live && hh == 0 && a.scale) a.scale[slot * a.H + h] = g;
        }
        for (int m = 0; m < a.M; ++m) {
            const int set = h * a.M + m;
            halfx8 frag[T];
            uint32_t mk[W];                         // candidates: bit 16 b + v of word i is place 64 i + 32 b + 8 (v / 4) + 4 hh + v % 4
            float top[W];                           // the largest of score + e w of a word's codewords, at most
            float x2 = 0.f, e = 0.f, margin = 0.f, best = -inf;
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                landed();                                           // this part is there, and nobody needs the one before
                half ^= 1;
                const char *now = lds + half * L.bytes;
                const bool last = u == UNITS - 1 && m == a.M - 1;
                if (!last || after >= 0) stage(last ? after / groups * a.M : u == UNITS - 1 ? set + 1 : set, u == UNITS - 1 ? 0 : u + 1, half ^ 1);
                if (active) {
                    if (u == 0) {
                        const float *cc = reinterpret_cast<const float *>(now + L.consts);
                        HalfConsts c;
                        c.scale = cc[0];
                        c.h = cc[1];
                        c.rho = cc[2];
                        c.acc = cc[3];
                        c.hx = cc[4];
                        c.cmax = cc[5];
                        const floatv4 *mu4 = reinterpret_cast<const floatv4 *>(now + L.mu) + hh;
                        float xsq = 0.f, dsq = 0.f;
#pragma unroll
                        for (int t0 = 0; t0 < T; t0 += 4) {         // eight reads of LDS on their way at a time
                            floatv4 mu[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) mu[i] = mu4[4 * t0 + 2 * i];
                            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int t = t0 + i;
                                const floatv4 a = mu[2 * i], b = mu[2 * i + 1];
                                const halfx4 lo = half4(scaled(x[2 * t], c.scale, make_float4(a.x, a.y, a.z, a.w)), xsq, dsq);
                                const halfx4 hi = half4(scaled(x[2 * t + 1], c.scale, make_float4(b.x, b.y, b.z, b.w)), xsq, dsq);
                                frag[t] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                            }
                        }
                        const uint2 s2 = both_halves(__float_as_uint(xsq)), d2 = both_halves(__float_as_uint(dsq));
                        x2 = __uint_as_float(s2.x) + __uint_as_float(s2.y);
                        const float xn = sqrtf(x2) * 1.001f;
                        e = half_bound(x2, __uint_as_float(d2.x) + __uint_as_float(d2.y), xn, c);
                        // margin_half with the largest score there can be in place of the best
                        margin = margin_half(c, xn * c.cmax + 0.51f * c.cmax * c.cmax, xn, e);
                    }
                    const float *lds_h = reinterpret_cast<const float *>(now + L.hn), *lds_w = reinterpret_cast<const float *>(now + L.w);
                    const unsigned *lds_pair = reinterpret_cast<const unsigned *>(now + L.pairs);
                    const char *slot_of[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) slot_of[t] = now + half_slot(t, hh, r);
                    constexpr int GB = KBU < 2 ? 1 : 2;             // blocks whose products run together
                    // the dictionary's operands are read P products ahead, in an order that the scheduler may not change (contract_half)
                    constexpr int N = KBU * T, P = N < 4 ? N : 4;
                    auto operand = [&](int i) {
                        const int t = i % (T * GB) / GB, b = i / (T * GB) * GB + i % GB;
                        return *reinterpret_cast<const halfx8 *>(slot_of[t & 3] + (t * KBU + b) * 1024);
                    };
                    halfx8 ahead[P];
#pragma unroll
                    for (int i = 0; i < P; ++i) ahead[i] = operand(i);
                    constexpr int PAIRS = KBU / GB;
                    floatx16 acc[GB];
                    halfx4 right;
                    auto products = [&](int p) {
#pragma unroll
                        for (int j = 0; j < T * GB; ++j) {
                            const int i = p * T * GB + j, b = j % GB, t = j / GB;
                            acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ahead[i % P], frag[t], acc[b], 0, 0, 0);
                            if (i + P < N) ahead[i % P] = operand(i + P);
                            __builtin_amdgcn_sched_barrier(0x6);            // arithmetic may pass, products and memory not
                        }
                    };
                    auto threshold = [&](int p) {
                        const int i = (u * KBU + p * GB) / 2;
                        float low = -inf;
                        top[i] = -inf;
#pragma unroll
                        for (int b = 0; b < GB; ++b) {
                            const float most = block_max(acc[b]), w = lds_w[p * GB + b];
                            low = __builtin_elementwise_maximum(low, fmaf(-e, w, most));
                            top[i] = __builtin_elementwise_maximum(top[i], fmaf(e, w, most));
                        }
                        const uint2 low2 = both_halves(__float_as_uint(low));
                        best = __builtin_elementwise_maximum(__builtin_elementwise_maximum(best, __uint_as_float(low2.x)), __uint_as_float(low2.y));
                        // score + e w - (best - 2 margin), one more product of four terms: the threshold in three fp16 pieces (subtract_half), and e w
                        const float thr = fmaf(-2.f, margin, best);
                        const _Float16 p0 = (_Float16)(thr * -0.0009765625f);
                        const float rest = fmaf((float)p0, -1024.f, -thr);
                        const _Float16 p1 = (_Float16)rest;
                        right = (halfx4){p0, p1, (_Float16)((rest - (float)p1) * 1024.f), (_Float16)e};
                        if (hh) right = (halfx4){(_Float16)0.f, (_Float16)0.f, (_Float16)0.f, (_Float16)0.f};
                    };
                    auto subtract = [&](int p) {
#pragma unroll
                        for (int b = 0; b < GB; ++b) {
                            const uint2 left = make_uint2(__builtin_bit_cast(unsigned, (halfx2){(_Float16)1024.f, (_Float16)1.f}), lds_pair[32 * (p * GB + b) + r]);
                            acc[b] = __builtin_amdgcn_mfma_f32_32x32x8f16(__builtin_bit_cast(halfx4, left), right, acc[b], 0, 0, 0);
                        }
                        __builtin_amdgcn_sched_barrier(0x6);
                    };
                    auto reached = [&](int p) {
                        uint32_t word = 0u;
#pragma unroll
                        for (int b = GB - 1; b >= 0; --b)
#pragma unroll
                            for (int v = 15; v >= 0; --v) word = __builtin_amdgcn_alignbit(word, __float_as_uint(acc[b][v]), 31);  // (word << 1) | sign
                        mk[(u * KBU + p * GB) / 2] = KB == 1 ? ~word & 0xffffu : ~word;
                    };
#pragma unroll
                    for (int p = 0; p < PAIRS; ++p) {
                        init_acc<GB>(acc, lds_h + 32 * GB * p, hh);
                        products(p);
                        threshold(p);
                        subtract(p);
                        reached(p);
                    }
                }
            }
            if (!active) continue;
            const float thr = fmaf(-2.f, margin, best);
            const bool big = !(x2 < kHalfMaxNorm * kHalfMaxNorm && fabsf(best) + 2.f * margin < 0.5f * kHalfMaxThr);
#pragma unroll
            for (int i = 0; i < W; ++i) mk[i] = top[i] >= thr ? mk[i] : 0u;
            if (__ballot(big)) {                                    // may not fit fp16: all codewords that there are
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    uint32_t all = 0u;
                    for (int v = 0; v < (KB == 1 ? 16 : 32); ++v)
                        if (64 * i + 32 * (v >> 4) + 8 * ((v & 15) >> 2) + 4 * hh + (v & 3) < a.K) all |= 1u << v;
                    mk[i] = big ? all : mk[i];
                }
            }
            // the first and the last of the candidates left, the same in both lanes of the row; their number
            auto ends = [&](const uint32_t (&w)[W], int &front, int &back) {
                unsigned mine = 0u;
                uint32_t first = w[W - 1], last = w[0];
                int fi = W - 1, li = 0;
#pragma unroll
                for (int i = 0; i < W; ++i) mine += (unsigned)__popc(w[i]);
#pragma unroll
                for (int i = W - 2; i >= 0; --i)
                    if (w[i]) { first = w[i]; fi = i; }
#pragma unroll
                for (int i = 1; i < W; ++i)
                    if (w[i]) { last = w[i]; li = i; }
                const int f = __ffs(first) - 1, l = 31 - __clz(last);
                const uint2 n2 = both_halves(mine);
                const uint2 f2 = both_halves(first ? (unsigned)(64 * fi + 8 * (f >> 2) + 4 * hh + (f & 3)) : 256u);
                const uint2 l2 = both_halves(last ? (unsigned)(64 * li + 8 * (l >> 2) + 4 * hh + (l & 3)) : 0u);
                front = (int)min(f2.x, f2.y);
                back = (int)max(l2.x, l2.y);
                return n2.x + n2.y;
            };
            int front, back;
            const unsigned count = ends(mk, front, back);
            int place = front < a.K ? front : 0;
            const float *Cm = tab.C + (size_t)set * a.K * Dp;
            const uint8_t *order = tab.order + (size_t)set * 256;
            // Undecided rows, four at a time, sixteen lanes each: two candidates a round in fp32, which decides where the two nearest are further
            // apart than its error.  Their codewords are sent for before all others.
            const int g = lane >> 4, sub = lane & 15;
            float *rows = reinterpret_cast<float *>(stretch);
            const unsigned open = (unsigned)__ballot(live && count != 1u);
            int v[kTileBatch];                                      // the rows of a batch, -1: none
            bool one = false, two = false;                          // the lanes' row has one candidate, two
            floatv4 c0[NC], c1[NC];
            auto batch = [&](unsigned todo) {
#pragma unroll
                for (int j = 0; j < kTileBatch; ++j) {
                    v[j] = todo ? __ffs(todo) - 1 : -1;
                    todo &= todo - 1u;
                }
                int k0 = 256, k1 = 256;
#pragma unroll
                for (int j = 0; j < kTileBatch; ++j) {
                    const int f = __builtin_amdgcn_readlane(front, max(v[j], 0)), l = __builtin_amdgcn_readlane(back, max(v[j], 0));
                    if (g == j && v[j] >= 0) {
                        k0 = f;
                        k1 = l;
                    }
                }
                one = k0 < a.K;
                two = one && k1 != k0 && k1 < a.K;
                const floatv4 *at0 = reinterpret_cast<const floatv4 *>(Cm + (unsigned)((one ? k0 : 0) * Dp)) + sub;
                const floatv4 *at1 = reinterpret_cast<const floatv4 *>(Cm + (unsigned)((two ? k1 : 0) * Dp)) + sub;
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    c0[i] = at0[16 * i];
                    c1[i] = at1[16 * i];
                }
            };
            if (open) batch(open);
            // The first candidates' codewords: four lanes read 64 bytes of one.  (A lane that reads its own row's codeword touches a cache
            // line of its own.)
            const int row4 = lane >> 2, piece4 = lane & 3;
            const int p0 = __shfl(place, row4, kWave), p1 = __shfl(place, row4 + 16, kWave);
            floatv4 q0[T], q1[T];
            auto codeword4 = [&](int p) { return reinterpret_cast<const floatv4 *>(Cm + (unsigned)(p * Dp + 4 * piece4)); };
            {
                const floatv4 *first0 = codeword4(p0), *first1 = codeword4(p1);
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    q0[t] = first0[4 * t];
                    q1[t] = first1[4 * t];
                }
            }
            if (open) {
                uint32_t left[W];
                float least = inf, second = inf;
                const bool amb = (open >> r) & 1u;
#pragma unroll
                for (int i = 0; i < W; ++i) left[i] = mk[i];
                unsigned todo = open, more = count;
                while (todo) {
                    const int to = r == v[0] ? 0 : r == v[1] ? 1 : r == v[2] ? 2 : r == v[3] ? 3 : -1;
                    if (to >= 0) {
#pragma unroll
                        for (int s = 0; s < S; ++s) reinterpret_cast<float4 *>(rows + to * 64 * NC)[2 * s + hh] = x[s];
                    }
                    wave_lds_fence();
                    float d0 = 0.f, d1 = 0.f;
#pragma unroll
                    for (int i = 0; i < NC; ++i) {
                        const floatv4 w = reinterpret_cast<const floatv4 *>(rows + g * 64 * NC)[sub + 16 * i], e = w - c0[i], f = w - c1[i];
                        d0 = fmaf(e.w, e.w, fmaf(e.z, e.z, fmaf(e.y, e.y, fmaf(e.x, e.x, d0))));
                        d1 = fmaf(f.w, f.w, fmaf(f.z, f.z, fmaf(f.y, f.y, fmaf(f.x, f.x, d1))));
                    }
                    d0 = sum16(d0);
                    d1 = sum16(d1);
                    if (!one) d0 = inf;
                    if (!two) d1 = inf;
                    unsigned through = 0u;
#pragma unroll
                    for (int j = 0; j < kTileBatch; ++j) {
                        const float t0 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(d0), 16 * j)), t1 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(d1), 16 * j));
                        if (r == v[j]) {
                            second = t0 < least ? least : fminf(second, t0);
                            if (t0 < least) { least = t0; place = front; }
                            second = t1 < least ? least : fminf(second, t1);
                            if (t1 < least) { least = t1; place = back; }
                        }
                        if (v[j] >= 0) through |= 1u << v[j];
                    }
                    // the two are done with
                    const bool all = !__ballot(to >= 0 && more > 2u);
                    if (!all && to >= 0) {
#pragma unroll
                        for (int i = 0; i < W; ++i) {
                            const int f = front - 64 * i, l = back - 64 * i;
                            if (f >= 0 && f < 64 && ((f >> 2) & 1) == hh) left[i] &= ~(1u << (4 * (f >> 3) + (f & 3)));
                            if (l >= 0 && l < 64 && ((l >> 2) & 1) == hh) left[i] &= ~(1u << (4 * (l >> 3) + (l & 3)));
                        }
                    }
                    if (!all) more = ends(left, front, back);
                    todo &= all ? ~through : ~through | (unsigned)__ballot(more != 0u);
                    if (todo) batch(todo);
                    wave_lds_fence();
                }
                const float eta = (float)(4 * NC + 10) * 6.1e-8f;
                unsigned hard = (unsigned)__ballot(amb && !(least * (1.f + eta) < second * (1.f - eta) && second > 1e-25f));
                while (hard) {                                      // exact and nearly exact ties, one after another in 64 bits, by the whole wave
                    const int which = __ffs(hard) - 1;
                    hard &= hard - 1u;
                    if (r == which) {
#pragma unroll
                        for (int s = 0; s < S; ++s) reinterpret_cast<float4 *>(rows)[2 * s + hh] = x[s];
                    }
                    wave_lds_fence();
                    double db = __builtin_inf();
                    int kb = 0x7fffffff, pb = 0;
                    for (int i = 0; i < W; ++i) {
                        const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)mk[i], which), high = (uint32_t)__builtin_amdgcn_readlane((int)mk[i], which + 32);
                        const int p = 64 * i + lane, bit = 4 * (lane >> 3) + (lane & 3);
                        if (p >= a.K || !(((lane & 4 ? high : low) >> bit) & 1u)) continue;
                        const float *cw = Cm + (size_t)p * Dp;
                        double t = 0.0;
                        for (int d = 0; d < Dp; ++d) {
                            const double u = (double)rows[d] - (double)cw[d];
                            t += u * u;
                        }
                        const int k = order[p];
                        if (t < db || (t == db && k < kb)) { db = t; kb = k; pb = p; }
                    }
#pragma unroll
                    for (int o = 32; o > 0; o >>= 1) {
                        const double od = __shfl_xor(db, o, kWave);
                        const int ok = __shfl_xor(kb, o, kWave), op = __shfl_xor(pb, o, kWave);
                        if (od < db || (od == db && ok < kb)) { db = od; kb = ok; pb = op; }
                    }
                    if (r == which) place = pb;
                    wave_lds_fence();
                }
                // rows whose nearest is not the first candidate: their codewords again
                const int now0 = __shfl(place, row4, kWave), now1 = __shfl(place, row4 + 16, kWave);
                const floatv4 *other0 = codeword4(now0), *other1 = codeword4(now1);
                if (now0 != p0) {
#pragma unroll
                    for (int t = 0; t < T; ++t) q0[t] = other0[4 * t];
                }
                if (now1 != p1) {
#pragma unroll
                    for (int t = 0; t < T; ++t) q1[t] = other1[4 * t];
                }
            }
            if (live && hh == 0) a.codes[(slot * a.H + h) * a.M + m] = order[place];
            // a piece of 16 positions of all rows goes round through LDS to the lanes that hold the rows
            {
                floatv4 *around = reinterpret_cast<floatv4 *>(stretch);     // [32 rows][4 pieces], a piece at its number xor (row / 4) % 4
                const int in = 4 * row4 + (piece4 ^ ((row4 >> 2) & 3)), out = 4 * r, turn_of = (r >> 2) & 3;
                around[in] = q0[0];
                around[in + 64] = q1[0];
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    wave_lds_fence();
                    const floatv4 u = around[out + (hh ^ turn_of)], w = around[out + ((2 + hh) ^ turn_of)];
                    wave_lds_fence();
                    if (t + 1 < T) {                                // behind the reads: a wave's LDS operations stay in order
                        around[in] = q0[t + 1];
                        around[in + 64] = q1[t + 1];
                    }
                    x[2 * t] = make_float4(x[2 * t].x - u.x, x[2 * t].y - u.y, x[2 * t].z - u.z, x[2 * t].w - u.w);
                    x[2 * t + 1] = make_float4(x[2 * t + 1].x - w.x, x[2 * t + 1].y - w.y, x[2 * t + 1].z - w.z, x[2 * t + 1].w - w.w);
                }
                wave_lds_fence();
            }
        }
        job = after;
    }
}

}  // namespace hclae
