// Quantising the rows of a cache as they are written (hclae_cache_write): rows of H heads, each head with M dictionaries of its
// own, into slots of a paged cache.  Per row x and head
//   g = max |x|,  u = x / g  (u = x where no scales are kept),  r = u;
//   for m = 0..M-1:  i_m = argmin_k ||r - c_m(k)||^2 (the direct form in 64 bits, the lowest index of equals),  r = r - c_m(i_m) in 32 bits,
// which is the greedy encoding of Eq. 3 with one path on a row brought to a largest magnitude of one.
#pragma once
#include "decode.hpp"

namespace hclae {

constexpr int kCacheMaxD = 256;
constexpr int kFewThreads = 1024;

// Codewords a thread column of k_cache_write_few covers: 64, 128 or 256, and so the threads that share a codeword.
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

// The dictionaries as k_cache_write_few reads them: T[dictionary][piece of four coordinates][codeword], so that neighbouring lanes
// read neighbouring codewords; and a copy as they are.  A block per dictionary and 16 pieces.
__global__ __launch_bounds__(256) void k_cache_lay(const float *__restrict__ C, int K, int D, int columns, float *__restrict__ copy, float4 *__restrict__ T)
{
    const int d4 = D >> 2;
    const float4 *from = reinterpret_cast<const float4 *>(C + (size_t)blockIdx.x * K * D);
    float4 *to = T + (size_t)blockIdx.x * d4 * columns;
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
        if (p0 + j < d4) to[(size_t)(p0 + j) * columns + k0 + i] = tile[j][i];
        __syncthreads();
    }
}

// A few rows a head: a block takes R rows of one head through all dictionaries.  Every thread keeps a share of one codeword (its
// pieces q, q + Q, ...) in registers, the next dictionary's on their way meanwhile; the rows are in LDS, where all lanes read the
// same piece.  Distances in fp32, direct form, so a vector is hardly ever undecided (gap below some 1e-6); those are decided in 64
// bits.  The threads that hold the chosen codeword subtract it: no gather, a dictionary is read once.
template <int COLS, int P, int R>
__global__ __launch_bounds__(kFewThreads) void k_cache_write_few(const CacheRowsIn a, const float4 *__restrict__ T)
{
    constexpr int Q = kFewThreads / COLS;           // threads that share a codeword
    __shared__ float4 rows[R][kCacheMaxD / 4];
    __shared__ float part[R][Q][COLS];
    __shared__ int chosen[R];
    __shared__ int64_t slot[R];
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
    const int k = tid % COLS, q = tid / COLS, d4 = a.D >> 2;
    const int64_t jobs = (a.n + R - 1) / R * a.H;
    for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
    const int h = (int)(job % a.H);
    const int64_t n0 = job / a.H * R;
    const float4 *Th = T + (size_t)h * a.M * d4 * COLS;
    float4 c[P];
    auto fetch = [&](int m) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int p = q + i * Q;
            c[i] = p < d4 ? Th[((size_t)m * d4 + p) * COLS + k] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    };
    fetch(0);
    // the rows: a wave each
    if (wave < R) {
        const int64_t n = n0 + wave;
        const int64_t s = n < a.n ? a.slots[n] : -1;
        const bool live = s >= 0 && s < a.n_slots;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (live && lane < d4) v = load_in(a, n * a.row_stride + h * a.head_stride + 4 * lane);
        // magnitudes order as integers do, NaN above infinity
        int top = max(max(__float_as_int(fabsf(v.x)), __float_as_int(fabsf(v.y))), max(__float_as_int(fabsf(v.z)), __float_as_int(fabsf(v.w))));
        top = wave_max_int(top);
        float g = __int_as_float(top);
        if (top >= 0x7f800000) {                    // not a number: kept as a row of zeros whose scale says so
            v = make_float4(0.f, 0.f, 0.f, 0.f);
            g = __builtin_nanf("");
        } else if (a.scale && top) {
            v = make_float4(v.x / g, v.y / g, v.z / g, v.w / g);
        }
        rows[wave][lane] = v;
        if (lane == 0) {
            slot[wave] = live ? s : -1;
            if (live && a.scale) a.scale[s * a.H + h] = g;
        }
    }
    __syncthreads();
    for (int m = 0; m < a.M; ++m) {
        float d[R];
#pragma unroll
        for (int r = 0; r < R; ++r) d[r] = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float4 x = rows[r][min(q + i * Q, kCacheMaxD / 4 - 1)];
                if (q + i * Q < d4) {
                    const float e0 = x.x - c[i].x, e1 = x.y - c[i].y, e2 = x.z - c[i].z, e3 = x.w - c[i].w;
                    d[r] = fmaf(e3, e3, fmaf(e2, e2, fmaf(e1, e1, fmaf(e0, e0, d[r]))));
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) part[r][q][k] = d[r];
        __syncthreads();
        if (wave < R) {                             // a wave per row
            constexpr int N = COLS / kWave;
            const float inf = __builtin_inff();
            float s[N], best = inf, second = inf;
            int at = 0x7fffffff;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int kk = lane + kWave * i;
                s[i] = 0.f;
#pragma unroll
                for (int j = 0; j < Q; ++j) s[i] += part[wave][j][kk];
                if (kk >= a.K) s[i] = inf;
                second = s[i] < best ? best : fminf(second, s[i]);
                if (s[i] < best || at == 0x7fffffff) {
                    if (kk < a.K) at = kk;
                    best = fminf(best, s[i]);
                }
            }
#pragma unroll
            for (int o = 1; o < kWave; o <<= 1) {
                const float ob = __shfl_xor(best, o, kWave), os = __shfl_xor(second, o, kWave);
                const int oa = __shfl_xor(at, o, kWave);
                second = fminf(fmaxf(best, ob), fminf(second, os));
                if (ob < best || (ob == best && oa < at)) at = oa;
                best = fminf(best, ob);
            }
            // relative error of a sum: 4 P additions of squares with one rounding each in the difference, twice in the square, and Q more
            const float eta = (float)(4 * P + Q + 6) * 6.1e-8f;
            if (!(best * (1.f + eta) < second * (1.f - eta) && second > 1e-25f)) {
                // every codeword that may be the nearest, in 64 bits, ascending dimensions
                const float limit = best * (1.f + 4.f * eta) + 1e-30f;
                const float *row = reinterpret_cast<const float *>(rows[wave]);
                double db = __builtin_inf();
                int ka = 0x7fffffff;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int kk = lane + kWave * i;
                    if (kk >= a.K || !(s[i] <= limit || !(limit < inf))) continue;
                    double t = 0.0;
                    for (int p = 0; p < d4; ++p) {
                        const float4 u = Th[((size_t)m * d4 + p) * COLS + kk];
                        const double t0 = (double)row[4 * p] - (double)u.x, t1 = (double)row[4 * p + 1] - (double)u.y;
                        const double t2 = (double)row[4 * p + 2] - (double)u.z, t3 = (double)row[4 * p + 3] - (double)u.w;
                        t += t0 * t0;
                        t += t1 * t1;
                        t += t2 * t2;
                        t += t3 * t3;
                    }
                    if (t < db || (t == db && kk < ka)) { db = t; ka = kk; }
                }
#pragma unroll
                for (int o = 32; o > 0; o >>= 1) {
                    const double od = __shfl_xor(db, o, kWave);
                    const int ok = __shfl_xor(ka, o, kWave);
                    if (od < db || (od == db && ok < ka)) { db = od; ka = ok; }
                }
                at = ka;
            }
            at = at < a.K ? at : 0;                 // beyond only where a dictionary holds no numbers
            if (lane == 0) {
                chosen[wave] = at;
                const int64_t s0 = slot[wave];
                if (s0 >= 0) a.codes[(s0 * a.H + h) * a.M + m] = (uint8_t)at;
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (chosen[r] == k) {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const int p = q + i * Q;
                    if (p < d4) {
                        const float4 x = rows[r][p];
                        rows[r][p] = make_float4(x.x - c[i].x, x.y - c[i].y, x.z - c[i].z, x.w - c[i].w);
                    }
                }
            }
        }
        if (m + 1 < a.M) fetch(m + 1);
        __syncthreads();
    }
    }
}

}  // namespace hclae
