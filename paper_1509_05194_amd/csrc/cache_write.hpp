// Quantising the rows of a cache as they are written (hclae_cache_write): rows of H heads, each head with M dictionaries of its
// own, into slots of a paged cache.  Per row x and head
//   g = max |x|,  u = x / g  (u = x where no scales are kept),  r = u;
//   for m = 0..M-1:  i_m = argmin_k ||r - c_m(k)||^2 (the direct form in 64 bits, the lowest index of equals),  r = r - c_m(i_m) in 32 bits,
// which is the greedy encoding of Eq. 3 with one path on a row brought to a largest magnitude of one.
#pragma once
#include <type_traits>
#include "assign_half.hpp"
#include "decode.hpp"
#include "encode.hpp"
#include "encode_wave.hpp"

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


// Many rows a head: scores from the fp16 matrix cores, a wave per tile of 32 rows of one head, through all its dictionaries, the
// rows staying in registers.  Scores, their bounds and the margins are those of assign_half.hpp: score k is off by at most
// e w_k + h, so that with L the largest of (score - e w) - h a codeword is a candidate while score + e w + h >= L.
// Here w is one for all 32 codewords of a block, the largest: the codewords are laid out by ascending norm (k_cache_sort), so that it
// is nearly each one's own.  L runs along with the blocks: the candidates of a block are those that reach the L of that
// time, and blocks whose best does not reach the last L drop out at the end.  No score is kept beyond its block.
struct CacheTables {
    const char *img;                                // [H M] as k_encode_prep lays them out, of the sorted codewords
    const float *hn, *w, *negmu, *consts;           // w: [H M][KB], the largest of each block's
    const float *C;                                 // [H][M][K][D] sorted
    const uint8_t *order;                           // [H M][256]: the codeword at a place
};

// Codewords in ascending order of their distance from the mean of a few, equal ones by index.  A block per dictionary.
__global__ __launch_bounds__(256) void k_cache_sort(const float *__restrict__ C, int K, int D, float *__restrict__ sorted, uint8_t *__restrict__ order)
{
    __shared__ float norm[256];
    __shared__ uint8_t at[256];
    const float *Cm = C + (size_t)blockIdx.x * K * D;
    const int lane = lane_id(), wave = threadIdx.x >> 6, d4 = D >> 2;
    float4 mu = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < kMuRows; ++i) {
        const float4 v = load_row_piece(Cm, (int)((unsigned)(i * K) / kMuRows), 4 * lane, K, D, D);
        mu = make_float4(mu.x + v.x / kMuRows, mu.y + v.y / kMuRows, mu.z + v.z / kMuRows, mu.w + v.w / kMuRows);
    }
    for (int k = wave; k < K; k += 4) {
        const float4 v = load_row_piece(Cm, k, 4 * lane, K, D, D);
        const float a = v.x - mu.x, b = v.y - mu.y, c = v.z - mu.z, d = v.w - mu.w;
        float s = 4 * lane < D ? a * a + b * b + c * c + d * d : 0.f;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
        if (lane == 0) norm[k] = s;
    }
    __syncthreads();
    if ((int)threadIdx.x < K) {
        const float mine = norm[threadIdx.x];
        int rank = 0;
        for (int k = 0; k < K; ++k) rank += norm[k] < mine || (!(norm[k] > mine) && k < (int)threadIdx.x) ? 1 : 0;
        rank = min(rank, K - 1);                    // codewords that are no numbers
        at[rank] = (uint8_t)threadIdx.x;
    }
    __syncthreads();
    if ((int)threadIdx.x < 256) order[(size_t)blockIdx.x * 256 + threadIdx.x] = (int)threadIdx.x < K ? at[threadIdx.x] : 0;
    for (int i = threadIdx.x; i < K * d4; i += 256) {
        const int k = i / d4, p = i - k * d4;
        reinterpret_cast<float4 *>(sorted + (size_t)blockIdx.x * K * D)[i] = reinterpret_cast<const float4 *>(Cm + (size_t)min((int)at[k], K - 1) * D)[p];
    }
}

// The largest w of every block of 32 codewords (wtab: [blocks][32]).
__global__ __launch_bounds__(256) void k_cache_block_w(const float *__restrict__ wtab, int64_t blocks, float *__restrict__ w)
{
    const int64_t b = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    float v = b < blocks ? wtab[b * 32 + (threadIdx.x & 31)] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, kWave));
    if (b < blocks && (threadIdx.x & 31) == 0) w[b] = v;
}

// LDS of k_cache_write_tiles: a dictionary (or half of one) and the next, and what undecided rows are decided in.
constexpr int kTileBatch = 4;                       // undecided rows of a wave at a time, sixteen lanes each
struct TileLds {
    int unit;                                       // bytes of an image
    int img, hn, mu, w, rows, masks, total;  // byte offsets; all but the last two of them twice
};
__host__ __device__ constexpr TileLds tile_lds(int kbu, int nc, int waves)
{
    TileLds l = {};
    l.unit = kbu * nc * 4096;
    l.img = 0;
    l.hn = 2 * l.unit;
    l.mu = l.hn + 2 * 128 * kbu;
    l.w = l.mu + 2 * 256 * nc;
    l.rows = l.w + 2 * 32;
    l.masks = l.rows + waves * kTileBatch * 256 * nc;
    l.total = l.masks + waves * kTileBatch * 32;
    return l;
}

// The sum over the sixteen lanes of a row, the same in all of them.
__device__ __forceinline__ float sum16(float v)
{
    auto from = [](float x, auto c) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(c)::value, 0xf, 0xf, true)); };
    v += from(v, std::integral_constant<int, 0xB1>());     // quad_perm 1 0 3 2
    v += from(v, std::integral_constant<int, 0x4E>());     // quad_perm 2 3 0 1
    v += from(v, std::integral_constant<int, 0x141>());    // row_half_mirror
    v += from(v, std::integral_constant<int, 0x140>());    // row_mirror
    return v;
}

// KB: blocks of 32 codewords.  NC: 64-dim chunks (1, 2 or 4).  UNITS: parts in which a dictionary passes through LDS.
template <int KB, int NC, int UNITS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_cache_write_tiles(const CacheRowsIn a, const CacheTables tab, int groups)
{
    extern __shared__ float4 smem4[];
    char *lds = reinterpret_cast<char *>(smem4);
    constexpr int KBU = KB / UNITS, T = 4 * NC, S = 8 * NC;
    constexpr TileLds L = tile_lds(KBU, NC, WAVES);
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hh = lane >> 5, r = lane & 31;
    const float inf = __builtin_inff();
    const int D = a.D;
    // blocks go round the XCDs: neighbouring groups of tiles, of one head, to one of them
    const int jobs = groups * a.H, per_xcd = (jobs + 7) / 8;
    const int stride = gridDim.x >> 3, mine0 = blockIdx.x >> 3;
    auto job_of = [&](int i) {                      // -1: none
        const int j = mine0 + i * stride;
        const int job = (int)(blockIdx.x & 7) * per_xcd + j;
        return j < per_xcd && job < jobs ? job : -1;
    };
    // part u of dictionary `set` into a half of LDS, all waves together
    auto stage = [&](int set, int u, int half) {
        const char *from = tab.img + (size_t)set * UNITS * L.unit + 16 * lane;
        char *to = lds + L.img + half * L.unit;
        constexpr int pieces = L.unit / 1024;
#pragma unroll
        for (int i = 0; i < (pieces + WAVES - 1) / WAVES; ++i) {
            const int at = i * WAVES + wave;        // kilobyte (t, b) of the part
            if (pieces % WAVES == 0 || at < pieces) load_to_lds(from + ((at / KBU) * KB + u * KBU + at % KBU) * 1024, to + at * 1024);
        }
        const int tid = threadIdx.x;
        for (int i = tid; i < 32 * KBU; i += 64 * WAVES)
            reinterpret_cast<float *>(lds + L.hn + half * 128 * KBU)[i] = tab.hn[(size_t)set * 32 * KB + u * 32 * KBU + i];
        for (int i = tid; i < 64 * NC; i += 64 * WAVES) reinterpret_cast<float *>(lds + L.mu + half * 256 * NC)[i] = tab.negmu[(size_t)set * 64 * NC + i];
        if (wave == WAVES - 1 && lane < KBU) reinterpret_cast<float *>(lds + L.w + half * 32)[lane] = tab.w[(size_t)set * KB + u * KBU + lane];
    };
    auto landed = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0f70);         // vmcnt(0)
        __syncthreads();
    };
    int half = 0, job = job_of(0);
    if (job < 0) return;                            // the whole block
    stage(job / groups * a.M, 0, 0);
    landed();
    for (int turn = 0; job >= 0; ++turn) {
        const int h = job / groups, after = job_of(turn + 1);
        const int64_t n0 = ((int64_t)(job - h * groups) * WAVES + wave) * kTileVec, n = n0 + r;
        const bool active = n0 < a.n;
        const int64_t slot = n < a.n ? a.slots[n] : -1;
        const bool live = slot >= 0 && slot < a.n_slots;
        float4 x[S];
#pragma unroll
        for (int s = 0; s < S; ++s) {
            x[s] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (live && 8 * s + 4 * hh < D) x[s] = load_in(a, n * a.row_stride + h * a.head_stride + 8 * s + 4 * hh);
        }
        {
            int top = 0;                            // magnitudes order as integers do, NaN above infinity
#pragma unroll
            for (int s = 0; s < S; ++s)
                top = max(max(max(__float_as_int(fabsf(x[s].x)), __float_as_int(fabsf(x[s].y))), max(__float_as_int(fabsf(x[s].z)), __float_as_int(fabsf(x[s].w)))), top);
            const uint2 both = both_halves((unsigned)top);
            top = (int)max(both.x, both.y);
            float g = __int_as_float(top);
            const bool bad = top >= 0x7f800000;
            if (bad) g = __builtin_nanf("");
            if (bad) {
#pragma unroll
                for (int s = 0; s < S; ++s) x[s] = make_float4(0.f, 0.f, 0.f, 0.f);
            } else if (a.scale && top) {
#pragma unroll
                for (int s = 0; s < S; ++s) x[s] = make_float4(x[s].x / g, x[s].y / g, x[s].z / g, x[s].w / g);
            }
            if (live && hh == 0 && a.scale) a.scale[slot * a.H + h] = g;
        }
        for (int m = 0; m < a.M; ++m) {
            const int set = h * a.M + m;
            const float *cc = tab.consts + (size_t)set * kEncodeConsts;
            HalfConsts c;
            c.scale = cc[0];
            c.h = cc[1];
            c.rho = cc[2];
            c.acc = cc[3];
            c.hx = cc[4];
            c.cmax = cc[5];
            halfx8 frag[T];
            uint32_t mk[(KB + 1) / 2];
            float top[KB];
            float x2 = 0.f, e = 0.f, margin = 0.f, best = -inf;
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                // the next part travels while this one is contracted
                const bool last = u == UNITS - 1 && m == a.M - 1;
                if (!last || after >= 0) stage(last ? after / groups * a.M : u == UNITS - 1 ? set + 1 : set, u == UNITS - 1 ? 0 : u + 1, half ^ 1);
                if (active) {
                    if (u == 0) {
                        const float4 *mu4 = reinterpret_cast<const float4 *>(lds + L.mu + half * 256 * NC) + hh;
                        float xsq = 0.f, dsq = 0.f;
#pragma unroll
                        for (int t = 0; t < T; ++t) {
                            const halfx4 lo = half4(scaled(x[2 * t], c.scale, mu4[4 * t]), xsq, dsq);
                            const halfx4 hi = half4(scaled(x[2 * t + 1], c.scale, mu4[4 * t + 2]), xsq, dsq);
                            frag[t] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                        }
                        const uint2 s2 = both_halves(__float_as_uint(xsq)), d2 = both_halves(__float_as_uint(dsq));
                        x2 = __uint_as_float(s2.x) + __uint_as_float(s2.y);
                        const float xn = sqrtf(x2) * 1.001f;
                        e = half_bound(x2, __uint_as_float(d2.x) + __uint_as_float(d2.y), xn, c);
                        // margin_half with the largest score there can be in place of the best
                        margin = margin_half(c, xn * c.cmax + 0.51f * c.cmax * c.cmax, xn, e);
                    }
                    const char *base = lds + L.img + half * L.unit;
                    const float *lds_h = reinterpret_cast<const float *>(lds + L.hn + half * 128 * KBU), *lds_w = reinterpret_cast<const float *>(lds + L.w + half * 32);
                    const char *slot_of[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) slot_of[t] = base + half_slot(t, hh, r);
                    constexpr int GB = KBU < 2 ? 1 : 2;             // blocks whose products run together
#pragma unroll
                    for (int b0 = 0; b0 < KBU; b0 += GB) {
                        floatx16 acc[GB];
                        init_acc<GB>(acc, lds_h + 32 * b0, hh);
#pragma unroll
                        for (int t = 0; t < T; ++t)
#pragma unroll
                            for (int b = 0; b < GB; ++b)
                                acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const halfx8 *>(slot_of[t & 3] + (t * KBU + b0 + b) * 1024), frag[t],
                                                                                acc[b], 0, 0, 0);
#pragma unroll
                        for (int b = 0; b < GB; ++b) {
                            const int blk = u * KBU + b0 + b;
                            const float ew = e * lds_w[b0 + b];
                            top[blk] = block_max(acc[b]) + ew;      // an upper bound but for h
                            const uint2 t2 = both_halves(__float_as_uint(top[blk]));
                            best = fmaxf(best, fmaxf(__uint_as_float(t2.x), __uint_as_float(t2.y)) - 2.f * ew);
                            floatx16 one[1] = {acc[b]};
                            subtract_half<1>(one, best - 2.f * margin - ew, hh);
                            uint32_t below = 0u;
#pragma unroll
                            for (int v = 15; v >= 0; --v) below = __builtin_amdgcn_alignbit(below, __float_as_uint(one[0][v]), 31);
                            const uint32_t bits = ~below & 0xffffu;
                            if (blk & 1) mk[blk >> 1] |= bits << 16;
                            else mk[blk >> 1] = bits;
                        }
                    }
                }
                landed();                                           // the next part is there, this one is free
                half ^= 1;
            }
            if (!active) continue;
            const bool big = !(x2 < kHalfMaxNorm * kHalfMaxNorm && fabsf(best) + 2.f * margin + 2.f * e * c.cmax < 0.5f * kHalfMaxThr);
            unsigned mine = 0u;
            int place = 256;
#pragma unroll
            for (int b = KB - 1; b >= 0; --b) {
                uint32_t bits = (mk[b >> 1] >> (16 * (b & 1))) & 0xffffu, real = 0xffffu;
                if (!(top[b] >= best - 2.f * margin)) bits = 0u;
                if (big) bits = 0xffffu;                            // may not fit fp16: all codewords that there are
                if (32 * (b + 1) > a.K) {
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (32 * b + 8 * (v >> 2) + 4 * hh + (v & 3) >= a.K) real &= ~(1u << v);
                }
                bits &= real;
                mk[b >> 1] = b & 1 ? (mk[b >> 1] & 0xffffu) | bits << 16 : (mk[b >> 1] & 0xffff0000u) | bits;
                mine += (unsigned)__popc(bits);
                const int v = __ffs(bits) - 1;
                if (bits) place = 32 * b + 8 * (v >> 2) + 4 * hh + (v & 3);
            }
            const uint2 count = both_halves(mine), at2 = both_halves((unsigned)place);
            place = (int)min(at2.x, at2.y);
            place = place < a.K ? place : 0;
            unsigned who = (unsigned)__ballot(live && count.x + count.y != 1u);
            const float *Cm = tab.C + (size_t)set * a.K * D;
            const uint8_t *order = tab.order + (size_t)set * 256;
            while (who) {
                // up to four undecided rows, sixteen lanes each: fp32 direct form where the two best are further apart than its error
                int v[kTileBatch];
#pragma unroll
                for (int j = 0; j < kTileBatch; ++j) {
                    v[j] = who ? __ffs(who) - 1 : -1;
                    who &= who - 1u;
                }
                float *rows = reinterpret_cast<float *>(lds + L.rows) + wave * kTileBatch * 64 * NC;
                uint16_t *masks = reinterpret_cast<uint16_t *>(lds + L.masks) + wave * kTileBatch * 16;
                const int to = r == v[0] ? 0 : r == v[1] ? 1 : r == v[2] ? 2 : r == v[3] ? 3 : -1;
                if (to >= 0) {
#pragma unroll
                    for (int s = 0; s < S; ++s) reinterpret_cast<float4 *>(rows + to * 64 * NC)[2 * s + hh] = x[s];
#pragma unroll
                    for (int b = 0; b < KB; ++b) masks[to * 16 + 2 * b + hh] = (uint16_t)(mk[b >> 1] >> (16 * (b & 1)));
                }
                wave_lds_fence();
                const int g = lane >> 4, sub = lane & 15;
                const float4 *row = reinterpret_cast<const float4 *>(rows + g * 64 * NC);
                const unsigned *words = reinterpret_cast<const unsigned *>(masks + g * 16);
                const bool have = (g == 0 ? v[0] : g == 1 ? v[1] : g == 2 ? v[2] : v[3]) >= 0;
                int word = 0;
                unsigned left = have ? words[0] : 0u;
                auto take = [&]() {                                 // the next candidate, -1 beyond the last
                    while (!left && have && word + 1 < KB) left = words[++word];
                    if (!left) return -1;
                    const int p = __ffs(left) - 1;
                    left &= left - 1u;
                    return 32 * word + 8 * ((p & 15) >> 2) + 4 * (p >> 4) + (p & 3);
                };
                float least = inf, second = inf;
                int at = 0;
                for (int k0 = take(); __ballot(k0 >= 0); k0 = take()) {
                    const int k1 = take();
                    float4 q[2][NC];
#pragma unroll
                    for (int i = 0; i < NC; ++i) {
                        const int p = sub + 16 * i;
                        q[0][i] = q[1][i] = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (k0 >= 0 && 4 * p < D) q[0][i] = reinterpret_cast<const float4 *>(Cm + (size_t)k0 * D)[p];
                        if (k1 >= 0 && 4 * p < D) q[1][i] = reinterpret_cast<const float4 *>(Cm + (size_t)k1 * D)[p];
                    }
                    float d[2] = {0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < NC; ++i) {
                        const float4 w = row[sub + 16 * i];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const float e0 = w.x - q[j][i].x, e1 = w.y - q[j][i].y, e2 = w.z - q[j][i].z, e3 = w.w - q[j][i].w;
                            d[j] = fmaf(e3, e3, fmaf(e2, e2, fmaf(e1, e1, fmaf(e0, e0, d[j]))));
                        }
                    }
                    const float d0 = k0 >= 0 ? sum16(d[0]) : inf, d1 = k1 >= 0 ? sum16(d[1]) : inf;
                    second = d0 < least ? least : fminf(second, d0);
                    if (d0 < least) { least = d0; at = k0; }
                    second = d1 < least ? least : fminf(second, d1);
                    if (d1 < least) { least = d1; at = k1; }
                }
                const float eta = (float)(4 * NC + 10) * 6.1e-8f;
                const bool sure = least * (1.f + eta) < second * (1.f - eta) && second > 1e-25f;
                unsigned long long hard = __ballot(have && !sure && sub == 0);
                while (hard) {                                      // exact and nearly exact ties, in 64 bits by the whole wave
                    const int which = (__ffsll(hard) - 1) >> 4;
                    hard &= hard - 1ull;
                    const float *one = rows + which * 64 * NC;
                    const unsigned *bits = reinterpret_cast<const unsigned *>(masks + which * 16);
                    double db = __builtin_inf();
                    int kb = 0x7fffffff, pb = 0;
                    for (int p = lane; p < a.K; p += kWave) {
                        const int i = p & 31, bit = 4 * (i >> 3) + (i & 3) + 16 * ((i >> 2) & 1);
                        if (!((bits[p >> 5] >> bit) & 1u)) continue;
                        const float *cw = Cm + (size_t)p * D;
                        double t = 0.0;
                        for (int d = 0; d < D; ++d) {
                            const double u = (double)one[d] - (double)cw[d];
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
                    if (g == which) at = pb;
                }
#pragma unroll
                for (int j = 0; j < kTileBatch; ++j) {
                    const int decided = __builtin_amdgcn_readlane(at, 16 * j);
                    if (r == v[j]) place = decided;
                }
                wave_lds_fence();
            }
            if (live && hh == 0) a.codes[(slot * a.H + h) * a.M + m] = order[place];
#pragma unroll
            for (int s = 0; s < S; ++s) {
                float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
                if (8 * s + 4 * hh < D) q = reinterpret_cast<const float4 *>(Cm + (size_t)place * D)[2 * s + hh];
                x[s] = make_float4(x[s].x - q.x, x[s].y - q.y, x[s].z - q.z, x[s].w - q.w);
            }
        }
        job = after;
    }
}

}  // namespace hclae
