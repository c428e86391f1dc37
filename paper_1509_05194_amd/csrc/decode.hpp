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
    __device__ static __forceinline__ float4 load(const void *p, int64_t at)
    {
        const h4 v = *reinterpret_cast<const h4 *>(static_cast<const _Float16 *>(p) + at);
        return make_float4((float)v.x, (float)v.y, (float)v.z, (float)v.w);
    }
    __device__ static __forceinline__ void store(void *p, int64_t at, const float4 &v)
    {
        *reinterpret_cast<h4 *>(static_cast<_Float16 *>(p) + at) = (h4){(_Float16)v.x, (_Float16)v.y, (_Float16)v.z, (_Float16)v.w};
    }
};
struct Bf16 {
    static constexpr int bytes = 2;
    typedef __bf16 b4 __attribute__((ext_vector_type(4)));
    __device__ static __forceinline__ float4 load(const void *p, int64_t at)
    {
        const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p) + at);
        return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
    }
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
};

struct CacheRows {                                  // hclae_cache_read
    const int32_t *tables, *starts;
    int B, max_pages, page;
    int64_t pages;                                  // of the cache
    // The sequence of row t is the last one that starts at or before it; whatever `starts` holds, the search ends inside [0, B).
    __host__ __device__ constexpr int64_t at(int64_t t) const
    {
        if (t < starts[0] || t >= starts[B]) return kSkip;
        int lo = 0, hi = B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (starts[mid] <= t) lo = mid;
            else hi = mid;
        }
        const int64_t pos = t - starts[lo];
        if (pos < 0 || pos > 0x7fffffff) return kSkip;
        const unsigned p = (unsigned)pos / (unsigned)page, off = (unsigned)pos - p * (unsigned)page;
        if (p >= (unsigned)max_pages) return kNoRow;
        const int32_t q = tables[(int64_t)lo * max_pages + p];
        return q >= 0 && q < pages ? (int64_t)q * page + off : kNoRow;
    }
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

}  // namespace hclae
