// What hclae.hip (arguments, scratch, order of calls) and serve.hip (kernels that serve a paged cache of codes) share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace hclae {

// The rows of a paged cache as its tables name them.
struct PagedRows {
    const int32_t *tables, *lengths;                // [B][max_pages], [B]
    int B, max_pages, page;
    int64_t pages;                                  // of the cache
};

struct AttendArgs {                                 // hclae_cache_attend
    const void *Q;
    int64_t q_row, q_head;                          // strides, elements
    const uint8_t *codes;                           // [slots][2 G][M]
    const float *scale;                             // [slots][2 G] or null
    PagedRows rows;
    const int32_t *begins, *picked;                 // [B] or null; [B][G][n_picked] or null
    int n_picked;
    float factor;
    const float *C;                                 // [2 G][M][K][D]
    int G, R, M, K, D;                              // key heads, query heads of each
    void *out;
    int64_t o_row, o_head;
    float *lse;                                     // [B][G R] or null
};
// Bytes of scratch that the call needs.
size_t attend_scratch(const AttendArgs &a, int type, int cus);
// raised: the kernels whose limit of LDS this ctx has raised, a bit each.
hipError_t attend_launch(const AttendArgs &a, int type, int cus, char *scratch, uint64_t *raised, hipStream_t stream);

struct SelectArgs {                                 // hclae_cache_select
    const void *Q;
    int64_t q_row, q_head;
    const uint8_t *codes;                           // [pages][G][M]
    const float *scale;                             // [pages][G] or null
    PagedRows rows;
    const float *C;                                 // [G][M][K][D]
    int G, R, M, K, D;
    int first, recent, k;
    int32_t *picked;                                // [B][G][k]
};
size_t select_scratch(const SelectArgs &a);
hipError_t select_launch(const SelectArgs &a, int type, char *scratch, uint64_t *raised, hipStream_t stream);

struct PageArgs {                                   // hclae_cache_extend and hclae_cache_compact
    int32_t *tables, *lengths;
    int B, max_pages, page;
    int64_t n_pages;
    // extend
    const int32_t *starts;
    int64_t n;
    int64_t *slots;
    int32_t *src, *dst, *rows;
    // compact: src, dst too
    int32_t *used;
};
size_t extend_scratch(const PageArgs &a);
hipError_t extend_launch(const PageArgs &a, int cus, char *scratch, uint64_t *raised, hipStream_t stream);
size_t compact_scratch(const PageArgs &a);
hipError_t compact_launch(const PageArgs &a, int cus, char *scratch, hipStream_t stream);

struct CopyArgs {                                   // hclae_cache_copy
    uint8_t *codes;
    float *scale;                                   // or null
    int64_t n_pages;
    int page, row_codes, row_scales;                // bytes and floats of a row
    const int32_t *src, *dst, *rows;                // rows: or null
    int64_t n;
};
hipError_t copy_launch(const CopyArgs &a, int cus, hipStream_t stream);

}  // namespace hclae
