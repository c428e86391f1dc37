"""Coded caches and tables without a GPU: what the calls refuse before any HIP call, and where the kernels look for a row's
codes, as facts the compiler checks (tables with bad pages, sequences beyond their pages, starts in any order)."""
import os
import subprocess

from paper_1509_05194_amd import build, hclae

CHECKS = r'''
#include "decode.hpp"
#include "cache_write.hpp"
using namespace hclae;
// two sequences of 5 and 7 rows, an empty one between them, pages of 4 slots, a cache of 6 pages
constexpr int32_t tables[] = {3, 0, 9, 9, 9, 9, 5, -1, 6};
constexpr int32_t starts[] = {0, 5, 5, 12};
constexpr CacheRows cache{tables, starts, 3, 3, 4, 6};
static_assert(cache.at(0) == 12 && cache.at(3) == 15 && cache.at(4) == 0, "pages in the table's order, the last one not full");
static_assert(cache.at(5) == 20 && cache.at(8) == 23, "an empty sequence has no rows");
static_assert(cache.at(9) == kNoRow && cache.at(11) == kNoRow, "a page below zero");
static_assert(cache.at(12) == kSkip && cache.at(1 << 30) == kSkip, "behind the last sequence");
// a page beyond the cache; a sequence with more rows than its pages hold
constexpr int32_t long_starts[] = {0, 40};
constexpr int32_t long_table[] = {5, 6};
constexpr CacheRows longer{long_table, long_starts, 1, 2, 4, 6};
static_assert(longer.at(3) == 23 && longer.at(4) == kNoRow && longer.at(8) == kNoRow && longer.at(39) == kNoRow, "out of range");
constexpr CacheRows no_pages{nullptr, long_starts, 1, 0, 4, 6};
static_assert(no_pages.at(0) == kNoRow, "no table");
// starts that do not begin at zero, or are in no order: a row of some sequence, zeros or nothing, but never outside the table
constexpr int32_t late[] = {3, 5};
static_assert(CacheRows{long_table, late, 1, 2, 4, 6}.at(2) == kSkip && CacheRows{long_table, late, 1, 2, 4, 6}.at(3) == 20, "late");
constexpr int32_t mixed[] = {0, 9, 2, -7, 11};
constexpr int32_t four[] = {0, 1, 2, 3};
constexpr bool inside()
{
    for (int t = -3; t < 14; ++t) {
        const int64_t r = CacheRows{four, mixed, 4, 1, 4, 6}.at(t);
        if (r != kSkip && r != kNoRow && (r < 0 || r >= 24)) return false;
    }
    return true;
}
static_assert(inside(), "any starts");
constexpr bool quotients()
{
    const int pages[] = {1, 2, 3, 5, 7, 16, 24, 641, 65535, 65537, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, 0x7ffffffe, 0x7fffffff};
    for (int page : pages)
        for (int64_t i = 0; i < 9; ++i) {
            const int64_t q = (0x7fffffffll / page) * i / 8;        // multiples over the range, and what is next to them
            for (int64_t x = q * page - 2; x <= q * page + 2; ++x)
                if (x >= 0 && x <= 0x7fffffff && (int64_t)((uint64_t)x * page_mul(page) >> (31 + page_shift(page))) != x / page) return false;
        }
    return true;
}
static_assert(quotients(), "pos / page");
// rows of a table
constexpr int64_t rows[] = {2, -1, 7, 6, 1ll << 40, -(1ll << 62)};
constexpr TableRows table{rows, 7};
static_assert(table.at(0) == 2 && table.at(1) == kNoRow && table.at(2) == kNoRow && table.at(3) == 6 && table.at(4) == kNoRow && table.at(5) == kNoRow, "rows");
static_assert(TableRows{nullptr, 7}.at(6) == 6 && TableRows{nullptr, 7}.at(7) == kNoRow, "all rows");
static_assert(few_columns(1) == 64 && few_columns(64) == 64 && few_columns(65) == 128 && few_columns(129) == 256 && few_columns(256) == 256, "columns");
'''


def test_where_rows_are(tmp_path):
    src = tmp_path / "rows.hip"
    src.write_text(CHECKS)
    p = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-std=c++17", "--offload-arch=gfx950", "--cuda-host-only",
                        "-fsyntax-only", "-I", build.CSRC, str(src)], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr


def test_null_ctx_is_einval():
    L = hclae.lib()
    assert L.hclae_cache_begin(None, None, 1, 4, 16, 16) == hclae.EINVAL
    assert L.hclae_cache_write(None, None, 0, 0, 16, 16, None, 0, None, None) == hclae.EINVAL
    assert L.hclae_cache_read(None, None, None, 0, None, 0, 0, 1, None, 0, None, 0, 16, 16) == hclae.EINVAL
    assert L.hclae_lookup(None, None, 0, None, 0, 1.0, None, 4, 16, 16, None, 0, 16) == hclae.EINVAL
    assert L.hclae_lookup_grad(None, None, 0, None, 0, 1.0, None, 0, 16, 4, 16, 16, None) == hclae.EINVAL
