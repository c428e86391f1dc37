"""Serving from a paged cache without a GPU: what the calls refuse before any HIP call, and which rows and pages the kernels take, as facts the
compiler checks (tables with bad pages, lengths and picks outside them, rows of no sequence)."""
import os
import subprocess

from paper_1509_05194_amd import build, hclae

CHECKS = r'''
#include "attend.hpp"
#include "pages.hpp"
#include "select.hpp"
using namespace hclae;
// two sequences in tables of three pages of 4 slots, a cache of 6 pages
constexpr int32_t tables[] = {3, 0, 9, 5, -1, 2};
constexpr int32_t lengths[] = {7, 99};
constexpr int32_t begins[] = {2, -5};
constexpr int32_t none_left[] = {7, 12};
constexpr int32_t negative[] = {-1, -2147483647 - 1};
constexpr int32_t picks[] = {1, -1, 0, 7, 2, 2, 1, -2147483647 - 1};
constexpr AttendArgs args(const int32_t *from, const int32_t *picked, int n, const int32_t *l = lengths)
{
    AttendArgs a = {};
    a.rows = {tables, l, 2, 3, 4, 6};
    a.begins = from;
    a.picked = picked;
    a.n_picked = n;
    a.G = 1;
    a.R = 1;
    return a;
}
constexpr SeqRows s0(args(nullptr, nullptr, 0), 0, 0), s1(args(nullptr, nullptr, 0), 1, 0);
static_assert(s0.count == 7 && s0.slot(0) == 12 && s0.slot(3) == 15 && s0.slot(4) == 0 && s0.slot(6) == 2, "pages in the table's order");
static_assert(s1.count == 12 && s1.slot(0) == 20 && s1.slot(4) == kNoRow && s1.slot(7) == kNoRow && s1.slot(11) == 11, "no further than the table, a page below zero");
constexpr SeqRows from2(args(begins, nullptr, 0), 0, 0), from0(args(begins, nullptr, 0), 1, 0);
static_assert(from2.count == 5 && from2.slot(0) == 14 && from2.slot(2) == 0 && from0.count == 12, "from a first row on");
static_assert(SeqRows(args(none_left, nullptr, 0), 0, 0).count == 0 && SeqRows(args(none_left, nullptr, 0), 1, 0).count == 0, "nothing left");
static_assert(SeqRows(args(none_left, picks, 4), 0, 0).count == 0, "nothing to pick from");
static_assert(SeqRows(args(nullptr, nullptr, 0, negative), 0, 0).count == 0 && SeqRows(args(nullptr, nullptr, 0, negative), 1, 0).count == 0, "no length");
constexpr SeqRows p0(args(nullptr, picks, 4), 0, 0), p1(args(begins, picks, 4), 0, 0), p2(args(nullptr, picks, 4), 1, 0);
static_assert(p0.count == 16 && p0.slot(0) == 0 && p0.slot(2) == 2 && p0.slot(3) == kNoRow && p0.slot(5) == kNoRow && p0.slot(8) == 12 && p0.slot(13) == kNoRow, "picked pages");
static_assert(p1.slot(8) == kNoRow && p1.slot(9) == kNoRow && p1.slot(10) == 14, "picked pages from a first row on");
static_assert(p2.slot(0) == 8 && p2.slot(4) == 8 && p2.slot(7) == 11 && p2.slot(8) == kNoRow && p2.slot(15) == kNoRow, "a page twice, a page that is not there");
static_assert(heads_at_once(1) == 1 && heads_at_once(2) == 2 && heads_at_once(3) == 4 && heads_at_once(16) == 4, "query heads of a block");
// growth
constexpr int32_t starts[] = {1, 4, 4, 3, 900};
constexpr int32_t grow[] = {7, 8, -3, 12};
constexpr PageArgs pages(int64_t n)
{
    PageArgs a = {};
    a.lengths = const_cast<int32_t *>(grow);
    a.B = 4;
    a.max_pages = 3;
    a.page = 4;
    a.n_pages = 6;
    a.starts = starts;
    a.n = n;
    return a;
}
constexpr Growth g0(pages(10), 0), g1(pages(10), 1), g2(pages(10), 2), g3(pages(10), 3);
static_assert(g0.first == 1 && g0.add == 3 && g0.length == 7 && g0.old_pages == 2 && g0.new_pages == 3 && g0.fits, "rows of a batch");
static_assert(g1.add == 0 && g2.add == 0 && g2.length == 0, "no rows, rows in no order");
static_assert(g3.first == 3 && g3.add == 7 && g3.new_pages == 5 && !g3.fits, "no further than the batch, a full table");
static_assert(pages_of(0, 4) == 0 && pages_of(1, 4) == 1 && pages_of(4, 4) == 1 && pages_of(5, 4) == 2 && held(13, 3, 4) == 12 && words_of(32) == 1 && words_of(33) == 2, "pages");
'''

KEYS = r'''
#include "select.hpp"
#include <stdio.h>
#include <math.h>
using namespace hclae;
int main()
{
    const double v[] = {-INFINITY, -1e300, -1.0, -0x1p-1074, 0.0, 0x1p-1074, 1e-300, 1.0, 1e300, INFINITY};
    for (int i = 0; i < 10; ++i)
        for (int j = 0; j < 10; ++j)
            if ((v[i] < v[j]) != (score_key(v[i]) < score_key(v[j]))) return 1;
    if (score_key(-0.0) != score_key(0.0) || score_key(NAN) != score_key(-INFINITY) || score_key(-INFINITY) == 0 || score_key(INFINITY) == ~0ull) return 2;
    return 0;
}
'''


def test_which_rows_and_pages(tmp_path):
    src = tmp_path / "rows.hip"
    src.write_text(CHECKS)
    p = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-std=c++17", "--offload-arch=gfx950", "--cuda-host-only",
                        "-fsyntax-only", "-I", build.CSRC, str(src)], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr


def test_keys_sort_as_scores_do(tmp_path):
    src = tmp_path / "keys.hip"
    src.write_text(KEYS)
    exe = tmp_path / "keys"
    p = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-std=c++17", "-O1", "--offload-arch=gfx950", "-I", build.CSRC, "-o", str(exe), str(src)],
                       capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr
    assert subprocess.run([str(exe)], timeout=60).returncode == 0


def test_null_ctx_is_einval():
    L = hclae.lib()
    assert L.hclae_cache_attend(None, None, 0, 1, 1, 16, 16, None, None, 0, None, 0, 1, None, None, None, 0, 1.0, None, 16, 16, None) == hclae.EINVAL
    assert L.hclae_cache_select(None, None, 0, 1, 1, 16, 16, None, None, 0, None, 0, 1, None, 0, 0, 1, None) == hclae.EINVAL
    assert L.hclae_cache_extend(None, None, None, 0, 0, 1, 0, None, 0, None, None, None, None) == hclae.EINVAL
    assert L.hclae_cache_compact(None, None, None, 0, 0, 1, 0, None, None, None) == hclae.EINVAL
    assert L.hclae_cache_copy(None, None, None, 0, 1, None, None, None, 0) == hclae.EINVAL
