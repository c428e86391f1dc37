// Launches of the kernels that serve a paged cache of codes: attention, the choice of pages, and the pages themselves.  Arguments have
// been checked by the entry points in hclae.hip; scratch is theirs.
#include <algorithm>

#include "attend.hpp"
#include "pages.hpp"
#include "select.hpp"
#include "serve.hpp"

namespace hclae {

namespace {

constexpr int kServeLds = 156 * 1024;               // LDS that a kernel asks for at its launch; the rest of a workgroup's 160 KB is for what it declares

size_t up(size_t bytes) { return (bytes + 255) / 256 * 256; }

#define TRY(call)                         \
    do {                                  \
        const hipError_t e__ = (call);    \
        if (e__ != hipSuccess) return e__; \
    } while (0)

template <typename K>
hipError_t raise_lds(K kern, int bit, uint64_t *raised, int bytes = kServeLds)
{
    if (*raised >> bit & 1u) return hipSuccess;
    TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    *raised |= 1ull << bit;
    return hipSuccess;
}

constexpr int kPickLds = 136 * 1024;                // as above: k_select_pages declares 20 KB

enum RaisedBit { kRaisedSelect = 0, kRaisedCodes = 1, kRaisedOut = 36, kRaisedPages = 54 };         // 35 from kRaisedCodes on, 18 from kRaisedOut on

// ---- attention ----------------------------------------------------------------------------------

int64_t direct_jobs(const AttendArgs &a, int splits)
{
    const int RB = heads_at_once(a.R);
    return (int64_t)a.rows.B * a.G * ((a.R + RB - 1) / RB) * splits;
}

template <typename T, int RB>
hipError_t launch_direct(const AttendArgs &a, int splits, char *scratch, hipStream_t stream)
{
    const int64_t jobs = direct_jobs(a, splits);
    PartStat *stats = reinterpret_cast<PartStat *>(scratch);
    float *sums = reinterpret_cast<float *>(scratch + up(sizeof(PartStat) * jobs * RB));
    hipLaunchKernelGGL((k_attend_rows<T, RB>), dim3((unsigned)jobs), dim3(kDirectThreads), 0, stream, a, splits, stats, sums);
    TRY(hipGetLastError());
    hipLaunchKernelGGL((k_attend_join<T, RB>), dim3((unsigned)(a.rows.B * a.G * a.R)), dim3(kWave), 0, stream, a, splits, (const PartStat *)stats, (const float *)sums);
    return hipGetLastError();
}

// The sequences of a call are taken in rounds, which bounds its scratch and its grids.
constexpr int64_t kAttendRound = 1 << 14;           // query heads of a round, of all its sequences
int attend_round(const AttendArgs &a) { return (int)std::max<int64_t>(1, std::min<int64_t>(a.rows.B, kAttendRound / ((int64_t)a.G * a.R))); }
AttendArgs round_of(const AttendArgs &a, int b0, int n, int bytes)
{
    AttendArgs r = a;
    r.Q = static_cast<const char *>(a.Q) + (int64_t)b0 * a.q_row * bytes;
    r.out = static_cast<char *>(a.out) + (int64_t)b0 * a.o_row * bytes;
    r.rows.tables += (int64_t)b0 * a.rows.max_pages;
    r.rows.lengths += b0;
    r.rows.B = n;
    if (a.begins) r.begins += b0;
    if (a.picked) r.picked += (int64_t)b0 * a.G * a.n_picked;
    if (a.lse) r.lse += (int64_t)b0 * a.G * a.R;
    return r;
}

// Whether the rows go through tables: not where a sequence can have few rows only, which are decoded before the tables are there, unless there are many such
// sequences.  G = 8, R = 4, D = 128, K = 256, bf16 in pages of 16, us decoded and through tables, in a graph: one sequence, M = 8, 64 rows 15.8 and 22.9, 128 rows 16.6 and
// 23.1, 256 rows 19.1 and 23.3, 384 rows 23.7 and 24.1, 512 rows 28.8 and 24.6, 2048 rows 63 and 27; M = 16, 128 rows 23.0 and 33.5, 256 rows 35.8 and 34.3; R = 1, 256 rows 16.6
// and 19.4, 384 rows 20.2 and 20.0; fp32, 256 rows 18.9 and 25.2, 384 rows 23.6 and 25.5, 512 rows 28.9 and 26.5; K = 64, 256 rows 18.9 and 19.8, 384 rows 21.4 and 21.1.
// 32 sequences, M = 8, 64 rows 27.9 and 42.1, 128 rows 43.2 and 41.6, 2048 rows 481 and 49.
constexpr int64_t kFewRows = 400, kFewInAll = 96 * 256;
CodesPlan plan_of(const AttendArgs &a, int type)
{
    const int64_t rows = attend_capacity(a) * std::max(8, a.M) / 8, RB = heads_at_once(a.R);
    if (rows <= kFewRows && rows * a.rows.B * a.G * ((a.R + RB - 1) / RB) <= kFewInAll) return {0, false, 0, 0};
    return codes_plan(a.R, a.M, a.K, type == kRowF32);
}

int splits_of(const AttendArgs &a, const CodesPlan &plan, int cus)
{
    return codes_splits(a, plan.RB, codes_threads(plan.RB, plan.wide, a.M <= 8 ? 2 : a.M <= 16 ? 4 : 8) == 512 ? 2 : 1, cus);
}

struct CodesRoom {
    size_t tab, stats, sums, joined;
};
CodesRoom codes_room(const AttendArgs &a, const CodesPlan &plan, int splits)
{
    const int64_t seqs = (int64_t)a.rows.B * a.G * ((a.R + plan.RB - 1) / plan.RB), rows = seqs * splits * plan.RB;
    return {up(sizeof(float) * seqs * tab_row(a.M, a.K, plan.RB)), up(sizeof(CodesStat) * rows), up(sizeof(float) * rows * sums_row(a.M, a.K)), up(sizeof(CodesStat) * seqs * plan.RB)};
}

template <int RB, bool WIDE, int MW, bool FULL, bool BY_WAVE>
hipError_t launch_codes_as(const AttendArgs &a, const CodesPlan &plan, const CodesArgs &x, uint64_t *raised, hipStream_t stream)
{
    constexpr int bit = kRaisedCodes + (BY_WAVE ? 25 : FULL ? 15 : 0) + (MW == 2 ? 0 : MW == 4 ? 5 : 10) + (RB == 1 ? 0 : RB == 2 ? 1 : 3) + (RB > 1 && WIDE ? 1 : 0);
    auto kern = &k_attend_codes<RB, WIDE, MW, FULL, BY_WAVE>;
    TRY(raise_lds(kern, bit, raised));
    const int64_t heads = (int64_t)a.G * ((a.R + RB - 1) / RB), units = (int64_t)a.rows.B * x.splits;
    hipLaunchKernelGGL(kern, dim3((unsigned)((x.grouped ? (units + 7) / 8 * 8 : units) * heads)), dim3(codes_threads(RB, WIDE, MW)), plan.lds, stream, a, x);
    return hipGetLastError();
}
template <int RB, bool WIDE, int MW>
hipError_t launch_codes(const AttendArgs &a, const CodesPlan &plan, int splits, const float *tab, CodesStat *stats, float *sums, uint64_t *raised, hipStream_t stream)
{
    const int64_t row = 2ll * a.G * a.M;
    const CodesArgs x = {splits, (int64_t)a.rows.B * splits >= 32, a.M % 4 == 0 && reinterpret_cast<uintptr_t>(a.codes) % 4 == 0,
                         a.rows.page < 1 << 24 && a.rows.page * row < (int64_t)1 << 32, tab, stats, sums};
    if constexpr (MW <= 4) {
        if (a.K == 256 && a.M == 4 * MW && x.words)
            return a.rows.page % kWave == 0 && !a.begins ? launch_codes_as<RB, WIDE, MW, true, true>(a, plan, x, raised, stream)
                                                         : launch_codes_as<RB, WIDE, MW, true, false>(a, plan, x, raised, stream);
    }
    return launch_codes_as<RB, WIDE, MW, false, false>(a, plan, x, raised, stream);
}

template <typename T, int RB>
hipError_t launch_through_tables(const AttendArgs &a, const CodesPlan &plan, int cus, char *scratch, uint64_t *raised, hipStream_t stream)
{
    const int splits = splits_of(a, plan, cus);
    const CodesRoom room = codes_room(a, plan, splits);
    float *tab = reinterpret_cast<float *>(scratch);
    CodesStat *stats = reinterpret_cast<CodesStat *>(scratch + room.tab);
    float *sums = reinterpret_cast<float *>(scratch + room.tab + room.stats);
    const int tiles = (a.rows.B * ((a.R + RB - 1) / RB) * RB + 15) / 16, groups = a.G * ((a.M * a.K + 63) / 64);
    constexpr int N = T::bytes == 4 ? 3 : __is_same(T, F16) ? 2 : 1;    // bf16 parts of a query
    auto tables = a.D <= 64 ? &k_attend_tables<T, RB, 2, N> : a.D <= 128 ? &k_attend_tables<T, RB, 4, N> : &k_attend_tables<T, RB, 8, N>;
    const int queries = table_queries(N, a.D <= 64 ? 2 : a.D <= 128 ? 4 : 8), stages = (a.rows.B * ((a.R + RB - 1) / RB) * RB + queries - 1) / queries;
    const dim3 grid((unsigned)groups, (unsigned)std::max(1, std::min(stages, (4 * cus + groups - 1) / groups)));
    hipLaunchKernelGGL(tables, grid, dim3(kTableThreads), 0, stream, a, stages, tab);
    TRY(hipGetLastError());
    const int mw = a.M <= 8 ? 2 : a.M <= 16 ? 4 : 8;
#define CODES(WIDE, MW) TRY((launch_codes<RB, WIDE, MW>(a, plan, splits, tab, stats, sums, raised, stream)))
    if constexpr (RB > 1) {
        if (!plan.wide) {
            if (mw == 2) CODES(false, 2);
            else if (mw == 4) CODES(false, 4);
            else CODES(false, 8);
        }
    }
    if (plan.wide) {
        if (mw == 2) CODES(true, 2);
        else if (mw == 4) CODES(true, 4);
        else CODES(true, 8);
    }
#undef CODES
    int parts = splits;
    if (splits >= kFoldFrom) {                      // the first parts' sums are those of all then
        const int64_t rows = (int64_t)a.rows.B * a.G * ((a.R + RB - 1) / RB) * RB;
        CodesStat *joined = reinterpret_cast<CodesStat *>(scratch + room.tab + room.stats + room.sums);
        hipLaunchKernelGGL(k_attend_fold<RB>, dim3((unsigned)rows, (unsigned)((sums_row(a.M, a.K) / 4 + kFoldThreads - 1) / kFoldThreads)), dim3(kFoldThreads), 0, stream, a, splits,
                           (const CodesStat *)stats, sums, joined);
        TRY(hipGetLastError());
        stats = joined;
        parts = 1;
    }
    // 64 coordinates a block where that leaves enough of them
    const bool wide = (int64_t)tiles * a.G * ((a.D + 63) / 64) >= cus / 2;
    const int slices = (a.D + (wide ? 63 : 15)) / (wide ? 64 : 16);
    auto out = wide ? &k_attend_out<T, RB, 4> : &k_attend_out<T, RB, 1>;
    TRY(raise_lds(out, kRaisedOut + (wide ? 1 : 0) + 2 * (RB == 1 ? 0 : RB == 2 ? 1 : 2) + 6 * (T::bytes == 4 ? 0 : __is_same(T, F16) ? 1 : 2), raised));
    hipLaunchKernelGGL(out, dim3((unsigned)((tiles * a.G * slices + 7) / 8 * 8)), dim3(kOutThreads), (size_t)out_lds(wide ? 4 : 1), stream, a, parts, splits, tiles, (const CodesStat *)stats,
                       (const float *)sums);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_attend(const AttendArgs &a, int type, int cus, char *scratch, uint64_t *raised, hipStream_t stream)
{
    const CodesPlan plan = plan_of(a, type);
    switch (plan.RB) {
    case 1: return launch_through_tables<T, 1>(a, plan, cus, scratch, raised, stream);
    case 2: return launch_through_tables<T, 2>(a, plan, cus, scratch, raised, stream);
    case 4: return launch_through_tables<T, 4>(a, plan, cus, scratch, raised, stream);
    }
    const int splits = direct_splits(a, cus);
    switch (heads_at_once(a.R)) {
    case 1: return launch_direct<T, 1>(a, splits, scratch, stream);
    case 2: return launch_direct<T, 2>(a, splits, scratch, stream);
    default: return launch_direct<T, 4>(a, splits, scratch, stream);
    }
}

// ---- the choice of pages ------------------------------------------------------------------------

// As with attention, in rounds: at most 256 MB of tables and keys.
int select_round(const SelectArgs &a)
{
    const int64_t each = 8ll * a.G * ((int64_t)a.M * a.K + a.rows.max_pages);
    return (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)a.rows.B, (256ll << 20) / each, (int64_t)(1 << 18) / a.G}));
}
SelectArgs round_of(const SelectArgs &a, int b0, int n, int bytes)
{
    SelectArgs r = a;
    r.Q = static_cast<const char *>(a.Q) + (int64_t)b0 * a.q_row * bytes;
    r.rows.tables += (int64_t)b0 * a.rows.max_pages;
    r.rows.lengths += b0;
    r.rows.B = n;
    r.picked += (int64_t)b0 * a.G * a.k;
    return r;
}

size_t table_bytes(const SelectArgs &a) { return up(sizeof(double) * (size_t)a.rows.B * a.G * a.M * a.K); }

template <typename T>
hipError_t launch_select(const SelectArgs &a, char *scratch, uint64_t *raised, hipStream_t stream)
{
    double *tab = reinterpret_cast<double *>(scratch);
    uint64_t *keys = reinterpret_cast<uint64_t *>(scratch + table_bytes(a));
    hipLaunchKernelGGL(k_select_tables<T>, dim3((unsigned)(a.G * ((a.M * a.K + 63) / 64) * ((a.rows.B + kSelectSeqs - 1) / kSelectSeqs))), dim3(kSelectThreads), 0, stream, a, tab);
    TRY(hipGetLastError());
    const size_t lds = pick_lds(a.M, a.K, a.rows.max_pages);
    const dim3 grid((unsigned)(a.rows.B * a.G));
    if (lds <= (size_t)kPickLds) {
        TRY(raise_lds(&k_select_pages<true>, kRaisedSelect, raised, kPickLds));
        hipLaunchKernelGGL(k_select_pages<true>, grid, dim3(kPickThreads), lds, stream, a, (const double *)tab, keys);
    } else {
        hipLaunchKernelGGL(k_select_pages<false>, grid, dim3(kPickThreads), 0, stream, a, (const double *)tab, keys);
    }
    return hipGetLastError();
}

// ---- pages --------------------------------------------------------------------------------------

size_t bitmap_bytes(const PageArgs &a) { return up(4 * (size_t)words_of(a.n_pages)); }

dim3 table_blocks(const PageArgs &a, int cus)
{
    const int64_t jobs = (int64_t)a.B * table_chunks(a.max_pages);
    return dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(jobs, 8ll * cus)));
}

// Bitmaps at the front of the scratch: pages named once or more and, if twice, pages named twice or more.
hipError_t launch_marks(const PageArgs &a, bool twice, int cus, char *scratch, hipStream_t stream)
{
    const int64_t words = (int64_t)((twice ? 2 : 1) * bitmap_bytes(a) / 4);
    hipLaunchKernelGGL(k_pages_clear, dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>((words + kPageThreads - 1) / kPageThreads, 8ll * cus))), dim3(kPageThreads), 0, stream,
                       reinterpret_cast<unsigned *>(scratch), words);
    TRY(hipGetLastError());
    hipLaunchKernelGGL(k_pages_mark, table_blocks(a, cus), dim3(kPageThreads), 0, stream, a, reinterpret_cast<unsigned *>(scratch),
                       twice ? reinterpret_cast<unsigned *>(scratch + bitmap_bytes(a)) : nullptr);
    return hipGetLastError();
}

// Pages that the sequences of a call can ask for: each the copy of its last one, and a page begun and those that its rows fill.
size_t extend_room(const PageArgs &a) { return (size_t)std::min<int64_t>(a.n_pages, 2ll * a.B + a.n / a.page); }

}  // namespace

size_t attend_scratch(const AttendArgs &a, int type, int cus)
{
    size_t most = 0;
    for (int n : {attend_round(a), a.rows.B % attend_round(a)}) {   // whole rounds, and the last one
        if (n == 0) continue;
        const AttendArgs r = round_of(a, 0, n, 0);
        const CodesPlan plan = plan_of(r, type);
        if (plan.RB) {
            const CodesRoom room = codes_room(r, plan, splits_of(r, plan, cus));
            most = std::max(most, room.tab + room.stats + room.sums + room.joined);
            continue;
        }
        const int RB = heads_at_once(r.R);
        const int64_t jobs = direct_jobs(r, direct_splits(r, cus));
        most = std::max(most, up(sizeof(PartStat) * jobs * RB) + up(sizeof(float) * jobs * RB * r.D));
    }
    return most;
}

hipError_t attend_launch(const AttendArgs &a, int type, int cus, char *scratch, uint64_t *raised, hipStream_t stream)
{
    const int step = attend_round(a);
    for (int b0 = 0; b0 < a.rows.B; b0 += step) {
        const AttendArgs r = round_of(a, b0, std::min(step, a.rows.B - b0), type == kRowF32 ? 4 : 2);
        TRY(type == kRowF32 ? launch_attend<F32>(r, type, cus, scratch, raised, stream) : type == kRowF16 ? launch_attend<F16>(r, type, cus, scratch, raised, stream)
                                                                                                  : launch_attend<Bf16>(r, type, cus, scratch, raised, stream));
    }
    return hipSuccess;
}

size_t select_scratch(const SelectArgs &a)
{
    const SelectArgs r = round_of(a, 0, select_round(a), 0);
    return table_bytes(r) + up(sizeof(uint64_t) * (size_t)r.rows.B * r.G * r.rows.max_pages);
}

hipError_t select_launch(const SelectArgs &a, int type, char *scratch, uint64_t *raised, hipStream_t stream)
{
    const int step = select_round(a);
    for (int b0 = 0; b0 < a.rows.B; b0 += step) {
        const SelectArgs r = round_of(a, b0, std::min(step, a.rows.B - b0), type == kRowF32 ? 4 : 2);
        TRY(type == kRowF32 ? launch_select<F32>(r, scratch, raised, stream) : type == kRowF16 ? launch_select<F16>(r, scratch, raised, stream)
                                                                                             : launch_select<Bf16>(r, scratch, raised, stream));
    }
    return hipSuccess;
}

size_t extend_scratch(const PageArgs &a)
{
    if (extend_in_block(a, (int64_t)extend_room(a))) return 0;
    return 2 * bitmap_bytes(a) + up(4 * (size_t)a.B) + up(4 * extend_room(a)) + 256;
}

hipError_t extend_launch(const PageArgs &a, int cus, char *scratch, uint64_t *raised, hipStream_t stream)
{
    if (extend_in_block(a, (int64_t)extend_room(a))) {
        TRY(raise_lds(&k_extend_block, kRaisedPages, raised));
        hipLaunchKernelGGL(k_extend_block, dim3(1), dim3(kPlanThreads), (size_t)extend_lds(a, (int64_t)extend_room(a)), stream, a, (unsigned)extend_room(a));
        return hipGetLastError();
    }
    TRY(launch_marks(a, true, cus, scratch, stream));
    ExtendScratch s;
    char *p = scratch;
    s.used = reinterpret_cast<unsigned *>(p);
    s.shared = reinterpret_cast<unsigned *>(p += bitmap_bytes(a));
    s.upto = reinterpret_cast<unsigned *>(p += bitmap_bytes(a));
    s.free = reinterpret_cast<unsigned *>(p += up(4 * (size_t)a.B));
    s.found = reinterpret_cast<unsigned *>(p += up(4 * extend_room(a)));
    s.room = (unsigned)extend_room(a);
    hipLaunchKernelGGL(k_extend_plan, dim3(1), dim3(kPlanThreads), 0, stream, a, s);
    TRY(hipGetLastError());
    hipLaunchKernelGGL(k_extend_rows, dim3((unsigned)std::max(1, std::min((a.B + 3) / 4, 1 << 16))), dim3(kPageThreads), 0, stream, a, s);
    return hipGetLastError();
}

size_t compact_scratch(const PageArgs &a) { return a.n_pages > 0 && compact_in_block(a) ? 0 : 2 * bitmap_bytes(a); }

hipError_t compact_launch(const PageArgs &a, int cus, char *scratch, hipStream_t stream)
{
    if (a.n_pages > 0 && compact_in_block(a)) {
        hipLaunchKernelGGL(k_compact_block, dim3(1), dim3(kPlanThreads), (size_t)(8 * words_of(a.n_pages) + 4 * (int64_t)a.B), stream, a);
        return hipGetLastError();
    }
    TRY(launch_marks(a, false, cus, scratch, stream));
    CompactScratch s = {reinterpret_cast<unsigned *>(scratch), reinterpret_cast<unsigned *>(scratch + bitmap_bytes(a))};
    hipLaunchKernelGGL(k_compact_plan, dim3(1), dim3(kPlanThreads), 0, stream, a, s);
    TRY(hipGetLastError());
    const int64_t entries = (int64_t)a.B * a.max_pages;
    if (a.n_pages == 0 || entries == 0) return hipSuccess;
    hipLaunchKernelGGL(k_compact_tables, table_blocks(a, cus), dim3(kPageThreads), 0, stream, a, s);
    return hipGetLastError();
}

hipError_t copy_launch(const CopyArgs &a, int cus, hipStream_t stream)
{
    // a block about 4 KB of codes
    const int64_t bytes = (int64_t)a.page * a.row_codes;
    const int parts = (int)std::max<int64_t>(1, std::min<int64_t>({(bytes + 4095) / 4096, (int64_t)a.page, (int64_t)64}));
    hipLaunchKernelGGL(k_pages_copy, dim3((unsigned)std::min<int64_t>(a.n * parts, 1 << 20)), dim3(kPageThreads), 0, stream, a, parts);
    return hipGetLastError();
}

}  // namespace hclae
