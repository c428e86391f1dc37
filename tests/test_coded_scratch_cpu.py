"""What a context keeps for coded caches and tables, without a GPU: who frees it, how much there is of it."""
import os
import re
import subprocess

from paper_1509_05194_amd import build


def body(name):
    """The text of a function of hclae.hip, from its name to the brace in the first column."""
    text = open(os.path.join(build.CSRC, "hclae.hip")).read()
    found = re.findall(r"^(?:static )?\w+ %s\([^;{]*\)\n\{\n(.*?)^\}" % name, text, flags=re.S | re.M)
    assert len(found) == 1, name
    return found[0]


def test_growing_the_multi_path_scratch_frees_nothing_else():
    """hclae_encode_beam and hclae_beam_step free and allocate their arrays again when a call needs more; the dictionaries of a cache and the
    rows of a gradient live on until hclae_destroy."""
    text = body("beam_release")
    freed = re.findall(r"ctx->(\w+(?:\[\d\])?)", re.search(r"dev\[\] = \{(.*?)\};", text, flags=re.S).group(1))
    assert freed and all(f.startswith("beam_") for f in freed), freed
    cleared = re.findall(r"ctx->(\w+(?:\[\d\])?) = (?=[^;]*nullptr)", text)
    assert sorted(cleared) == sorted(freed)                # nothing is freed twice
    at_the_end = re.findall(r"ctx->(\w+(?:\[\d\])?)", re.search(r"dev\[\] = \{(.*?)\};", body("hclae_destroy"), flags=re.S).group(1))
    assert len(set(at_the_end)) == len(at_the_end)
    assert set(freed) | {"cache_C", "cache_T", "cache_buf", "grad_buf"} <= set(at_the_end)


ROOM = r'''
#include "lookup_grad.hpp"
using namespace hclae;
// A step of the chunk ends at a multiple of 512 waves of rows, a step of the range at a power of two: the most items and ranges are there.
constexpr bool every(int64_t first, int64_t last)
{
    const int64_t step = (int64_t)kGradItems * kWave, most = (1ll << 31) - 1;
    for (int64_t j = first; j <= last; ++j)
        for (int64_t T = j * step - 1; T <= j * step + 1; ++T) {
            if (T <= kGradFew || T > most) continue;
            const GradPlan p = grad_plan(T, 256);
            // alone, and in a context with room for more: where the range changes, and for all there can be
            const int64_t rooms[] = {T, T + 1, 32768, 32769, 131072, 131073, 524288, 524289, most};
            for (int64_t N : rooms)
                if (N >= T && N <= most && !fits(p, grad_room(N, 256))) return false;
            if (p.chunk % kWave || p.chunk < 2 * kWave || (int64_t)p.range * p.ranges < T || (p.max_items - 256) > kGradItems) return false;
        }
    return true;
}
static_assert(every(0, 8192), "to 2^28 rows");
static_assert(every(65536 - 4096, 65536), "the last rows there are");
// any other number of rows there: no step is passed over
constexpr bool dense(int64_t from, int64_t to)
{
    for (int64_t T = from; T < to; ++T)
        if (!fits(grad_plan(T, 256), grad_room(T, 256))) return false;
    return true;
}
static_assert(dense(kGradFew + 1, 270000), "the first steps");
// codewords of n_k rows each: the items and partial sums that k_grad_items lays out
constexpr bool laid_out(int64_t T, int K)
{
    const GradPlan p = grad_plan(T, K);
    for (int shape = 0; shape < 4; ++shape) {
        int64_t items = 0, parts = 0, left = T;
        for (int k = 0; k < K; ++k) {
            // evenly; one row beyond a chunk each; all in one; one chunk each
            int64_t n = shape == 0 ? T / K : shape == 1 ? p.chunk + 1 : shape == 2 ? T : p.chunk;
            if (n > left || k == K - 1) n = left;
            left -= n;
            const int64_t i = n > p.chunk ? (n + p.chunk - 1) / p.chunk : 1;
            items += i;
            parts += i > 1 ? i : 0;
        }
        if (items > p.max_items || parts > p.max_parts) return false;
    }
    return true;
}
static_assert(laid_out(4097, 256) && laid_out(65663, 256) && laid_out(65664, 256) && laid_out(66047, 256) && laid_out(98815, 64) && laid_out(131583, 256) &&
              laid_out(700001, 3) && laid_out((1ll << 31) - 1, 256) && laid_out(66047, 1), "items");
'''


def test_the_gradients_scratch_has_room_for_every_number_of_rows(tmp_path):
    src = tmp_path / "room.hip"
    src.write_text(ROOM)
    p = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-std=c++17", "--offload-arch=gfx950", "--cuda-host-only", "-fconstexpr-steps=200000000",
                        "-fsyntax-only", "-I", build.CSRC, str(src)], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr
