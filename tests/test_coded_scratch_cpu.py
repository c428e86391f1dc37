"""What a context keeps for coded caches and tables, without a GPU: who frees it, how much there is of it."""
import os
import re

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
