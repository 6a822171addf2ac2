"""A word of LDS that a function of the sampler stores to before its first barrier is its own (no GPU needed: the source is read).

find_token clears its `s_found` before any barrier.  A caller that lent it a word which slower waves still test would send these down another
path than the rest of their block, whose barriers then pair wrongly."""
import os
import re

from paper_2506_03887_amd import build


def test_the_word_that_find_token_clears_has_no_other_use():
    with open(os.path.join(build.CSRC, "sample_kernels.hip")) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    lent = re.findall(r"(?:s_part|s\.part_tokens),\s*&(?:s\.)?(\w+)", code)
    assert len(lent) == 4                                    # every call that says which word it is
    for word in set(lent):
        assert len(re.findall(rf"\b{word}\b", code)) == lent.count(word) + 1, f"{word} has uses besides its declaration and find_token's calls"
