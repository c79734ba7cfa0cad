"""Shared memory that is read in wider words than its type is declared with their alignment, checked in the source."""
import os
import re

from test_launch_rules import CSRC, _strip_comments


def test_keys_read_in_fours_are_aligned_for_it():
    text = _strip_comments(open(os.path.join(CSRC, "mwu_adapters.cu")).read())
    assert "reinterpret_cast<const int4 *>(&o->key[j])" in text
    assert re.search(r"struct Sorter \{\s*alignas\(16\) int key\[", text)
