"""How the cache's kernels reach what is only 4-byte aligned (no GPU needed): weights and positions may start anywhere, so
several of them at a time go through a type that says so."""
import glob
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_09244_amd", "csrc")


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "cache_*.hip"))), ids=os.path.basename)
def test_no_aligned_wide_access_of_weights_and_positions(path):
    src = open(path).read()
    names = set(re.findall(r"(\w+) = \w+\.(?:weight|pos) \+", src))    # pointers that are made from them
    for as_type, operand in re.findall(r"reinterpret_cast<(?:const )?(\w+)\s*\*>\(&?([^;]*?)\)", src):
        start = operand.split("+")[0]
        reached = re.search(r"\.(weight|pos)\b", start) or names & set(re.findall(r"(?<![.\w])\w+", start))
        assert not reached or not re.match(r"(float|int|uint|double)[24]$", as_type), (as_type, operand)


def test_the_header_says_what_is_checked():
    text = " ".join(open(os.path.join(ROOT, "include", "mvla.h")).read().replace("*", " ").split())
    assert "k, v, k_scale, v_scale 16-byte aligned, pos and weight 4-byte aligned" in text
    api = open(os.path.join(CSRC, "api.hip")).read()
    assert "!aligned(c->pos, 4) || !aligned(c->weight, 4)" in api
