"""What the dependent kernels of sampling and of shared prefixes wait for, by reading
the CUDA sources (no GPU): as test_dependent_launch.py does for the cache's."""
import os
import re

import pytest

from test_dependent_launch import CSRC, declared_read_only, kernels, written

SOURCES = [os.path.join(CSRC, name) for name in ("tq_sample.cu", "tq_share.cu")]
# what the kernels of one call hand over (members of SplitArgs)
HANDED_OVER = ("rows", "part", "winner", "groups", "steps", "list")


def test_the_dependent_kernels_are_found():
    found = {name for path in SOURCES for name, _, body in kernels(path) if "griddep_wait()" in body}
    assert found == {"k_sample_cut", "k_sample_race", "k_sample_finish", "k_share_groups"}


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_what_is_waited_for_is_not_declared_read_only(path):
    every = list(kernels(path))
    for name, params, body in every:
        if "griddep_wait()" in body:
            others = set().union(*(written(p) for other, p, _ in every if other != name))
            assert not declared_read_only(params) & others, name
            assert "__restrict__" not in params, name


def test_nothing_handed_over_is_read_in_front_of_the_wait():
    """In front of it a reference to a row's record may be taken, no more."""
    for name, _, body in kernels(SOURCES[0]):
        if "griddep_wait()" in body:
            front = re.sub(r"RowRecord& rec = q\.rows\[[^\]]*\];", "", body[: body.index("griddep_wait()")])
            assert not re.search(r"q\.(%s)\b|\brec\b" % "|".join(HANDED_OVER), front), name


def test_the_read_only_path_is_taken_for_inputs_alone():
    with open(SOURCES[0]) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert re.findall(r"__ldg\(([^;]*)\);", text) == ["reinterpret_cast<const float4*>(noise + v + i)"]
