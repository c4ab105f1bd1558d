"""What the cache's and verification's dependent kernels wait for, by reading the
CUDA sources (no GPU).  A kernel with griddep_wait may be resident while the
one in front of it still writes.  What that one writes must not be declared
read-only for the dependent's whole life (const with __restrict__): the compiler
could then take the read-only path, or move the load in front of the wait."""
import glob
import os
import re

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2607_16973_gb300", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "tq_kv*.cu*")) + [os.path.join(CSRC, "tq_verify.cu")])


def kernels(path):
    """(name, parameters, body) of the kernels in a source."""
    with open(path) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    for m in re.finditer(r"__global__[^;{]*?void\s+(\w+)\(", text):
        depth, at = 1, m.end()
        while depth:  # the parameters' closing bracket
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        params, begin = text[m.end(): at - 1], text.index("{", at)
        depth, at = 1, begin + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        yield m.group(1), params, text[begin: at]


def declared_read_only(params):
    return set(re.findall(r"const\s+\w+\s*\*\s*__restrict__\s+(\w+)", params))


def written(params):
    """Pointers to what a kernel may write."""
    return {m.group(2) for p in params.split(",") if (m := re.match(r"\s*(\w+)\s*\*\s*(?:__restrict__\s+)?(\w+)\s*$", p))}


def test_the_dependent_kernels_are_found():
    found = {name for path in SOURCES for name, _, body in kernels(path) if "griddep_wait()" in body}
    assert found == {"k_kv_join", "k_kv_copy_parts", "k_kv_move", "k_kv_rename", "k_verify_finish"}


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_what_is_waited_for_is_not_declared_read_only(path):
    every = list(kernels(path))
    for name, params, body in every:
        if "griddep_wait()" in body:
            others = set().union(*(written(p) for other, p, _ in every if other != name))
            assert not declared_read_only(params) & others, name
