"""The cut of attention's work into runs, on the CPU (kv_runs.cpp): every block
of tokens that a tile of rows sees is taken once, whatever order a block's
warps run in, and the runs that share an item are the ones that are joined."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from conftest import ROOT
from paper_2607_16973_gb300 import build

CSRC = os.path.join(ROOT, "paper_2607_16973_gb300", "csrc")
ROWS, BLOCK = {"stream8": 8, "stream16": 16, "tile": 256}, {"stream8": 16, "stream16": 16, "tile": 128}

# The headers that the cut needs are compiled as they are; of tq_topk.cuh, which is device code throughout, these names.
TOPK = """#pragma once
#include <cuda_runtime.h>
namespace tq { namespace {
constexpr unsigned FULL = 0xffffffffu;
inline void griddep_wait() {}
template <typename... P, typename... A>
cudaError_t launch_maybe_pdl(bool, void (*)(P...), dim3, dim3, size_t, cudaStream_t, A...);
} }
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv_runs")
    for name in ("tq_kv_attend.cuh", "tq_kv.cuh", "tq_kv.h"):
        shutil.copy(os.path.join(CSRC, name), d)
    (d / "tq_topk.cuh").write_text(TOPK)
    for name in ("tq_internal.h", "tq_kernels.h"):
        (d / name).write_text(f'#include "{os.path.join(CSRC, name)}"\n')
    exe = d / "kv_runs"
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build._nvcc()))), "include")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fwrapv", "-w", "-I", str(d), "-I", os.path.join(ROOT, "include"), "-isystem",
                    cuda, os.path.join(ROOT, "tests", "kv_runs.cpp"), "-o", str(exe)], check=True)
    return exe


def span(kernel, length, count, group, tile, window):
    """Blocks that a tile's rows see: (first, behind the last)."""
    rows = range(tile * ROWS[kernel], min(count * group, (tile + 1) * ROWS[kernel]))
    places = (length - count + rows[0] // group, length - count + rows[-1] // group)
    if places[1] < 0:
        return None
    lo = max(0, max(places[0], 0) - window + 1) if window else 0
    return lo // BLOCK[kernel], places[1] // BLOCK[kernel] + 1


def check(program, kernel, ahead, grid, lens, counts, group=1, kv_heads=2, window=0, page=16, max_pages=None):
    max_pages = max_pages or max(1, -(-max(lens) // page))
    text = f"{kernel} {ahead} {grid} {len(lens)} {group} {kv_heads} {window} {max_pages} {page}\n"
    text += "\n".join(f"{a} {b}" for a, b in zip(lens, counts))
    out = subprocess.run([program], input=text, capture_output=True, text=True, check=True, timeout=300).stdout
    lines = [line.split() for line in out.splitlines()]
    assert lines and lines[-1] == ["status", "0"], lines[-1:]
    got, splits = {}, {}
    for name, *x in lines:
        x = [int(v) for v in x]
        if name == "segment":
            c, token, tile, head, b_first, b_last, blocks, first, _, _, whole, row0, rows = x
            assert row0 == tile * ROWS[kernel] and whole == (b_first == 0 and b_last == blocks)
            got.setdefault((token, tile, head), []).append((c, b_first, b_last, blocks, first, rows))
        elif name == "split":
            c, first, last, token, head, row0, rows = x
            splits[token, row0 // ROWS[kernel], head] = c, first, last
    starts = np.concatenate([[0], np.cumsum(counts)])
    for token, length, count in zip(starts, lens, counts):
        for tile in range(-(-count * group // ROWS[kernel])):
            want = span(kernel, length, count, group, tile, window)
            for head in range(kv_heads):
                parts = sorted(got.pop((token, tile, head)))
                first, end = want or (parts[0][4], parts[0][4])
                assert all(p[3:] == (end - first, first, count * group) for p in parts)
                at = 0
                for _, b_first, b_last, *_ in parts:
                    assert b_first == at and b_last >= at
                    at = b_last
                assert at == end - first
                runs = [p[0] for p in parts]
                if len(runs) > 1:
                    assert splits.pop((token, tile, head)) == (runs[1], runs[0], runs[-1])
                    assert runs == list(range(runs[0], runs[-1] + 1))
    assert not got and not splits


AHEAD = pytest.mark.parametrize("ahead", [0, 1, 3])  # the warp that runs in front of the others
KERNELS = pytest.mark.parametrize("kernel", ["stream8", "stream16", "tile"])


@AHEAD
@KERNELS
def test_few_sequences(program, kernel, ahead):
    check(program, kernel, ahead, 13, [0, 1, 700, 4000, 17], [1, 1, 5, 300, 17], group=4)
    check(program, kernel, ahead, 13, [5000], [1], group=3, kv_heads=1)
    check(program, kernel, ahead, 5, [300, 20, 6], [0, 2, 9], group=2, window=37)


@AHEAD
@KERNELS
@pytest.mark.parametrize("n", [512, 513, 1300])
def test_more_sequences_than_are_summed_at_a_time(program, kernel, ahead, n):
    rng = np.random.default_rng(n)
    counts = rng.integers(0, 4, n)
    lens = counts + rng.integers(0, 300, n)
    check(program, kernel, ahead, 11, lens.tolist(), counts.tolist(), group=4, kv_heads=1)


@KERNELS
@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 3])
def test_a_window_as_wide_as_int_allows(program, kernel, window):
    """Sequences that bring more queries than they hold tokens: places below 0."""
    check(program, kernel, 0, 7, [1, 3, 900, 0], [4, 8, 40, 3], group=2, window=window)
    check(program, kernel, 0, 7, [1, 300], [2000, 5], group=2, window=window)
