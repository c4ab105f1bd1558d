"""A workspace of attention that is kept for the largest call serves the smaller ones."""
import ctypes as C

import numpy as np
import pytest

from test_kvcache_host import cache, lib  # noqa: F401  (a fixture)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_bytes_grow_with_the_call(lib, dim):
    """Whatever kernel the smaller call takes: fewer sequences bring more rows each."""
    c = cache(head_dim=dim, slots=65536)

    def bytes_of(n, total, heads):
        need = C.c_size_t()
        assert lib.tq_kv_attend_workspace(c, n, total, heads, C.byref(need)) == 0
        return need.value

    rng = np.random.default_rng(dim)
    for _ in range(300):
        n, total, group = (int(2 ** rng.uniform(0, k)) for k in (8, 11, 5))
        smaller = bytes_of(int(rng.integers(0, n + 1)), int(rng.integers(0, total + 1)), 4 * int(rng.integers(1, group + 1)))
        assert smaller <= bytes_of(n, total, 4 * group)
    assert bytes_of(1, 33, 32) <= bytes_of(64, 64, 32)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_a_kept_workspace(cuda_lib, dim):
    """One for 40 single tokens is enough for prompts of fewer sequences, whose kernels need more than that call's own."""
    import torch

    from test_gpu_kvcache import Case, compare
    ws = None
    for lens, new in (([50] * 40, [1] * 40), ([90], [40]), ([90, 30], [20, 20]), ([70, 2000, 9], [3, 3, 3]), ([1000], [1])):
        case = Case(cuda_lib, lens, new, dim=dim, seed=len(lens)).fill()
        cache, q = case.cache(), case.queries(4 * 2, "bfloat16")
        if ws is None:
            ws = torch.empty(cache.attention_workspace(40, 40, 8), dtype=torch.uint8, device="cuda")
        out, lse = cache.attention(case.layer, case.device(case.slots), case.device(case.starts), q, workspace=ws,
                                   return_lse=True)
        cache.check()
        compare(case, q, out, lse)
