"""Plans whose groups do not agree, and groups of more requests than a block of threads
looks at (KVCache.shared_attention), against plain attention."""
import numpy as np
import pytest

from test_gpu_kvcache import compare
from test_gpu_shared import Batch

pytestmark = pytest.mark.gpu

# (first, members, tokens) of six requests that hold the same 192 tokens; all of them have an entry that does not fit
OVERLAPPING = [
    [(0, 4, 192)] * 2 + [(2, 2, 128)] * 2 + [(4, 2, 192)] * 2,          # a group that ends in another
    [(0, 3, 128), (1, 2, 64), (1, 2, 64)] + [(3, 3, 192)] * 3,          # one within another, fewer tokens
    [(0, 6, 64)] * 2 + [(2, 3, 192)] * 3 + [(0, 6, 64)],
    [(0, 2, 64)] * 3 + [(3, 3, 64)] * 3,                                # one that names a group behind its end
    [(0, 6, 64)] * 5 + [(0, 6, 65)],
    [(0, 6, 64)] * 3 + [(3, 1, 0)] + [(0, 6, 64)] * 2,
    [(1, 3, 64)] * 4 + [(4, 2, 192)] * 2,                               # one in front of its group's first
    [(0, 6, 64)] * 3 + [(0, 5, 64)] * 3,
]


@pytest.mark.parametrize("plan", OVERLAPPING)
@pytest.mark.parametrize("dim,group,new", [(128, 2, 1), (64, 4, 1), (256, 2, 2), (128, 16, 8), (64, 16, 8)])
def test_groups_that_overlap(cuda_lib, plan, dim, group, new):
    """Their requests are attended by themselves, and the status says so; few rows a request and many."""
    case = Batch(cuda_lib, [192], [[new + i for i in range(6)]], [[new] * 6], dim=dim, seed=dim + group).fill()
    q = case.queries(2 * group, "bfloat16")
    for groups in (1, 6):
        cache = case.cache()
        out, lse = cache.shared_attention(case.layer, case.device(case.slots), case.device(case.starts),
                                          case.device(np.array(plan, np.int32).T.copy()), q, groups=groups, return_lse=True)
        with pytest.raises(cuda_lib.TQError, match="left out"):
            cache.check()
        compare(case, q, out, lse)


SIZES = [[2500], [1024, 1024], [1000, 1100, 3], [1023, 2, 1500], [1] * 1030 + [2] * 20]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda x: "-".join(map(str, x[-3:])))
def test_large_groups(cuda_lib, sizes):
    """Groups across a block's ends; then one entry of each kind of place that names something else."""
    n = sum(sizes)
    case = Batch(cuda_lib, [16] * len(sizes), [[1 + i % 3 for i in range(k)] for k in sizes], [[1] * k for k in sizes], page=16,
                 dim=64, kv_heads=1, layers=1, seed=len(sizes)).fill()
    q = case.queries(2, "float16")
    args = case.layer, case.device(case.slots), case.device(case.starts)
    good, ref = case.plan(), case.expected(q.double().cpu().numpy())
    case.expected = lambda *_: ref
    cache = case.cache()
    compare(case, q, *cache.shared_attention(*args, case.device(good), q, groups=len(sizes), return_lse=True))
    cache.check()
    for i in {0, 1, 1023, 1024, 1025, n - 1}:
        if good[1, i] > 1:
            bad = good.copy()
            bad[2, i] = 8
            cache = case.cache()
            compare(case, q, *cache.shared_attention(*args, case.device(bad), q, groups=len(sizes), return_lse=True))
            with pytest.raises(cuda_lib.TQError, match="left out"):
                cache.check()
