"""Attention at the ends of what it is given: queries that are not finite, windows as wide as int, queries that no
sequence brings."""
import numpy as np
import pytest

from test_gpu_kvcache import Case, compare

pytestmark = pytest.mark.gpu


def attend(case, q, window=0, **kw):
    cache = case.cache()
    out, lse = cache.attention(case.layer, case.device(case.slots), case.device(case.starts), q, window=window,
                               return_lse=True, **kw)
    cache.check()
    return out, lse


# sequences whose work is cut over several runs, ones that a run takes whole, of one token and of none;
# up to 8 rows per key head, up to 16, one row tile of the tensor cores, two
SHAPES = pytest.mark.parametrize("lens,new,dim,group", [
    ([3000, 40, 1, 0], [1, 1, 1, 1], 128, 4), ([2000, 50, 9, 0], [2, 2, 2, 2], 64, 8), ([1500, 30, 2], [3, 2, 2], 256, 2),
    ([3000, 60, 61, 30], [60, 60, 60, 60], 128, 1), ([2500, 200, 201, 130], [200, 200, 200, 200], 64, 1)])


@SHAPES
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("type", ["bfloat16", "float16"])
def test_a_query_that_is_not_finite_gives_nan(cuda_lib, lens, new, dim, group, codes, value, type):
    """In the row itself, in every element and in its lse, if it sees a token; the other rows are what they were, up to
    the order of the running maximum's steps."""
    import torch
    case = Case(cuda_lib, lens, new, dim=dim, codes=codes, seed=dim + len(lens)).fill()
    clean = case.queries(2 * group, type)
    q = clean.clone()
    bad = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    seen = torch.zeros_like(bad)
    for i, (length, count) in enumerate(zip(lens, new)):
        at = int(case.starts[i])
        seen[at + max(0, count - length): at + count] = True
        for r in {0, count // 2, count - 1}:
            h = (r + i) % (2 * group)
            bad[at + r, h] = True
            q[at + r, h, (7 * r + i) % dim] = value
    want, want_lse = attend(case, clean)
    out, lse = attend(case, q)
    hit = bad & seen
    assert hit.any() and (bad & ~seen).any() == (min(lens) == 0 or any(n > x for n, x in zip(new, lens)))
    assert out[hit].isnan().all() and lse[hit].isnan().all()
    compare(case, clean, torch.where(hit[..., None], want, out), torch.where(hit, want_lse, lse))


@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 4, 2**31 + 3, 2**32 + 5, 2**63])
@pytest.mark.parametrize("lens,new,dim,group", [
    ([1, 3, 40, 0], [4, 8, 40, 3], 128, 2), ([2, 700, 5], [9, 9, 9], 64, 1), ([3, 200], [60, 60], 128, 1),
    ([5, 129, 400], [300, 300, 300], 64, 1)])
def test_a_window_that_hides_nothing(cuda_lib, lens, new, dim, group, window):
    """As wide as int allows, or wider: the results without one, also where a sequence brings more queries than it has
    tokens."""
    case = Case(cuda_lib, lens, new, dim=dim, seed=dim + len(lens)).fill()
    q = case.queries(2 * group, "bfloat16")
    want = attend(case, q)
    got = attend(case, q, window=window)
    assert all(case.torch.equal(a, b) for a, b in zip(got, want))
    compare(case, q, *got)


@pytest.mark.parametrize("rows", [1, 3, 60, 200])
@pytest.mark.parametrize("front,behind", [(0, 5), (2, 0), (3, 300)])
def test_queries_that_no_sequence_brings(cuda_lib, rows, front, behind):
    """A step padded to a size that is kept: queries in front of the first sequence's and behind the last one's get what
    a query that sees nothing gets, and the others what they get without them."""
    import torch
    case = Case(cuda_lib, [700, 30, 250], [rows] * 3, dim=64, kv_heads=1, seed=rows).fill()
    q = case.queries(2, "float16")
    want, want_lse = attend(case, q)
    total = front + q.shape[0] + behind
    padded = torch.randn(total, 2, 64, device="cuda").to(q.dtype)
    padded[front: front + q.shape[0]] = q
    out, lse = torch.full_like(padded, float("nan")), torch.full((total, 2), float("nan"), device="cuda")
    cache = case.cache()
    cache.attention(case.layer, case.device(case.slots), case.device(case.starts + front), padded, out=out, lse=lse)
    cache.check()
    inside = slice(front, front + q.shape[0])
    # (which kernel takes a call goes by its queries, so the order of sums may differ)
    compare(case, q, out[inside], lse[inside])
    outside = torch.ones(total, dtype=torch.bool, device="cuda")
    outside[inside] = False
    assert not out[outside].any() and (lse[outside] == -float("inf")).all()


def test_queries_of_sequences_that_bring_none(cuda_lib):
    import torch
    case = Case(cuda_lib, [70, 30], [0, 0], dim=128, seed=1).fill()
    q = torch.randn(9, 4, 128, device="cuda").to(torch.bfloat16)
    out, lse = torch.full_like(q, 3), torch.full((9, 4), 3.0, device="cuda")
    cache = case.cache()
    cache.attention(case.layer, case.device(case.slots), case.device(case.starts), q, out=out, lse=lse)
    cache.check()
    assert not out.any() and (lse == -float("inf")).all()
