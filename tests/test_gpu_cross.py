"""Attention over all tokens that a slot holds (KVCache.cross_attention) against a
plain form in 64 bits."""
import numpy as np
import pytest

import kvref
from test_gpu_kvcache import Case, compare

pytestmark = pytest.mark.gpu


class Readers(Case):
    """Slots that hold `lens` tokens, with `new` queries each that are none of them."""

    def expected(self, q, window=0, scale=None):
        scale = q.shape[2] ** -0.5 if scale is None else scale
        parts = []
        for i, slot in enumerate(self.slots):
            n = int(self.lens[slot])
            k, v = (kvref.read(self.pool[x][self.layer], self.scale[x][self.layer], self.table, slot, n, self.codes)
                    for x in "kv")
            for r in range(self.starts[i], self.starts[i + 1]):  # (one query stands at the end: it sees all)
                parts.append(kvref.attention(k, v, q[r: r + 1], scale, 0) if n else
                             (np.zeros((1,) + q.shape[1:]), np.full((1, q.shape[1]), -np.inf), np.zeros((1,) + q.shape[1:]),
                              np.zeros((1, q.shape[1]))))
        return [np.concatenate(x) for x in zip(*parts)]


def check(case, q, scale=None, **kw):
    cache = case.cache()
    out, lse = cache.cross_attention(case.layer, case.device(case.slots), case.device(case.starts), q, scale=scale,
                                     return_lse=True, **kw)
    cache.check()
    compare(case, q, out, lse, 0, scale)
    return out, lse


# fewer tokens than queries, none at all, one; blocks, pages and tiles that end inside or at the length
LENGTHS = [([1], [1]), ([0, 1, 15, 16, 17, 33], [1] * 6), ([700, 64, 65, 128], [1] * 4), ([3, 0, 200, 1], [9, 4, 5, 60]),
           ([40, 129, 256], [70, 1, 66]), ([1], [300]), ([1031], [30])]


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,new", LENGTHS)
@pytest.mark.parametrize("dim,group,type", [(128, 4, "bfloat16"), (64, 5, "float16"), (256, 1, "bfloat16")])
def test_cross(cuda_lib, codes, lens, new, dim, group, type):
    case = Readers(cuda_lib, lens, new, dim=dim, codes=codes, seed=sum(lens) + dim).fill()
    check(case, case.queries(2 * group, type))


@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("dim,kv_heads,group", [(64, 1, 16), (128, 3, 7)])
def test_cross_cut_into_many_runs(cuda_lib, page, dim, kv_heads, group):
    case = Readers(cuda_lib, [2500, 31], [40, 3], page=page, dim=dim, kv_heads=kv_heads, seed=page + dim).fill()
    check(case, case.queries(kv_heads * group, "bfloat16"))


def test_one_slot_read_by_several_sequences(cuda_lib):
    case = Readers(cuda_lib, [300, 20], [3, 2], seed=5).fill()
    case.slots = case.slots[[0, 1, 0, 0]]
    case.starts = np.array([0, 3, 5, 6, 40], np.int32)
    check(case, case.queries(8, "float16"))


def test_strided_queries_scale_out_and_workspace(cuda_lib):
    torch = __import__("torch")
    case = Readers(cuda_lib, [90, 300], [4, 2], codes="e4m3", seed=6).fill()
    wide = case.queries(8, "bfloat16").repeat_interleave(3, 1)
    q = wide[:, 1:17:2]
    out, lse = torch.empty(6, 8, 128, dtype=q.dtype, device="cuda"), torch.empty(6, 8, device="cuda")
    ws = torch.empty(case.cache().attention_workspace(2, 6, 8), dtype=torch.uint8, device="cuda")
    got, _ = check(case, q, scale=-0.05, out=out, lse=lse, workspace=ws)
    assert got is out


def test_padded_and_invalid_entries(cuda_lib):
    """Queries that no sequence brings and those of a slot that is not there get zeros and -inf; the status says the latter."""
    case = Readers(cuda_lib, [50, 60, 70], [2, 3, 4], seed=7).fill()
    cache, q = case.cache(), case.queries(8, "bfloat16")
    slots = case.slots.copy()
    slots[1] = len(case.lens)
    starts = np.array([1, 2, 5, 7], np.int32)
    out, lse = cache.cross_attention(case.layer, case.device(slots), case.device(starts), q, return_lse=True)
    with pytest.raises(cuda_lib.TQError, match="left out"):
        cache.check()
    case.slots, case.starts = case.slots[[0, 2]], np.array([0, 1, 3], np.int32)
    compare(case, q[[1, 5, 6]], out[[1, 5, 6]], lse[[1, 5, 6]])
    rest = [0, 2, 3, 4, 7, 8]
    assert not out[rest].any() and (lse[rest] == -np.inf).all()


@pytest.mark.parametrize("new", [2, 60])
def test_queries_that_are_not_finite(cuda_lib, new):
    case = Readers(cuda_lib, [200], [new], seed=8).fill()
    cache, q = case.cache(), case.queries(8, "float16")
    args = case.layer, case.device(case.slots), case.device(case.starts)
    good = cache.cross_attention(*args, q)
    q[1, 3, 5] = float("nan")
    q[0, 2, 7] = float("inf")
    out, lse = cache.cross_attention(*args, q, return_lse=True)
    assert out[1, 3].isnan().all() and out[0, 2].isnan().all() and lse[1, 3].isnan() and lse[0, 2].isnan()
    out[1, 3], out[0, 2] = good[1, 3], good[0, 2]
    assert out.equal(good)
