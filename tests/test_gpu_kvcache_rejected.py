"""What drafts that are cut off again leave in the cache: the block that they shared with kept tokens has the scale
that they gave it and its codes rounded to that; every other block is as if they had never been there."""
import numpy as np
import pytest

import kvref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("kept", [16, 20, 31, 32])
def test_rejected_drafts(cuda_lib, codes, kept):
    import torch
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rng = np.random.default_rng(kept)
    first, wide, last = (torch.from_numpy(rng.standard_normal((n, 2, 64)).astype(np.float32)).cuda() * w
                         for n, w in ((kept, 1), (3, 6), (1, 1)))
    cache = cuda_lib.KVCache(6, 1, 4, 2, 64, 16, codes=codes)
    plain = np.zeros((6, 2, 16, 64), np.uint8), np.zeros((6, 2, 1), np.float32)
    table = np.arange(4)[None]

    def bring(x, length):
        cache.extend(i32(0), i32(len(x)))
        cache.append(0, i32(0), i32(0, len(x)), x, x)
        kvref.append(*plain, table, [length + len(x)], [0], [0, len(x)], x.cpu().numpy(), codes)

    def state():
        return cache.k[0].cpu().numpy().copy(), cache.k_scale[0].cpu().numpy().copy()

    def values(pool, scale, n):
        return kvref.read(pool, scale, table, 0, n, codes)

    bring(first, 0)
    before = state()
    bring(wide, kept)
    cache.truncate(i32(0), i32(kept))
    after = state()
    whole = kept // 16  # blocks (and pages, here) that hold kept tokens only
    assert np.array_equal(after[0][:whole], before[0][:whole]) and np.array_equal(after[1][:whole], before[1][:whole])
    if kept % 16:
        old, new = before[1][whole], after[1][whole]
        assert (new > old).all()  # (the drafts are six times as wide)
        off = np.abs(values(*after, kept) - values(*before, kept))[whole * 16:].max((0, 2))
        # half a step of the new scale: of int8 1, of e4m3 up to 32 (its values from 256 to 448)
        assert (off <= (0.5 if codes == "int8" else 16) * new[:, 0] * (1 + 2.0 ** -20)).all()
    bring(last, kept)
    cache.check()
    got = state()
    # the next token: the definition, on a block that the drafts have been in, or on one that begins with it
    assert np.array_equal(values(*got, kept + 1), values(*plain, kept + 1))
    if kept % 16:
        assert np.array_equal(got[1][whole], after[1][whole])
    else:
        qmax = kvref.QMAX[codes]
        assert np.array_equal(got[1][whole][:, 0], np.abs(last.cpu().numpy()[0]).max(1) / qmax)
