"""The example that searches, shares a passage's pages, drafts from its words and
verifies them: what its cache holds at the end follows from what it says."""
import os
import sys

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_answer(cuda_lib, codes):
    import torch
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import answer as example
    passages, requests, steps = 16, 4, 6
    told, found, cache, accepted = example.answer(requests, steps, passages=passages, codes=codes)
    lens, refs, table = cache.lens.tolist(), cache.refs.tolist(), cache.table.tolist()
    for i, p in enumerate(found):
        # the passage, five words of question, and in each step the last word and the accepted drafts
        assert lens[passages + i] == lens[p] + 5 + steps + sum(a[i] for a in accepted)
        assert len(told[i]) == steps + sum(a[i] for a in accepted) and all(0 <= w < example.VOCAB for w in told[i])
        # whole pages of the passage are shared, the one it fills in part is not
        whole = lens[p] // 32
        assert table[passages + i][:whole] == table[p][:whole]
        assert lens[p] % 32 == 0 or table[passages + i][whole] != table[p][whole]
    held = [p for row, n in zip(table, lens) for p in row[: -(-n // 32)]]
    assert all(refs[p] == held.count(p) for p in set(held)) and sum(refs) == len(held)
    cache.truncate(example.ints(range(passages, passages + requests)), example.ints([0] * requests))
    used = cache.compact()
    cache.check()
    assert int(used) == sum(-(-n // 32) for n in cache.lens.tolist()) == int((cache.refs > 0).sum())
    assert (cache.refs[: int(used)] > 0).all()
    again, _, _, _ = example.answer(requests, steps, passages=passages, codes=codes)
    assert again == told  # given random numbers: the same run
