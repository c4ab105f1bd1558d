"""The key-value cache at sizes that the kernels split their work by: more
sequences than are summed at a time, rows on both sides of the choice of a kernel
and of its row tiles, and entries that cannot be served among many rows."""
import numpy as np
import pytest

from test_gpu_kvcache import Case, check_append, check_attention, run_append

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,new,heads", [(1300, 1, 4), (1100, 3, 8), (700, 12, 4)])
def test_attention_over_many_sequences(cuda_lib, n, new, heads):
    """Sequences' work is summed 512 at a time; the last one brings 12 x 4 rows (the tiles), the others fewer."""
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 45, n)
    case = Case(cuda_lib, lens.tolist(), [new] * n, kv_heads=1, dim=64, page=16, seed=n, layers=1).fill()
    check_attention(case, case.queries(heads, "bfloat16"))


def test_append_for_many_sequences(cuda_lib):
    import torch
    rng = np.random.default_rng(5)
    new = rng.integers(0, 4, 1300)
    lens = new + rng.integers(0, 40, 1300)
    case = Case(cuda_lib, lens.tolist(), new.tolist(), kv_heads=1, dim=64, page=16, seed=5, layers=1).fill()
    x = case.device(case.rng.standard_normal((int(new.sum()), 1, 64)).astype(np.float32)).to(torch.bfloat16)
    check_append(case, run_append(case, x, x), x, x)


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("dim,rows", [(128, 26), (128, 27), (64, 40), (64, 41), (128, 127), (128, 128), (128, 129),
                                      (64, 256), (128, 257), (64, 300)])
def test_attention_rows(cuda_lib, codes, dim, rows):
    """One query head per key head: as many rows as new tokens.  Lengths around the tiles' 128 tokens."""
    lens = [rows, rows + 1, 128, 129, 383, 700]
    case = Case(cuda_lib, [max(x, rows) for x in lens], [rows] * len(lens), kv_heads=1, dim=dim, page=32, codes=codes,
                seed=rows, layers=1).fill()
    check_attention(case, case.queries(1, "float16"))


@pytest.mark.parametrize("window", [1, 100, 129, 1000])
@pytest.mark.parametrize("rows", [60, 200])
def test_attention_tiles_with_a_window(cuda_lib, window, rows):
    case = Case(cuda_lib, [900, 200, rows], [rows] * 3, kv_heads=1, dim=128, seed=window, layers=1).fill()
    check_attention(case, case.queries(1, "bfloat16"), window=window)


@pytest.mark.parametrize("rows", [60, 200])
def test_attention_tiles_on_rising_scores(cuda_lib, rows):
    """Scores that grow by hundreds over the sequence: the reference moves from tile to tile, and O with it."""
    case = Case(cuda_lib, [1500], [rows], kv_heads=1, dim=64, seed=9, layers=1).fill(0.0)
    pages = case.table[case.slots[0]]
    for i, p in enumerate(pages[pages >= 0]):
        case.scale["k"][0, p] *= np.float32(0.1 + i)
    check_attention(case, case.queries(1, "float16"))


@pytest.mark.parametrize("rows", [60, 200])
def test_attention_tiles_leave_out_bad_entries(cuda_lib, rows):
    case = Case(cuda_lib, [300, 290, 280], [rows] * 3, kv_heads=1, dim=128, seed=10, layers=1).fill()
    q = case.queries(1, "bfloat16")
    args = (case.device(case.starts), q)
    good = case.cache().attention(0, case.device(case.slots), *args)
    for what in ("slot", "page"):
        cache, slots = case.cache(), case.slots.copy()
        if what == "slot":
            slots[1] = -5
        else:
            cache.table[int(slots[1]), 1] = -7
        out = cache.attention(0, case.device(slots), *args)
        with pytest.raises(cuda_lib.TQError, match="TQ_EINVAL"):
            cache.check()
        for i in (0, 2):  # (served as before, up to where the work is cut)
            a, b = (x[i * rows: (i + 1) * rows].float() for x in (out, good))
            assert (a - b).abs().max() <= 2.0 ** -7 * b.abs().max()
        assert case.torch.isfinite(out.float()).all()
        if what == "slot":
            assert not out[rows: 2 * rows].any()
