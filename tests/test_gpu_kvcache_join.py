"""How the parts of a sequence that is cut are joined (tq_kv_attend)."""
import numpy as np
import pytest

from test_gpu_kvcache import Case, compare

pytestmark = pytest.mark.gpu


def test_parts_of_one_warp_are_added_first_at_head_dim_256(cuda_lib):
    """384 tokens in six parts of 64, each block of 16 its scale: what cancels between the first part and the fifth, which one
    of four warps takes, leaves the second's in place.  Scores are 0, so a part's sum is its values'."""
    torch = __import__("torch")
    case = Case(cuda_lib, [384], [1], kv_heads=1, dim=256, page=64, seed=1)
    for name in "kv":
        case.pool[name][:] = 0
        case.scale[name][:] = 1.0
    pages = case.table[case.slots[0]]
    for token, code, scale in ((5, 127, 2.0 ** 30), (4 * 64 + 5, -127, 2.0 ** 30), (64 + 9, 127, 1.0)):
        p, inside = pages[token // 64], token % 64
        case.pool["v"][case.layer, p, 0, inside] = np.uint8(code % 256)
        case.scale["v"][case.layer, p, 0, inside // 16] = scale
    q = torch.zeros(1, 1, 256, dtype=torch.float16, device="cuda")
    out = case.cache().attention(case.layer, case.device(case.slots), case.device(case.starts), q)
    assert (out == torch.tensor(127 / 384, dtype=torch.float16, device="cuda")).all()


@pytest.mark.parametrize("length", [700, 1300])
def test_a_part_that_a_row_does_not_see_is_left_out(cuda_lib, length):
    """256 prompted tokens in parts of 128, up to eight and more: values that are not numbers behind the first queries' places do
    not reach them, whatever they are multiplied by."""
    case = Case(cuda_lib, [length], [256], kv_heads=1, dim=128, codes="e4m3", seed=length).fill()
    q = case.queries(1, "bfloat16")
    last = length // 128 * 128
    good = case.expected(q.double().cpu().numpy())
    for token in range(last, length):
        case.pool["v"][case.layer, case.table[case.slots[0], token // case.page], 0, token % case.page] = 0x7F
    out, lse = case.cache().attention(case.layer, case.device(case.slots), case.device(case.starts), q, return_lse=True)
    n = last - (length - 256)  # queries in front
    case.expected = lambda *_: [x[:n] for x in good]
    compare(case, q[:n], out[:n], lse[:n])
    assert out[n:].isnan().all()
