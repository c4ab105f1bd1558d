"""tq_sample of rows that are views of larger tensors."""
import pytest

from test_gpu_sample import check, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [700, 20_000, 128_000])
def test_one_row_of_any_stride(cuda_lib, vocab):
    """The last of 2^31 / vocab and more positions: the stride of the only row is no distance to another one."""
    logits, noise = rows(1, vocab, "bfloat16", seed=vocab, likely=9)
    settings = dict(temperature=[0.9], top_p=[0.9])
    want = check(cuda_lib, logits, noise, **settings)
    wide = [x.as_strided((1, vocab), (2 ** 33, 1)) for x in (logits, noise)]
    assert check(cuda_lib, *wide, **settings).equal(want)


def test_every_third_row_and_one_noise_for_all(cuda_lib):
    logits, noise = rows(9, 5003, seed=2, likely=9)
    check(cuda_lib, logits[1::3], noise[4:5].expand(3, -1), top_p=[0.9] * 3)
