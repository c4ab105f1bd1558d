"""tq_sample's cut of top-p where many small weights make it up, against the definition
in 64 bits: noise lets a token win that stands a little in front of the cut, or a
little behind it."""
import numpy as np
import pytest

from test_gpu_sample import check

pytestmark = pytest.mark.gpu


def row(vocab, x=0.0, type="float32"):
    torch = __import__("torch")
    return torch.full((2, vocab), x, device="cuda").to(getattr(torch, type)), torch.ones(2, vocab, device="cuda")


def test_weights_that_are_small_beside_the_first(cuda_lib):
    """99,999 tokens of 2^-33 beside one of 1, the last of them not among the first k: 1.2e-5 of the weight, half of it kept."""
    vocab = 100_000
    logits, noise = row(vocab, -33 * float(np.log(2.0)))
    logits[:, 0] = 0.0
    noise[:, 0] = 2.0 ** 20
    noise[0, 30_000] = noise[1, 70_000] = 2.0 ** -60
    tokens = check(cuda_lib, logits, noise, top_k=[vocab - 1] * 2, top_p=[1 - 6e-6] * 2)
    assert int(tokens[0]) == 30_000 and int(tokens[1]) < 50_000


@pytest.mark.parametrize("type", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab,top_p", [(128_000, 0.99999), (100_003, 0.9), (1_000_003, 0.5)])
def test_equal_tokens(cuda_lib, vocab, top_p, type):
    """A cut by the tokens' own order, through a row of one weight (a temperature without bound, values far apart)."""
    torch = __import__("torch")
    logits, noise = row(vocab, type=type)
    g = torch.Generator(device="cuda").manual_seed(vocab)
    logits.copy_(torch.randn(vocab, device="cuda", generator=g))
    order = torch.argsort(logits[0].float(), descending=True, stable=True)
    count = int(np.ceil(np.float32(top_p).astype(np.float64) * vocab))  # (kept)
    noise[0, order[count - 1]] = noise[1, order[count]] = 2.0 ** -60
    tokens = check(cuda_lib, logits, noise, temperature=[float("inf")] * 2, top_p=[top_p] * 2)
    assert int(tokens[0]) == int(order[count - 1]) and int(tokens[1]) != int(order[count])
