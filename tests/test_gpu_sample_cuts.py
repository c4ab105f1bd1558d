"""tq_sample's cut of top-p where many small weights make it up, against the definition
in 64 bits: noise lets a token win that stands a little in front of the cut, or a
little behind it."""
import numpy as np
import pytest

from test_gpu_sample import check, rows

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


def short_of(unit, values):
    """Of `values`, (first, second) for which e^(first / 32) lies in a step whose weight, in parts of 1 / unit of its upper
    end, is rounded down the most."""
    best = max(values, key=lambda v: (lambda w: (w - np.rint(w)) if w - np.rint(w) > 0 else 0)(
        unit * np.exp((v - np.floor(v + 0.5) - 0.5) / 32)))
    return best


def test_a_first_token_that_is_nearly_all(cuda_lib):
    """One token and 4e-6 of its weight in 1,000 others, half of which are kept: steps whose weights are rounded do not see
    where."""
    torch = __import__("torch")
    vocab = 20_000
    top = short_of(2.0 ** 16, np.arange(0, 64, 1 / 64)) / 32
    logits = torch.full((2, vocab), -np.inf, device="cuda")
    logits[:, 100:1100] = torch.from_numpy((top + np.log(4e-9) - np.arange(1000) * 1e-5).astype(np.float32)).cuda()
    logits[:, 7000] = float(top)
    noise = torch.ones_like(logits)
    noise[:, 7000] = 2.0 ** 20
    noise[0, 150] = noise[1, 1050] = 2.0 ** -60
    tokens = check(cuda_lib, logits, noise, top_p=[1 - 2e-6] * 2)
    assert tokens.tolist() == [150, 7000]  # (the first: 2^-20 in the race, the others 4e-9)


def test_a_first_token_that_is_nearly_all_of_a_long_row(cuda_lib):
    """The same in a batch of long rows."""
    torch = __import__("torch")
    n, vocab = 64, 128_000
    logits, noise = rows(n, vocab, "bfloat16", seed=41, likely=9)
    temperature = np.float32(32 / short_of(2.0 ** 17, np.arange(31, 33, 1 / 256)))  # (the first token's logit is 1)
    weight = float(np.exp(-19.5 / np.float64(temperature)))
    count = int(3e-6 / weight)
    logits[:2] = -float("inf")
    logits[:2, 100: 100 + count] = -18.5
    logits[:2, 70_000] = 1.0
    noise[:2] = 1.0
    noise[:2, 70_000] = 2.0 ** 20
    noise[0, 100 + count // 50] = noise[1, 99 + count] = 2.0 ** -60
    given = dict(temperature=[float(temperature)] * n, top_p=[1 - 1.5e-6] * n)
    tokens = cuda_lib.sample_tokens(logits, noise, **{k: torch.tensor(v, device="cuda") for k, v in given.items()})
    alone = check(cuda_lib, logits[:2], noise[:2], **{k: v[:2] for k, v in given.items()})
    assert tokens[:2].tolist() == alone.tolist() == [100 + count // 50, 70_000]


@pytest.mark.parametrize("vocab", [20_000, 100_003])
def test_values_on_either_side_of_where_steps_have_numbers(cuda_lib, vocab):
    """x / T of 10^6 / 32 and more, where a part's largest value has no step but the row's largest has one."""
    torch = __import__("torch")
    logits = torch.full((2, vocab), -40.0, device="cuda")
    logits[:, :100] = -31.2499
    logits[:, 9000:10_000] = -31.2501
    noise = torch.ones_like(logits)
    noise[0, 9400] = noise[1, 9800] = 2.0 ** -60
    tokens = check(cuda_lib, logits, noise, temperature=[1e-3] * 2, top_p=[0.5] * 2)
    assert int(tokens[0]) == 9400 and int(tokens[1]) < 9500


@pytest.mark.parametrize("place", [10, 300, 70_000])
def test_a_small_top_p_of_many_tokens(cuda_lib, place):
    """top-p a few float32 steps below what `place` of 10^6 equal tokens have: the one behind them stays out."""
    vocab = 1_000_000
    top_p = np.float32(place * (1 - 4e-6) / vocab)
    assert place - 1 < float(top_p) * vocab < place * (1 - 2.0 ** -19)
    logits, noise = row(vocab)
    noise[0, place - 1] = noise[1, place] = 2.0 ** -60
    tokens = check(cuda_lib, logits, noise, top_p=[float(top_p)] * 2)
    assert int(tokens[0]) == place - 1 and int(tokens[1]) == 0


@pytest.mark.parametrize("type", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("vocab", [900, 20_000, 128_000])
def test_rows_of_the_lowest_value(cuda_lib, vocab, type):
    """All tokens at the type's lowest value, which masks nothing: they are kept in their own order."""
    torch = __import__("torch")
    logits, noise = row(vocab, torch.finfo(getattr(torch, type)).min, type)
    noise[0, vocab // 2 - 1] = noise[1, vocab // 2 + 1] = 2.0 ** -60
    tokens = check(cuda_lib, logits, noise, top_p=[0.5] * 2)
    assert tokens.tolist() == [vocab // 2 - 1, 0]
    assert check(cuda_lib, logits, noise, top_p=[0.5] * 2, temperature=[1e30] * 2).tolist() == [vocab // 2 - 1, 0]
