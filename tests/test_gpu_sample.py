"""tq_sample on the GPU against its definition in 64 bits."""
import numpy as np
import pytest

from sampleref import sample

pytestmark = pytest.mark.gpu

SLACK = 2.0 ** -20  # what a weight, or a sum of weights, may be off next to a border


def check(tq, logits, noise, **settings):
    """logits, noise: tensors on the GPU; settings: lists, or None.  Equality with the definition, or with one whose borders
    lie SLACK to either side; the logprob within float32's rounding (2^-24) of it and of a sum that is 2^-21 off."""
    torch = __import__("torch")
    n = logits.shape[0]
    kinds = {"temperature": torch.float32, "top_k": torch.int32, "top_p": torch.float32, "min_p": torch.float32}
    given = {name: torch.tensor(x, dtype=kinds[name], device="cuda") for name, x in settings.items() if x is not None}
    tokens, logprobs = tq.sample_tokens(logits, noise, **given, return_logprobs=True)
    assert tokens.dtype == torch.int32 and logprobs.dtype == torch.float32
    again, _ = tq.sample_tokens(logits, noise, **given, return_logprobs=True)
    assert tokens.equal(again)
    x, e = logits.double().cpu().numpy(), noise.double().cpu().numpy()
    rows = {name: t.double().cpu().tolist() for name, t in given.items()}
    for i in range(n):
        s = {name: (int(v[i]) if name == "top_k" else v[i]) for name, v in rows.items()}
        want = [sample(x[i], e[i], **s, slack=slack) for slack in (0.0, SLACK, -SLACK)]
        token, logprob = int(tokens[i]), float(logprobs[i])
        assert token in [t for t, _ in want], (i, s, token, want)
        ref = dict(want)[token]
        assert logprob == ref or abs(logprob - ref) <= 2.0 ** -24 * abs(ref) + 2.0 ** -21, (i, s, logprob, ref)
    return tokens


def rows(n, vocab, type="float32", seed=0, spread=2.0, likely=0, stride=0):
    torch = __import__("torch")
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, vocab + stride, device="cuda", generator=g) * spread
    if likely:
        x.scatter_add_(1, torch.randint(vocab, (n, likely), device="cuda", generator=g),
                       torch.rand(n, likely, device="cuda", generator=g) * 8 + 4)
    e = torch.empty(n, vocab + stride, device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    return x.to(getattr(torch, type))[:, :vocab], e[:, :vocab]


MIXED = [(1.0, 0, 1.0, 0.0), (0.7, 50, 0.95, 0.0), (1.0, 0, 0.9, 0.0), (1.3, 40, 1.0, 0.0), (1.0, 0, 1.0, 0.05),
         (0.0, 0, 1.0, 0.0), (0.5, 600, 0.8, 0.01), (1.0, 5000, 0.5, 0.0), (2.0, 3, 0.3, 0.2), (1.0, 1, 1.0, 0.0),
         (1.0, 0, 1e-6, 0.0), (0.02, 0, 0.999, 0.0), (5.0, 0, 0.99, 0.0), (1.0, 2 ** 31 - 1, 1.5, -1.0), (1.0, -3, 0.5, 0.0),
         (1.0, 0, 0.9999999, 0.0)]


@pytest.mark.parametrize("type", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 1000, 1025, 32_000, 100_003, 128_000])
@pytest.mark.parametrize("likely", [0, 24])
def test_sample(cuda_lib, type, vocab, likely):
    logits, noise = rows(len(MIXED), vocab, type, seed=vocab + likely, likely=likely)
    check(cuda_lib, logits, noise, **dict(zip(("temperature", "top_k", "top_p", "min_p"), map(list, zip(*MIXED)))))


@pytest.mark.parametrize("n,vocab,stride", [(1, 300_000, 0), (3, 5001, 3), (70, 4097, 1), (300, 64, 0), (700, 2000, 16)])
@pytest.mark.parametrize("type", ["float32", "bfloat16"])
def test_batches_and_strides(cuda_lib, n, vocab, stride, type):
    logits, noise = rows(n, vocab, type, seed=n, likely=5, stride=stride)
    check(cuda_lib, logits, noise, temperature=[0.8] * n, top_p=[0.92] * n)
    check(cuda_lib, logits, noise, top_k=[20] * n)
    check(cuda_lib, logits, noise)


@pytest.mark.parametrize("vocab", [3000, 70_000])
@pytest.mark.parametrize("type", ["float32", "bfloat16"])
def test_ties(cuda_lib, vocab, type):
    """Few values, all one value, and two: the lower token comes first, among the kept and in the race."""
    torch = __import__("torch")
    settings = dict(top_k=[0, 700, 100, 1, 0, 2500, 0, 3], top_p=[0.3, 1.0, 0.5, 1.0, 0.9, 0.5, 1.0, 1.0])
    for values in (1, 2, 5):
        x, noise = rows(8, vocab, seed=vocab + values)
        x = (x * 10).long().remainder(values).to(getattr(torch, type)) * 0.25
        check(cuda_lib, x, noise, **settings)
        check(cuda_lib, x, torch.ones_like(noise), **settings)
        check(cuda_lib, x * -400, noise, temperature=[3.0] * 8, **settings)


@pytest.mark.parametrize("type", ["float32", "bfloat16", "float16"])
def test_masks_and_values_that_are_not_finite(cuda_lib, type):
    torch = __import__("torch")
    inf, nan = float("inf"), float("nan")
    low = torch.finfo(getattr(torch, type)).min
    x, noise = rows(12, 2500, type, seed=4, likely=3)
    x[0] = -inf                       # no token at all
    x[1, 5:] = -inf
    x[2, :2499] = -inf                # one
    x[3, ::2] = nan
    x[4] = nan
    x[5, 7] = x[5, 2000] = inf
    x[6] = low                        # masked by the lowest value: all alike
    x[7, 100:] = low
    x[8, :] = -inf
    x[8, 1234] = low
    x[9, 3] = inf
    x[9, 4:] = low
    x[10, ::3] = -inf
    x[11] = inf
    for settings in (dict(), dict(top_p=[0.8] * 12), dict(top_k=[30] * 12), dict(top_k=[2000] * 12, top_p=[0.7] * 12),
                     dict(min_p=[0.02] * 12), dict(temperature=[0.0] * 12), dict(temperature=[1e-30] * 12),
                     dict(temperature=[1e30] * 12, top_p=[0.5] * 12)):
        tokens = check(cuda_lib, x, noise, **settings)
        assert tokens[0] == 0 and tokens[2] == 2499 and tokens[8] == 1234


def test_settings_that_are_not_numbers_keep_the_first(cuda_lib):
    nan = float("nan")
    x, noise = rows(4, 5000, seed=5)
    first = x.argmax(1).tolist()
    assert cuda_lib.sample_tokens(x, noise, temperature=x.new_tensor([nan, -1.0, 0.0, 1e-38])).tolist() == first
    assert cuda_lib.sample_tokens(x, noise, top_p=x.new_tensor([nan, -1.0, 0.0, 1e-38])).tolist() == first
    assert cuda_lib.sample_tokens(x, noise, min_p=x.new_tensor([nan, 2.0, 1.0, float("inf")])).tolist() == first


@pytest.mark.parametrize("vocab", [700, 20_000, 150_000])
@pytest.mark.parametrize("type", ["float32", "float16"])
def test_an_infinite_temperature(cuda_lib, vocab, type):
    """All tokens that are not masked weigh the same."""
    x, noise = rows(3, vocab, type, seed=24)
    x[1, 5::7] = -float("inf")
    x[2, : vocab - 3] = -float("inf")
    for t in (float("inf"), 1e35, 1e30):
        check(cuda_lib, x, noise, temperature=[t] * 3, top_p=[0.5] * 3)
        check(cuda_lib, x, noise, temperature=[t] * 3, top_k=[9] * 3, min_p=[0.5] * 3)
        check(cuda_lib, x, noise, temperature=[t] * 3)


def test_values_far_apart(cuda_lib):
    """Clusters of values many powers of two apart, in denormal steps too: the search for a cut goes on in the bits."""
    torch = __import__("torch")
    x, noise = rows(6, 9000, seed=6)
    x[0] = x[0].abs() * 1e-42
    x[1] = x[1] * 1e30
    x[2, ::2] *= 1e-30
    x[3] = x[3] * 1e-38
    x[3, 0] = 20.0
    x[4] = torch.nextafter(torch.ones_like(x[4]), x[4])
    x[5, 1000:] = x[5, 1000:] * 1e-3 + 3e38
    for t in (1.0, 1e25, 1e-25):
        check(cuda_lib, x, noise, temperature=[t] * 6, top_p=[0.5] * 6)
        check(cuda_lib, x, noise, temperature=[t] * 6, top_k=[3000] * 6, top_p=[0.5] * 6)


def test_quotients_that_float32_does_not_tell_apart(cuda_lib):
    """Noise that makes all quotients alike to 2^-24: the answer is that of 64 bits."""
    torch = __import__("torch")
    x, _ = rows(5, 3001, seed=7, spread=1.0)
    noise = torch.exp(x.double() - x.max(1, keepdim=True).values.double()).float()
    check(cuda_lib, x, noise)
    check(cuda_lib, x, noise, top_p=[0.7] * 5)
    check(cuda_lib, x, noise, top_k=[25] * 5)


def test_distribution(cuda_lib):
    """4,096 draws from one row: each kept token's count within 6 standard deviations, no other token drawn."""
    torch = __import__("torch")
    x, _ = rows(1, 12, seed=8, spread=1.0)
    n = 4096
    noise = torch.empty(n, 12, device="cuda").exponential_(generator=torch.Generator(device="cuda").manual_seed(9)).clamp_(min=1e-30)
    tokens = cuda_lib.sample_tokens(x.expand(n, 12), noise, top_k=torch.full((n,), 7, dtype=torch.int32, device="cuda"))
    p = torch.softmax(x[0].double(), 0)
    p[p.argsort(descending=True)[7:]] = 0
    p /= p.sum()
    count = torch.bincount(tokens.long(), minlength=12).double()
    assert ((count - n * p).abs() <= 6 * (n * p * (1 - p)).sqrt()).all()


def test_streams_and_kept_buffers(cuda_lib):
    torch = __import__("torch")
    x, noise = rows(9, 40_000, "bfloat16", seed=10, likely=5)
    want = cuda_lib.sample_tokens(x, noise, return_logprobs=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    tokens, logprobs = torch.empty(9, dtype=torch.int32, device="cuda"), torch.empty(9, device="cuda")
    got = cuda_lib.sample_tokens(x, noise, tokens=tokens, logprobs=logprobs, return_logprobs=True, stream=side)
    side.synchronize()
    assert got[0] is tokens and got[1] is logprobs and tokens.equal(want[0]) and logprobs.equal(want[1])
    assert cuda_lib.sample_tokens(x[:0], noise[:0]).shape == (0,)


def test_two_graphs(cuda_lib):
    """Captured twice, replayed in turn with other inputs."""
    torch = __import__("torch")
    x, noise = rows(5, 6000, seed=11, likely=4)
    p = torch.full((5,), 0.9, device="cuda")
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = cuda_lib.sample_tokens(x, noise, top_p=p)
        graphs.append((graph, out))
    for seed in (12, 13):
        a, b = rows(5, 6000, seed=seed, likely=4)
        x.copy_(a)
        noise.copy_(b)
        want = check(cuda_lib, x, noise, top_p=[0.9] * 5)
        for graph, out in graphs:
            graph.replay()
            assert out.equal(want)


@pytest.mark.parametrize("type,vocab", [("bfloat16", 65_528), ("bfloat16", 65_529), ("float32", 32_765), ("float32", 32_766),
                                        ("float16", 2041), ("float16", 2042), ("bfloat16", 4_300_001), ("float32", 2_200_003)])
def test_vocabularies_at_the_forms_ends(cuda_lib, type, vocab):
    """Either side of where a row is taken by another form, and beyond the most parts of a row; rows that begin off 16 bytes."""
    n = 3 if vocab < 10 ** 6 else 1
    x, noise = rows(n, vocab, type, seed=vocab, likely=9, stride=1)
    check(cuda_lib, x, noise, temperature=[0.9] * n, top_p=[0.95] * n)
    check(cuda_lib, x, noise, top_k=[64] * n, top_p=[0.95] * n)


@pytest.mark.parametrize("type", ["float32", "bfloat16"])
def test_more_rows_than_a_launch_takes(cuda_lib, type):
    """A batch gives what its parts give; its workspace serves them."""
    torch = __import__("torch")
    n, vocab = 530, 70_000
    x, noise = rows(n, vocab, type, seed=21, likely=9)
    g = torch.Generator(device="cuda").manual_seed(22)
    p = 0.5 + 0.5 * torch.rand(n, device="cuda", generator=g)
    k = torch.randint(0, 3, (n,), device="cuda", generator=g, dtype=torch.int32) * 30
    from paper_2607_16973_gb300.kvcache import _sample_need
    ws = torch.empty(_sample_need(n, vocab), dtype=torch.uint8, device="cuda")
    tokens, logprobs = cuda_lib.sample_tokens(x, noise, top_p=p, top_k=k, workspace=ws, return_logprobs=True)
    for a, b in ((0, 1), (1, 40), (40, 300), (300, 530)):
        some = cuda_lib.sample_tokens(x[a:b], noise[a:b], top_p=p[a:b], top_k=k[a:b], workspace=ws, return_logprobs=True)
        assert some[0].equal(tokens[a:b])
        assert (some[1] - logprobs[a:b]).abs().max() <= 2.0 ** -20  # (sums in another order, and float32's rounding below 16)
    check(cuda_lib, x[525:], noise[525:], top_p=p[525:].tolist(), top_k=k[525:].tolist())


@pytest.mark.parametrize("vocab", [3000, 100_000])
def test_noise_that_is_none(cuda_lib, vocab):
    """Zeros, negative numbers, NaN and infinities are taken as the ends of what counts: here all alike."""
    torch = __import__("torch")
    x, noise = rows(4, vocab, seed=23)
    noise[0] = 0.0
    noise[1] = -1.0
    noise[2] = float("nan")
    noise[3] = float("inf")
    for settings in (dict(), dict(top_p=x.new_full((4,), 0.9)), dict(top_k=torch.full((4,), 20, dtype=torch.int32, device="cuda"))):
        assert cuda_lib.sample_tokens(x, noise, **settings).tolist() == x.argmax(1).tolist()


@pytest.mark.parametrize("vocab", [20_000, 130_000])
def test_cuts_beside_a_step(cuda_lib, vocab):
    """Values on two levels, each with half of the weight but for some 2^-22: the cut of top-p 0.5 lies between them, closer
    than a step's weights are rounded."""
    torch = __import__("torch")
    x = torch.zeros(6, vocab, device="cuda")
    few = vocab // 50
    for i, off in enumerate((0.0, 2.0 ** -22, -2.0 ** -22, 2.0 ** -21, -2.0 ** -21, 1e-3)):
        x[i, :few] = float(np.log((vocab - few) / few * (1 + off)))
    noise = rows(6, vocab, seed=31)[1]
    check(cuda_lib, x, noise, top_p=[0.5] * 6)
