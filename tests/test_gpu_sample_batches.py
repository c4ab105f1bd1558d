"""tq_sample on batches of as many rows as take the longest parts, and rows whose weight
lies close together, against its definition in 64 bits."""
import numpy as np
import pytest

from sampleref import sample
from test_gpu_sample import MIXED, SLACK, rows

pytestmark = pytest.mark.gpu


def check(tq, logits, noise, picked=None, **settings):
    """As test_gpu_sample.check, for the rows `picked` of one call's answers."""
    torch = __import__("torch")
    kinds = {"temperature": torch.float32, "top_k": torch.int32, "top_p": torch.float32, "min_p": torch.float32}
    given = {name: torch.tensor(x, dtype=kinds[name], device="cuda") for name, x in settings.items()}
    tokens, logprobs = tq.sample_tokens(logits, noise, **given, return_logprobs=True)
    values = {name: t.double().cpu().tolist() for name, t in given.items()}
    for i in range(logits.shape[0]) if picked is None else picked:
        s = {name: (int(v[i]) if name == "top_k" else v[i]) for name, v in values.items()}
        x, e = logits[i].double().cpu().numpy(), noise[i].double().cpu().numpy()
        want = [sample(x, e, **s, slack=slack) for slack in (0.0, SLACK, -SLACK)]
        token, logprob = int(tokens[i]), float(logprobs[i])
        assert token in [t for t, _ in want], (i, s, token, want)
        ref = dict(want)[token]
        assert logprob == ref or abs(logprob - ref) <= 2.0 ** -24 * abs(ref) + 2.0 ** -21, (i, s, logprob, ref)
    return tokens


def favour(logits, noise, temperature, top_p, behind):
    """Noise that lets a token a little in front of the cut win, or one a little behind it that must not."""
    torch = __import__("torch")
    for i in range(logits.shape[0]):
        x = logits[i].double()
        order = torch.argsort(x, descending=True, stable=True)
        w = torch.exp((x[order] - x[order[0]]) / temperature[i])
        count = int((w.cumsum(0) - w < top_p[i] * w.sum()).sum())
        at = min(len(order) - 1, count + len(order) // 1000) if behind[i] else max(0, count - 1 - len(order) // 1000)
        noise[i, order[at]] = 2.0 ** -60


@pytest.mark.parametrize("type,vocab", [("bfloat16", 128_000), ("float16", 128_000), ("float32", 100_003), ("float32", 128_000)])
def test_rows_whose_weight_lies_in_few_steps(cuda_lib, type, vocab):
    """Equal logits, all of them at a step's upper end, a small spread, high temperatures: a part's tokens all in a few of the
    steps that the cut of top-p is found by."""
    torch = __import__("torch")
    n = 64
    logits, noise = rows(n, vocab, type, seed=vocab, spread=1.0)
    temperature, top_p, behind = [], [], []
    for i in range(n):
        kind = i % 6
        if kind == 0:
            logits[i] = 0.0
        elif kind == 1:
            logits[i] = 1 / 64
        elif kind < 4:
            logits[i] *= 0.01 * (kind - 1)
        else:
            logits[i] *= 2
        temperature.append((1.0, 1.0, 1.0, 1.0, 100.0, float("inf"))[kind])
        top_p.append((0.5, 0.9, 0.99999)[i // 6 % 3])
        behind.append(i // 18 % 2 == 0)
    favour(logits, noise, temperature, top_p, behind)
    check(cuda_lib, logits, noise, picked=range(42), temperature=temperature, top_p=top_p)


@pytest.mark.parametrize("n,vocab", [(64, 100_003), (64, 20_000), (64, 900)])
@pytest.mark.parametrize("temperature", [1.0, 1.3])
def test_near_ties_of_tokens_far_below_the_first(cuda_lib, n, vocab, temperature):
    """Two tokens of 2^-60 to 2^-110 whose noise makes their quotients alike to 2^-19, in different parts of the row: the one
    that is ahead in 64 bits."""
    torch = __import__("torch")
    rng = np.random.default_rng(vocab)
    logits, noise = rows(n, vocab, seed=vocab, spread=1.0)
    noise.fill_(1.0)
    x, e = logits.cpu().numpy(), noise.cpu().numpy()
    want = []
    for i in range(n):
        a, b = (int(v) for v in rng.choice(vocab // 2 - 1, 2) + [0, vocab // 2])
        x[i, [a, b]] = -rng.uniform(60, 110, 2) * np.log(2.0) * temperature
        top = x[i].astype(np.float64).max()
        w = np.exp((x[i, [a, b]].astype(np.float64) - top) / float(np.float32(temperature)))
        e[i, [a, b]] = w * 2.0 ** -10 * [1, 1 + rng.choice([-1, 1]) * 2.0 ** -19]
        want.append((a, b)[int(np.argmax(w / e[i, [a, b]].astype(np.float64)))])
    logits.copy_(torch.from_numpy(x))
    noise.copy_(torch.from_numpy(e))
    t = torch.full((n,), temperature, device="cuda")
    assert cuda_lib.sample_tokens(logits, noise, temperature=t).tolist() == want
    assert cuda_lib.sample_tokens(logits, noise, temperature=t, min_p=torch.full((n,), 2.0 ** -125, device="cuda")).tolist() == want


def test_a_border_of_min_p_far_below_the_first(cuda_lib):
    """Tokens of 2^-100, some 2^-17 in front of min-p's border and some behind, with noise that lets them win: those in front
    do, as if the others were not there."""
    torch = __import__("torch")
    n, vocab, temperature = 64, 100_003, 1.3
    rng = np.random.default_rng(3)
    logits, noise = rows(n, vocab, seed=3, spread=1.0)
    noise.fill_(1.0)
    x, e = logits.cpu().numpy(), noise.cpu().numpy()
    min_p, want = np.empty(n, np.float32), []
    for i in range(n):
        a, b = (int(v) for v in rng.choice(vocab, 2, replace=False))
        x[i, a] = -rng.uniform(90, 110) * np.log(2.0) * temperature
        x[i, b] = np.nextafter(x[i, a], np.float32(-np.inf))
        top = x[i].astype(np.float64).max()
        w = np.exp((x[i, [a, b]].astype(np.float64) - top) / float(np.float32(temperature)))
        min_p[i] = np.sqrt(w[0] * w[1])
        assert w[0] > min_p[i] * (1 + 2.0 ** -20) and w[1] < min_p[i] * (1 - 2.0 ** -20)
        e[i, a], e[i, b] = w[0] * 2.0 ** -10, w[1] * 2.0 ** -14
        want.append(a)
    logits.copy_(torch.from_numpy(x))
    noise.copy_(torch.from_numpy(e))
    t = torch.full((n,), temperature, device="cuda")
    assert cuda_lib.sample_tokens(logits, noise, temperature=t, min_p=torch.from_numpy(min_p).cuda()).tolist() == want


BATCHES = [("bfloat16", 128_000), ("float16", 128_000), ("float32", 100_003)]


@pytest.mark.parametrize("type,vocab", BATCHES)
@pytest.mark.parametrize("likely", [0, 24])
def test_settings_of_all_kinds(cuda_lib, type, vocab, likely):
    n = 64
    logits, noise = rows(n, vocab, type, seed=vocab + likely + 1, likely=likely)
    settings = [MIXED[i % len(MIXED)] for i in range(n)]
    check(cuda_lib, logits, noise, picked=range(24), **dict(zip(("temperature", "top_k", "top_p", "min_p"), map(list, zip(*settings)))))


@pytest.mark.parametrize("type,vocab", BATCHES)
@pytest.mark.parametrize("values", [1, 2, 5])
def test_ties_in_batches(cuda_lib, type, vocab, values):
    torch = __import__("torch")
    n = 64
    x, noise = rows(n, vocab, seed=vocab + values)
    x = (x * 10).long().remainder(values).to(getattr(torch, type)) * 0.25
    top_k, top_p = [0, 700, 100, 1, 0, 2500, 0, 3] * 8, [0.3, 1.0, 0.5, 1.0, 0.9, 0.5, 1.0, 1.0] * 8
    check(cuda_lib, x, noise, picked=range(8), top_k=top_k, top_p=top_p)
    check(cuda_lib, x, torch.ones_like(noise), picked=range(8, 16), top_k=top_k, top_p=top_p)
    check(cuda_lib, x * -400, noise, picked=range(8), temperature=[3.0] * n, top_k=top_k, top_p=top_p)


@pytest.mark.parametrize("type,vocab", BATCHES)
def test_masks_and_values_that_are_not_finite_in_batches(cuda_lib, type, vocab):
    torch = __import__("torch")
    inf, n = float("inf"), 64
    low = torch.finfo(getattr(torch, type)).min
    x, noise = rows(n, vocab, type, seed=4, likely=3)
    x[0] = -inf
    x[1, 5:] = -inf
    x[2, : vocab - 1] = -inf
    x[3, ::2] = float("nan")
    x[4, 7] = x[4, 2000] = inf
    x[5] = low
    x[6, 100:] = low
    x[7, ::3] = -inf
    x[8, 9000:] = -inf  # whole parts that are masked
    x[9, : vocab - 9000] = -inf
    for settings in (dict(), dict(top_p=0.8), dict(top_k=30), dict(top_k=2000, top_p=0.7), dict(min_p=0.02), dict(temperature=0.0),
                     dict(temperature=1e30, top_p=0.5)):
        tokens = check(cuda_lib, x, noise, picked=range(10), **{name: [v] * n for name, v in settings.items()})
        assert tokens[0] == 0 and tokens[2] == vocab - 1


@pytest.mark.parametrize("type,vocab", BATCHES)
def test_cuts_beside_a_step_in_batches(cuda_lib, type, vocab):
    """Values on two levels, each with half of the weight but for some 2^-22 (float32) or what the type rounds it to."""
    torch = __import__("torch")
    n, few = 64, vocab // 50
    x = torch.zeros(n, vocab, device="cuda")
    for i, off in enumerate((0.0, 2.0 ** -22, -2.0 ** -22, 2.0 ** -21, -2.0 ** -21, 1e-3)):
        x[i, :few] = float(np.log((vocab - few) / few * (1 + off)))
    noise = rows(n, vocab, seed=31)[1]
    check(cuda_lib, x.to(getattr(torch, type)), noise, picked=range(7), top_p=[0.5] * n)


@pytest.mark.parametrize("type,vocab", BATCHES)
def test_quotients_alike_in_batches(cuda_lib, type, vocab):
    torch = __import__("torch")
    n = 64
    x, _ = rows(n, vocab, type, seed=7, spread=1.0)
    noise = torch.exp(x.double() - x.max(1, keepdim=True).values.double()).float()
    check(cuda_lib, x, noise, picked=range(3))
    check(cuda_lib, x, noise, picked=range(3), top_p=[0.7] * n)
    check(cuda_lib, x, noise, picked=range(3), top_k=[25] * n)
