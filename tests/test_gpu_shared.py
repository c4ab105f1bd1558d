"""Which requests share tokens (KVCache.share), and attention that reads those once
(KVCache.shared_attention), against plain forms."""
import numpy as np
import pytest

from test_gpu_kvcache import Case, compare

pytestmark = pytest.mark.gpu


class Batch(Case):
    """Requests in groups: contexts[g] tokens in whole pages of which every request of group g holds the same, tails[g][i]
    tokens behind them, the last new[g] of which are new.  A context of 0: nothing is shared."""

    def __init__(self, tq, contexts, tails, new, *, page=64, part=False, **kw):
        held = [c // page * page for c in contexts]
        lens = [h + t for h, ts in zip(held, tails) for t in ts]
        counts = [m for ms in new for m in ms]
        super().__init__(tq, lens, counts, page=page, **kw)
        at = 0
        self.groups = [(0, 0)] * 0
        for h, ts in zip(held, tails):
            lead = self.slots[at]
            for j in range(at, at + len(ts)):
                self.table[self.slots[j], : h // page] = self.table[lead, : h // page]
            self.groups.append((at, len(ts), h))
            at += len(ts)
        self.refs[:] = np.bincount(self.table[self.table >= 0], minlength=len(self.refs))

    def plan(self):
        rows = []
        for first, members, tokens in self.groups:
            rows += [(first, members, tokens) if members > 1 and tokens else (i, 1, 0) for i in range(first, first + members)]
        return np.array(rows, np.int32).T.copy()


def expected_plan(table, lens, slots, starts, page):
    n, before = len(slots), [int(lens[s]) - int(starts[i + 1] - starts[i]) for i, s in enumerate(slots)]
    links = []
    for i in range(n - 1):
        same, a, b = 0, table[slots[i]], table[slots[i + 1]]
        while same < len(a) and a[same] == b[same] >= 0:
            same += 1
        links.append(max(0, min(before[i], before[i + 1], same * page)))
    out, i = np.zeros((3, n), np.int32), 0
    while i < n:
        j = i
        while j < n - 1 and links[j] > 0:
            j += 1
        out[:, i: j + 1] = [[i], [j - i + 1], [min(links[i: j]) if j > i else 0]]
        i = j + 1
    return out


@pytest.mark.parametrize("page,seed", [(16, 0), (64, 1), (256, 2)])
@pytest.mark.parametrize("n", [1, 2, 7, 33, 1023, 1025, 3000])
def test_share(cuda_lib, n, page, seed):
    """Random tables whose neighbours agree in some leading pages; some requests hold nothing or bring all that they hold."""
    torch = __import__("torch")
    rng = np.random.default_rng(seed + n)
    width = 300 if n < 100 else 20
    table = np.full((n + 2, width), -1, np.int32)
    slots = rng.permutation(n + 2)[:n].astype(np.int32)
    lens, new = np.zeros(n + 2, np.int32), rng.integers(0, 4, n)
    pages = 4 * width
    for i, s in enumerate(slots):
        have = int(rng.integers(0, width + 1)) if rng.random() < 0.9 else 0
        table[s, :have] = rng.integers(0, pages, have)
        if i and rng.random() < 0.8:
            same = int(rng.integers(0, width + 1)) if rng.random() < 0.7 else width
            table[s, :same] = table[slots[i - 1], :same]
        have = int((table[s] >= 0).cumprod().sum())
        lens[s] = rng.integers(0, have * page + 1)
        new[i] = min(new[i], lens[s])
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    d = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    z, f = torch.zeros(1, pages, 1, page, 64, dtype=torch.uint8, device="cuda"), torch.zeros(1, pages, 1, page // 16, device="cuda")
    cache = cuda_lib.KVCache.from_tensors(z, z, f, f, d(table), d(lens), d(np.zeros(pages, np.int32)))
    plan = cache.share(d(slots), d(starts))
    cache.check()
    assert np.array_equal(plan.cpu().numpy(), expected_plan(table, lens, slots, starts, page))


def test_share_of_invalid_entries(cuda_lib):
    """A slot that is not there, a length that is not valid, more new tokens than are held: alone; pages that are not there
    end what is shared."""
    torch = __import__("torch")
    case = Batch(cuda_lib, [256], [[10] * 8], [[1] * 8], seed=3)
    case.table[case.slots[7], 1] = case.table[case.slots[6], 1] = len(case.refs)
    cache = case.cache()
    slots, starts = case.slots.copy(), case.starts.copy()
    slots[2] = -1
    cache.lens[int(case.slots[4])] = 10 ** 6
    starts[6:] += 1000
    plan = cache.share(case.device(slots), case.device(starts))
    with pytest.raises(cuda_lib.TQError, match="left out"):
        cache.check()
    want = [[0, 2, 256], [0, 2, 256], [2, 1, 0], [3, 1, 0], [4, 1, 0], [5, 1, 0], [6, 2, 64], [6, 2, 64]]
    assert plan.t().tolist() == want
    out = torch.empty(3, 8, dtype=torch.int32, device="cuda")
    assert cache.share(case.device(case.slots), case.device(case.starts), plan=out) is out


def check(case, q, plan=None, groups=None, **kw):
    cache = case.cache()
    args = case.device(case.slots), case.device(case.starts)
    if plan is None:
        plan = cache.share(*args)
        cache.check()
        assert np.array_equal(plan.cpu().numpy(), case.plan())
    out, lse = cache.shared_attention(case.layer, *args, plan, q, groups=groups, return_lse=True, **kw)
    cache.check()
    compare(case, q, out, lse)
    return out, lse


BATCHES = [
    ([64], [[1, 1]], [[1, 1]]),                                                # nothing of their own but the new token
    ([0, 130], [[70], [3, 40]], [[1], [1, 1]]),                                # one alone
    ([200, 64, 0, 512], [[5, 1, 90], [20] * 4, [33], [200, 16, 17]], [[1] * 3, [1] * 4, [1], [1] * 3]),
    ([320], [[9, 30, 6, 100, 64]], [[9, 1, 5, 3, 1]]),                         # drafts
    ([1500], [[1] * 40], [[1] * 40]),                                          # a tile of rows, and several
    ([640, 64], [[130, 40], [257, 70]], [[120, 40], [130, 1]]),                # prompts behind a shared passage
]


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("contexts,tails,new", BATCHES)
@pytest.mark.parametrize("dim,group,type,tight", [(128, 4, "bfloat16", True), (64, 7, "float16", True),
                                                  (256, 2, "bfloat16", True), (128, 16, "float16", False)])
def test_shared(cuda_lib, codes, contexts, tails, new, dim, group, type, tight):
    case = Batch(cuda_lib, contexts, tails, new, dim=dim, codes=codes, seed=len(contexts) + dim).fill()
    check(case, case.queries(2 * group, type), groups=len(contexts) if tight else None)


@pytest.mark.parametrize("page", [16, 32, 256])
def test_shared_page_sizes(cuda_lib, page):
    case = Batch(cuda_lib, [900, 300], [[40, 7, 20], [1, 70, 3, 18]], [[1, 2, 1], [1, 1, 3, 1]], page=page, kv_heads=3, seed=page).fill()
    check(case, case.queries(12, "bfloat16"), groups=2)


@pytest.mark.parametrize("tokens", [1, 5, 16, 63, 130, 191])
def test_part_of_what_is_the_same_may_be_shared(cuda_lib, tokens):
    """A plan may name fewer tokens than the pages have in common: blocks and tiles begin inside."""
    case = Batch(cuda_lib, [192], [[3, 30, 1]], [[2, 1, 1]], codes="e4m3", seed=tokens).fill()
    plan = case.device(np.array([[0] * 3, [3] * 3, [tokens] * 3], np.int32))
    check(case, case.queries(8, "bfloat16"), plan, 1)
    wide = Batch(cuda_lib, [192], [[40, 30, 1]], [[33, 29, 1]], seed=tokens).fill()
    check(wide, wide.queries(16, "float16"), plan, 1)


def test_entries_that_do_not_fit_are_attended_by_themselves(cuda_lib):
    case = Batch(cuda_lib, [128, 192], [[4, 9, 30], [5, 20, 7, 1]], [[1, 2, 1], [1, 1, 1, 1]], seed=9).fill()
    q, good = case.queries(8, "bfloat16"), case.plan()
    for row, i, x in ((0, 1, 2), (0, 5, -1), (1, 0, 2), (1, 3, 70000), (2, 4, 10 ** 9), (2, 2, -7), (2, 0, 64), (0, 6, 2 ** 31 - 1),
                      (1, 6, 2 ** 31 - 1), (2, 3, 193 + 64)):
        bad = good.copy()
        bad[row, i] = x
        cache = case.cache()
        out, lse = cache.shared_attention(case.layer, case.device(case.slots), case.device(case.starts), case.device(bad), q,
                                          groups=2, return_lse=True)
        with pytest.raises(cuda_lib.TQError, match="left out"):
            cache.check()
        compare(case, q, out, lse)


def test_padding_empty_requests_and_invalid_slots(cuda_lib):
    """Rows in front of and behind the requests get zeros and -inf; a request without new tokens writes nothing; a
    member whose slot is not there is left out, the others of its group are not."""
    case = Batch(cuda_lib, [128], [[4, 9, 30, 6]], [[1, 0, 2, 1]], seed=10).fill()
    q = case.queries(8, "bfloat16")
    padded = q.repeat(3, 1, 1)
    cache = case.cache()
    slots = case.slots.copy()
    slots[3] = 99
    starts = case.starts + 4
    out, lse = cache.shared_attention(case.layer, case.device(slots), case.device(starts), case.device(case.plan()), padded,
                                      groups=1, return_lse=True)
    with pytest.raises(cuda_lib.TQError, match="left out"):
        cache.check()
    case.slots, case.starts = case.slots[:3], case.starts[:4]
    compare(case, q[:3], out[4:7], lse[4:7])
    rest = [0, 1, 2, 3] + list(range(7, 12))
    assert not out[rest].any() and (lse[rest] == -np.inf).all()


def test_queries_that_are_not_finite(cuda_lib):
    case = Batch(cuda_lib, [128], [[4, 9, 30]], [[1, 1, 2]], seed=11).fill()
    cache, q = case.cache(), case.queries(8, "bfloat16")
    args = case.layer, case.device(case.slots), case.device(case.starts), case.device(case.plan())
    good = cache.shared_attention(*args, q, groups=1)
    q[1, 3, 5] = float("nan")
    out, lse = cache.shared_attention(*args, q, groups=1, return_lse=True)
    assert out[1, 3].isnan().all() and lse[1, 3].isnan()
    out[1, 3] = good[1, 3]
    assert out.equal(good)


def test_a_kept_workspace_and_equal_calls(cuda_lib):
    torch = __import__("torch")
    most = Batch(cuda_lib, *BATCHES[4]).cache().shared_attention_workspace(40, 400, 8)
    ws = torch.empty(most, dtype=torch.uint8, device="cuda")
    for contexts, tails, new in BATCHES:
        case = Batch(cuda_lib, contexts, tails, new, seed=12).fill()
        ws.fill_(0xFF)
        q = case.queries(8, "bfloat16")
        a = check(case, q, groups=len(contexts), workspace=ws)
        b = check(case, q, groups=len(contexts), workspace=ws)
        assert a[0].equal(b[0]) and a[1].equal(b[1])


def test_a_step_of_a_server_in_a_graph(cuda_lib):
    """Passages prompted once, forked, extended; share, shared attention, cross attention and sampling captured together and
    replayed on another stream, against the same calls without sharing."""
    torch = __import__("torch")
    tq = cuda_lib
    g = torch.Generator(device="cuda").manual_seed(1)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = tq.KVCache(pages=64, slots=8, max_pages=8, kv_heads=2, head_dim=64, page_tokens=32)
    rows = lambda m, h: torch.randn(m, h, 64, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    passages, requests = ints(0, 1), ints(2, 3, 4, 5, 6)
    cache.extend(passages, ints(100, 77))
    cache.append(0, passages, ints(0, 100, 177), rows(177, 2), rows(177, 2))
    cache.fork(requests, ints(0, 0, 0, 1, 1))
    cache.extend(requests, ints(6, 2, 9, 3, 3))
    cache.append(0, requests, ints(0, 6, 8, 17, 20, 23), rows(23, 2), rows(23, 2))
    starts, counts = ints(0, 1, 2, 3, 4, 5), ints(1, 1, 1, 1, 1)
    q, k, v = rows(5, 8), rows(5, 2), rows(5, 2)
    head = torch.randn(8 * 64, 999, device="cuda", generator=g).to(torch.bfloat16) / 8
    noise = torch.empty(5, 999, device="cuda").exponential_(generator=g)

    def step():
        cache.extend(requests, counts)
        cache.append(0, requests, starts, k, v)
        plan = cache.share(requests, starts)
        o = cache.shared_attention(0, requests, starts, plan, q, groups=2)
        c = cache.cross_attention(0, ints_of, starts, q)
        logits = (o + c).flatten(1) @ head
        return plan, o, c, logits, tq.sample_tokens(logits, noise, top_p=p)

    ints_of, p = ints(0, 0, 0, 1, 1), torch.full((5,), 0.9, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            plan, o, c, logits, tokens = step()
        for _ in range(3):
            graph.replay()
    side.synchronize()
    cache.check()
    assert plan.t().tolist() == [[0, 3, 96]] * 3 + [[3, 2, 64]] * 2
    assert cache.lens[2:7].tolist() == [110, 106, 113, 84, 84]
    plain = cache.attention(0, requests, starts, q)
    assert (o.float() - plain.float()).abs().max() <= 2 ** -7 * plain.float().abs().max()
    assert tokens.equal(tq.sample_tokens(logits, noise, top_p=p))
