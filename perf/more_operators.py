"""What a generator asks besides its own decoding loop, as cases that can be timed.

Beside the calls that every step makes, a program that answers from retrieved
passages has these:

* ``cross``: queries over all tokens of an encoder's states in the 8-bit cache,
  whatever their own number and place (a reader over encoded passages);
* ``share``: which neighbouring requests of a batch hold the same first pages,
  and how many tokens those are;
* ``shared``: causal attention of such a batch, the shared tokens read once for
  all requests that hold them;
* ``sample``: the next token of each request from its logits, by temperature,
  top-k, top-p and min-p, from given random numbers.

Every case has a plain form in elementary torch operations (``own = False``)
beside the calls of the library (``own = True``).  A cache's pages lie in
shuffled order, as they do after some time of service.  The lengths of a batch
of queries are the same for every seed, in another order.
"""
import math

import torch

own = False

_BLOCK = 16  # tokens that share a scale
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    def cross(name, seqs, new, length, heads=16, kv_heads=16, dim=64, page=64, codes="int8", type="bf16"):
        return {"name": name, "op": "cross", "seqs": seqs, "new": new, "length": length, "heads": heads,
                "kv_heads": kv_heads, "dim": dim, "page": page, "codes": codes, "type": type}

    def share(name, seqs, contexts, length, alone=0, page=64):
        return {"name": name, "op": "share", "seqs": seqs, "contexts": contexts, "alone": alone, "length": length,
                "tail": 60, "new": 1, "page": page}

    def shared(name, seqs, contexts, length, tail, new=1, alone=0, heads=32, kv_heads=8, dim=128, page=64, codes="int8",
               type="bf16"):
        return {"name": name, "op": "shared", "seqs": seqs, "contexts": contexts, "alone": alone, "length": length,
                "tail": tail, "new": new, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "codes": codes,
                "type": type}

    def sample(name, seqs, vocab, kind, type="bf16", flat=False):
        return {"name": name, "op": "sample", "seqs": seqs, "vocab": vocab, "kind": kind, "type": type, "flat": flat}

    return [
        # one decoding step of one reader over a passage: latency
        cross("cross-one", 1, 1, 700),
        # a decoding step of a batch of readers, each over its own passages
        cross("cross-batch", 96, 1, 5000, codes="e4m3"),
        # the scores of candidate answers of 300 tokens, each over the passages of its question
        cross("cross-answers", 7, 300, 6001, heads=32, kv_heads=8, dim=128, type="fp16"),
        # a small server's step: four passages, sixteen requests
        share("share-16", 16, 4, 700),
        # a burst over long contexts in small pages, some requests with passages of their own
        share("share-2000", 2000, 61, 16_000, alone=40, page=16),
        # eight answers to one question: latency
        shared("shared-one", 8, 1, 1500, 40),
        # a decoding step of a server, a few contexts that many requests ask, some requests with their own
        shared("shared-batch", 64, 4, 12_000, 600, alone=3, codes="e4m3"),
        # everyone asks one long collection
        shared("shared-long", 256, 1, 60_001, 300),
        # drafted tokens scored at once, an odd group, a narrow head
        shared("shared-drafts", 24, 3, 8190, 200, new=5, heads=40, dim=64, codes="e4m3", type="fp16"),
        # one interactive request
        sample("sample-one", 1, 32_000, "both"),
        # a batch of requests with settings of their own
        sample("sample-batch", 256, 128_000, "mixed"),
        # flat distributions in float32, as a hot sampler of synthetic questions has them; rows that start off 16 bytes
        sample("sample-flat", 48, 100_003, "top_p", type="fp32", flat=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["cross", "share", "shared", "shared", "sample", "sample"])
    page = rng.choice([16, 32, 64, 64, 128])
    if op == "sample":
        seqs = _log_uniform(rng, 1, 256)
        return {"op": op, "seqs": seqs, "vocab": _log_uniform(rng, 1000, min(300_000, 32_000_000 // seqs)),
                "kind": rng.choice(["both", "mixed", "top_p", "top_k", "min_p", "free"]),
                "type": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "flat": rng.random() < 0.4}
    if op == "share":
        seqs = _log_uniform(rng, 4, 2000)
        return {"op": op, "seqs": seqs, "contexts": _log_uniform(rng, 2, max(3, min(61, seqs // 2))),
                "alone": rng.choice([0, seqs // 20]), "length": _log_uniform(rng, 20, 16_000), "tail": 60,
                "new": rng.choice([1, 1, 4]), "page": page}
    kv_heads, dim = rng.choice([1, 2, 4, 8, 8]), rng.choice([64, 128, 128, 128, 256])
    case = {"op": op, "heads": kv_heads * rng.choice([1, 2, 4, 4, 5, 7, 8, 16]), "kv_heads": kv_heads, "dim": dim,
            "page": page, "codes": rng.choice(["int8", "e4m3"]), "type": rng.choice(["bf16", "bf16", "fp16"])}
    if op == "cross":
        if rng.random() < 0.4:
            new, seqs = _log_uniform(rng, 2, 1000), rng.choice([1, 2, 3, 5])
            new = max(2, min(new, 32_768 // case["heads"]))
            length = _log_uniform(rng, 1, 7000 // seqs)
        else:
            new, seqs = 1, _log_uniform(rng, 1, 128)
            length = _log_uniform(rng, 1, min(100_000, 2_000_000 // (seqs * kv_heads * dim // 64)))
        return {**case, "seqs": seqs, "new": new, "length": length}
    seqs = _log_uniform(rng, 2, 256)
    contexts = _log_uniform(rng, 1, max(2, min(16, seqs // 2)))
    new = rng.choice([1, 1, 1, 2, 5])
    most = 8_000_000_000 // (4 * case["heads"] * new * seqs) // 2  # (the plain form's scores)
    return {**case, "seqs": seqs, "contexts": contexts, "alone": rng.choice([0, 0, 1]),
            "length": _log_uniform(rng, 20, max(30, min(60_000, most, 40_000_000 // (contexts * kv_heads * dim)))),
            "tail": _log_uniform(rng, 1, max(2, min(600, 20_000_000 // (seqs * kv_heads * dim)))), "new": new}


# ---- sizes ------------------------------------------------------------------

def _spread(n, most, least):
    """n lengths, from a quarter of `most` to `most` in even steps, none below `least`; one alone is `most`."""
    if n == 1:
        return [max(least, most)]
    return [max(least, most // 4 + (most - most // 4) * i // (n - 1)) for i in range(n)]


def _new_counts(case):
    """New tokens of each sequence: every second one has some fewer (a step of single tokens has one each)."""
    new = case["new"]
    return [new if i % 2 == 0 or new == 1 else max(1, new - 1 - i % max(1, new // 2)) for i in range(case["seqs"])]


def _batch(case):
    """A batch over shared contexts, request by request: [(context, its length, tokens behind it, new ones among them)];
    the last `alone` requests have a context each."""
    contexts, alone = case["contexts"], case["alone"]
    held = case["seqs"] - alone
    lengths = _spread(contexts, case["length"], 1) + _spread(alone, case["length"], 1)
    sizes = [held // contexts + (i < held % contexts) for i in range(contexts)]
    for i in range(0, contexts - 1, 2):  # (some are asked more often than others)
        moved = sizes[i] // 3
        sizes[i], sizes[i + 1] = sizes[i] - moved, sizes[i + 1] + moved
    owners = [c for c, size in enumerate(sizes) for _ in range(size)] + [contexts + i for i in range(alone)]
    tails = _spread(len(owners), case["tail"], 1)
    return [(c, lengths[c], tails[i * 7 % len(owners)] + new, new) for i, (c, new) in enumerate(zip(owners, _new_counts(case)))]


def _members(batch):
    """Requests of each context."""
    count = {}
    for c, *_ in batch:
        count[c] = count.get(c, 0) + 1
    return count


def work(case):
    op = case["op"]
    if op == "sample":  # the logits; the random numbers of the rows that keep every token
        size = {"fp32": 4, "bf16": 2, "fp16": 2}[case["type"]]
        free = sum(kind == "free" for kind in _kinds(case))
        return {"bytes": case["vocab"] * (case["seqs"] * size + free * 4) + case["seqs"] * 24, "flops": 0}
    if op == "share":
        pages = sum(length // case["page"] + 1 for _, length, *_ in _batch(case))
        return {"bytes": 4 * pages + case["seqs"] * (4 + 4 + 4 + 12), "flops": 0}
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    block = kv_heads * (_BLOCK * dim + 4)  # codes and scales of a block, keys or values
    per_query = heads * (2 * 2 * dim + 4)  # its query, output and sum
    if op == "cross":
        both = list(zip(_spread(case["seqs"], case["length"], 1), _new_counts(case)))
        return {"bytes": sum(2 * block * -(-length // _BLOCK) + new * per_query for length, new in both),
                "flops": 4 * dim * heads * sum(length * new for length, new in both)}
    batch, total, pairs = _batch(case), 0, 0
    for c, length in {c: length for c, length, *_ in batch}.items():
        total += 2 * block * -(-length // _BLOCK)
    for _, length, tail, new in batch:
        total += 2 * block * -(-tail // _BLOCK) + new * per_query
        pairs += sum(length + tail - new + i + 1 for i in range(new))
    return {"bytes": total, "flops": 4 * dim * heads * pairs}


# ---- inputs -----------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _codes(shape, codes, g):
    """Codes as quantised activations have them: bell-shaped, the largest of a block at the end of the range."""
    out = torch.empty(shape, dtype=torch.uint8, device="cuda")
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 28):
        part = flat[a: a + (1 << 28)]
        x = torch.randn(part.numel(), dtype=torch.float32, device="cuda", generator=g)
        if codes == "int8":
            part.copy_(x.mul_(36).round_().clamp_(-127, 127).to(torch.int8).view(torch.uint8))
        else:
            part.copy_(x.mul_(127).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    return out


def _scales(shape, codes, g):
    s = torch.randn(shape, dtype=torch.float32, device="cuda", generator=g).mul_(0.2).exp_()
    return s.mul_(1 / 36 if codes == "int8" else 1 / 127)


def _pool(pages, kv_heads, page, dim, codes, g):
    shape, scales = (1, pages, kv_heads, page, dim), (1, pages, kv_heads, page // _BLOCK)
    return {"k": _codes(shape, codes, g), "v": _codes(shape, codes, g), "k_scale": _scales(scales, codes, g),
            "v_scale": _scales(scales, codes, g), "codes": codes}


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "sample":
        return _prepare_sample(case, g)
    if case["op"] == "cross":
        return _prepare_cross(case, g)
    return _prepare_batch(case, g)


def _queries(case, total, g):
    """Queries as a projection gives them beside keys and values: a row of them all for each token."""
    heads, kv_heads = case["heads"], case["kv_heads"]
    rows = torch.randn(total, heads + 2 * kv_heads, case["dim"], dtype=torch.float32, device="cuda", generator=g)
    return rows.to(_TYPES[case["type"]])[:, :heads] * 2


def _prepare_cross(case, g):
    n, page = case["seqs"], case["page"]
    shuffle = torch.randperm(n, device="cuda", generator=g).tolist()
    lengths = [_spread(n, case["length"], 1)[i] for i in shuffle]
    counts = [_new_counts(case)[i] for i in shuffle]
    slots = n + 3
    slot = torch.randperm(slots, device="cuda", generator=g)[:n].tolist()
    need = [-(-length // page) for length in lengths]
    pages = sum(need) + 5
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((slots, max(need) + 1), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(slots, dtype=torch.int32, device="cuda")
    at = 0
    for s, length, k in zip(slot, lengths, need):
        table[s, :k] = order[at: at + k]
        lens[s] = length
        at += k
    starts = [0]
    for new in counts:
        starts.append(starts[-1] + new)
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[order[:at].long()] = 1
    return {"case": dict(case), **_pool(pages, case["kv_heads"], page, case["dim"], case["codes"], g), "table": table,
            "lens": lens, "refs": refs, "slots": _ints(slot), "starts": _ints(starts), "most_new": max(counts),
            "most": max(lengths), "q": _queries(case, starts[-1], g)}


def _prepare_batch(case, g):
    """Requests that hold the whole pages of their context together and the rest by themselves, those of one context side
    by side, the contexts in an order of the seed's."""
    page, batch = case["page"], _batch(case)
    n, count = len(batch), _members(batch)
    by_context = {c: [r for r in batch if r[0] == c] for c in count}
    names = list(by_context)
    order = [names[i] for i in torch.randperm(len(names), device="cuda", generator=g).tolist()]
    more = [0] * len(names)
    if case["op"] == "share":  # (its answer would be the same lengths otherwise)
        more = torch.randint(4 * page, (len(names),), device="cuda", generator=g).tolist()
    extra = dict(zip(names, more))
    rows = [(c, length + extra[c], tail, new) for c in order for _, length, tail, new in by_context[c]]
    whole = {c: length // page for c, length, _, _ in rows}
    rest = [-(-(length + tail) // page) - whole[c] for c, length, tail, _ in rows]
    pages = sum(whole.values()) + sum(rest) + 5
    free = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    slots = n + 3
    slot = torch.randperm(slots, device="cuda", generator=g)[:n]
    width = max(whole[c] + r for (c, *_), r in zip(rows, rest)) + 1
    # each row's pages: its context's, then its own; by their places in `free`
    first, at = {}, 0
    for c in order:
        first[c] = at
        at += whole[c]
    begin = []
    for r in rest:
        begin.append(at)
        at += r
    place = torch.arange(width, device="cuda")[None]
    w = _ints([whole[c] for c, *_ in rows])[:, None]
    where = torch.where(place < w, place + _ints([first[c] for c, *_ in rows])[:, None],
                        place - w + _ints(begin)[:, None])
    there = place < w + _ints(rest)[:, None]
    table = torch.full((slots, width), -1, dtype=torch.int32, device="cuda")
    table[slot] = torch.where(there, free[where.clamp(max=pages - 1).long()], torch.full_like(place, -1).to(torch.int32))
    lens = torch.zeros(slots, dtype=torch.int32, device="cuda")
    lens[slot] = _ints([length + tail for _, length, tail, _ in rows])
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    held = table[slot]
    refs.index_add_(0, held[held >= 0].long(), torch.ones_like(held[held >= 0]))
    starts = [0]
    for *_, new in rows:
        starts.append(starts[-1] + new)
    state = {"case": dict(case), "table": table, "lens": lens, "refs": refs, "slots": slot.to(torch.int32),
             "starts": _ints(starts)}
    if case["op"] == "share":
        return {**state, **_pool(pages, 1, page, 64, "int8", g)}
    # what `share` says of it: (first request, requests, tokens) of each request's group
    plan, at = [], 0
    for c in order:
        k = count[c]
        plan += [(at, k, whole[c] * page) if k > 1 and whole[c] else (i, 1, 0) for i in range(at, at + k)]
        at += k
    leads = sorted({(a, k, s) for a, k, s in plan if s})
    tails = [length + tail - s for (_, length, tail, _), (*_, s) in zip(rows, plan)]
    sizes = {"most_tail": max(tails), "leads": leads, "most_new": max(new for *_, new in rows)}
    return {**state, **_pool(pages, case["kv_heads"], page, case["dim"], case["codes"], g), **sizes,
            "plan": _ints(plan).t().contiguous(), "groups": len(names), "q": _queries(case, starts[-1], g)}


def _kinds(case):
    """What the settings of each row are."""
    if case["kind"] != "mixed":
        return [case["kind"]] * case["seqs"]
    return [("top_p", "both", "top_k", "min_p", "greedy", "top_p", "both", "free")[i % 8] for i in range(case["seqs"])]


#             temperature  top-k  top-p  min-p
_SETTINGS = {"top_p": (1.0, 0, 0.9, 0.0), "both": (0.7, 50, 0.95, 0.0), "top_k": (1.2, 40, 1.0, 0.0),
             "min_p": (1.0, 0, 1.0, 0.05), "greedy": (0.0, 0, 1.0, 0.0), "free": (1.0, 0, 1.0, 0.0)}


def _prepare_sample(case, g):
    n, vocab = case["seqs"], case["vocab"]
    logits = torch.randn(n, vocab, dtype=torch.float32, device="cuda", generator=g).mul_(2)
    if not case["flat"]:  # a few likely tokens, as a language model's rows have them
        likely = torch.randint(vocab, (n, 24), device="cuda", generator=g)
        gain = torch.rand(n, 24, device="cuda", generator=g).mul_(8).add_(4)
        logits.scatter_add_(1, likely, gain)
    noise = torch.empty(n, vocab, dtype=torch.float32, device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    temperature, top_k, top_p, min_p = zip(*[_SETTINGS[kind] for kind in _kinds(case)])
    floats = lambda x: torch.tensor(x, dtype=torch.float32, device="cuda")  # noqa: E731
    return {"case": dict(case), "logits": logits.to(_TYPES[case["type"]]), "noise": noise,
            "temperature": floats(temperature), "top_k": _ints(top_k), "top_p": floats(top_p), "min_p": floats(min_p)}


# ---- one pass ---------------------------------------------------------------

def _cache(state):
    import paper_2607_16973_gb300 as tq

    if "cache" not in state:  # the handle that a program keeps
        state["cache"] = tq.KVCache.from_tensors(state["k"], state["v"], state["k_scale"], state["v_scale"],
                                                 state["table"], state["lens"], state["refs"], codes=state["codes"])
    return state["cache"]


def run(state):
    op = state["case"]["op"]
    if op == "cross":
        if own:
            out, lse = _cache(state).cross_attention(0, state["slots"], state["starts"], state["q"], return_lse=True)
        else:
            out, lse = _plain_cross(state)
        return {"out": out, "lse": lse}
    if op == "share":
        return {"plan": _cache(state).share(state["slots"], state["starts"]) if own else _plain_share(state)}
    if op == "shared":
        if own:
            out, lse = _cache(state).shared_attention(0, state["slots"], state["starts"], state["plan"], state["q"],
                                                      groups=state["groups"], return_lse=True)
        else:
            out, lse = _plain_shared(state)
        return {"out": out, "lse": lse}
    if own:
        import paper_2607_16973_gb300 as tq

        tokens, logprobs = tq.sample_tokens(state["logits"], state["noise"], temperature=state["temperature"],
                                            top_k=state["top_k"], top_p=state["top_p"], min_p=state["min_p"],
                                            return_logprobs=True)
    else:
        tokens, logprobs = _plain_sample(state)
    return {"tokens": tokens, "logprobs": logprobs}


# ---- the plain forms --------------------------------------------------------

def _read(state, name, where):
    """Values of the pages `where` [n, width], float32 [n, kv_heads, width * page, dim]."""
    case = state["case"]
    n, width = where.shape
    kv_heads, page, dim = case["kv_heads"], case["page"], case["dim"]
    kind = torch.int8 if state["codes"] == "int8" else torch.float8_e4m3fn
    x = state[name][0][where].view(kind).float().view(n, width, kv_heads, page // _BLOCK, _BLOCK * dim)
    x = x * state[name + "_scale"][0][where][..., None]
    return x.view(n, width, kv_heads, page, dim).transpose(1, 2).reshape(n, kv_heads, width * page, dim)


def _padded_queries(state, first, count, most):
    """Queries first[i] .. first[i] + count[i] - 1, padded to `most`: float32 [n, kv_heads, group * most, dim]."""
    case = state["case"]
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    row = torch.arange(most, device=first.device)
    here = (first[:, None] + torch.minimum(row, (count[:, None] - 1).clamp(min=0))).clamp(max=state["q"].shape[0] - 1)
    q = state["q"][here].float().view(len(first), most, kv_heads, heads // kv_heads, dim).permute(0, 2, 3, 1, 4)
    return q.reshape(len(first), kv_heads, -1, dim)


def _sums(q, k, v, seen, dim):
    """Of rows [n, kv_heads, group * most, dim] over the tokens that `seen` [n, most, tokens] has: the largest score, the
    sum of the weights relative to it, and the weighted sum of the values."""
    n, kv_heads, _, tokens = k.shape[0], k.shape[1], q.shape[2], k.shape[2]
    s = torch.matmul(q, k.transpose(2, 3)) * (1 / math.sqrt(dim))
    s = s.view(n, kv_heads, -1, seen.shape[1], tokens).masked_fill_(~seen[:, None, None], float("-inf"))
    top = s.amax(4, keepdim=True)
    p = torch.exp(s - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    o = torch.matmul(p.view(n, kv_heads, -1, tokens), v).view(*p.shape[:4], dim)
    return top[..., 0], p.sum(4), o


def _by_token(x, most, count):
    """[n, kv_heads, group, most, ...] to the rows of the tokens that are there, [tokens, heads, ...]."""
    n, kv_heads, group = x.shape[:3]
    x = x.movedim(3, 1).reshape(n, most, kv_heads * group, *x.shape[4:])
    return x[(torch.arange(most, device=x.device) < count[:, None]).nonzero(as_tuple=True)]


def _finished(state, top, total, o):
    lse = top + torch.log(total)
    o = o / torch.where(total > 0, total, torch.ones_like(total))[..., None]
    return o.to(state["q"].dtype), lse


def _plain_cross(state):
    case = state["case"]
    slots, starts, most = state["slots"].long(), state["starts"].long(), state["most_new"]
    width, count = -(-state["most"] // case["page"]), starts[1:] - starts[:-1]
    where = state["table"].long()[slots, :width].clamp(min=0)
    token = torch.arange(width * case["page"], device=slots.device)
    seen = (token < state["lens"].long()[slots][:, None])[:, None].expand(-1, most, -1)
    q = _padded_queries(state, starts[:-1], count, most)
    found = _sums(q, _read(state, "k", where), _read(state, "v", where), seen, case["dim"])
    return _finished(state, *[_by_token(x, most, count) for x in found])


def _plain_share(state):
    page, table, slots, starts = state["case"]["page"], state["table"], state["slots"].long(), state["starts"]
    before = state["lens"][slots] - (starts[1:] - starts[:-1])
    held = table[slots]
    place = torch.arange(table.shape[1], device=table.device)
    same = (held[1:] == held[:-1]) & (held[1:] >= 0) & (place * page < torch.minimum(before[1:], before[:-1])[:, None])
    pages = same.to(torch.int32).cumprod(1).sum(1)
    common = torch.minimum(torch.minimum(before[1:], before[:-1]), pages * page)
    n = slots.numel()
    index = torch.arange(n, device=table.device)
    joined = torch.cat([torch.zeros_like(common[:1], dtype=torch.bool), common > 0])  # with the one in front
    first = torch.where(joined, torch.zeros_like(index), index).cummax(0).values
    members = torch.zeros_like(index).index_add_(0, first, torch.ones_like(index))[first]
    most = torch.full_like(index, 2**31 - 1)
    least = most.scatter_reduce(0, first[1:], torch.where(joined[1:], common.long(), most[1:]), "amin")[first]
    tokens = torch.where(members > 1, least, torch.zeros_like(least))
    return torch.stack([first, members, tokens]).to(torch.int32)


def _plain_shared(state):
    """The shared tokens once for each group, with the queries of all its requests; each request's own; joined."""
    case, page = state["case"], state["case"]["page"]
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    slots, starts, most = state["slots"].long(), state["starts"].long(), state["most_new"]
    first, members, shared = state["plan"].long()
    count, lens, table = starts[1:] - starts[:-1], state["lens"].long()[slots], state["table"].long()[slots]
    # each request's own tokens: from the first that is not shared on
    width = -(-state["most_tail"] // page) + 1
    place = shared[:, None] // page + torch.arange(width, device=slots.device)
    where = table.gather(1, place.clamp(max=table.shape[1] - 1)).clamp(min=0)
    token = (shared // page * page)[:, None] + torch.arange(width * page, device=slots.device)
    at = (lens - count)[:, None] + torch.arange(most, device=slots.device)  # place of each query
    seen = (token >= shared[:, None])[:, None] & (token[:, None] <= at[:, :, None])
    q = _padded_queries(state, starts[:-1], count, most)
    top, total, o = [_by_token(x, most, count)
                     for x in _sums(q, _read(state, "k", where), _read(state, "v", where), seen, dim)]
    if state["leads"]:
        lead, size, tokens = (torch.tensor(x, device=slots.device) for x in zip(*state["leads"]))
        width = -(-max(s for *_, s in state["leads"]) // page)
        where = table[lead, :width].clamp(min=0)
        begin, queries = starts[lead], starts[lead + size] - starts[lead]
        wide = max(k for _, k, _ in state["leads"]) * most
        token = torch.arange(width * page, device=slots.device)
        seen = (token < tokens[:, None])[:, None].expand(-1, wide, -1)
        q = _padded_queries(state, begin, queries, wide)
        here = _sums(q, _read(state, "k", where), _read(state, "v", where), seen, dim)
        inside = torch.arange(wide, device=slots.device)
        row = (begin[:, None] + inside)[inside < queries[:, None]]
        more_top, more_total, more_o = (_by_token(x, wide, queries) for x in here)
        peak = torch.maximum(top[row], more_top)
        old, new = torch.exp(top[row] - peak), torch.exp(more_top - peak)
        total[row] = total[row] * old + more_total * new
        o[row] = o[row] * old[..., None] + more_o * new[..., None]
        top[row] = peak
    return _finished(state, top, total, o)


def _plain_sample(state):
    """Sums and quotients in 64 bits: a token next to the border of what is kept, or next to the largest quotient, is on
    the right side of it."""
    x = state["logits"].float()
    n, vocab = x.shape
    order = torch.sort(x, dim=1, descending=True, stable=True)
    top = order.values[:, :1].double()
    sorted_x = order.values.double() - top
    temperature = state["temperature"].double()[:, None]
    hot = temperature > 0
    weight = torch.exp(sorted_x / torch.where(hot, temperature, torch.ones_like(temperature)))
    rank = torch.arange(vocab, device=x.device)
    k = state["top_k"].long()[:, None]
    kept = (rank < torch.where((k > 0) & (k < vocab), k, torch.full_like(k, vocab))) & (hot | (rank == 0))
    weight = weight * kept
    upto = weight.cumsum(1)
    p = state["top_p"].double()[:, None]
    kept &= (p >= 1) | (upto - weight < p * upto[:, -1:]) | (rank == 0)
    kept &= (weight >= state["min_p"].double()[:, None]) | (rank == 0)
    quotient = weight * kept / state["noise"].double().gather(1, order.indices)
    # the lowest token of equals
    best = quotient.amax(1, keepdim=True)
    tokens = torch.where(quotient == best, order.indices, torch.full_like(order.indices, vocab)).amin(1)
    lse = torch.log(torch.exp(sorted_x).sum(1)) + top[:, 0]
    logprobs = x.gather(1, tokens[:, None])[:, 0].double() - lse
    return tokens.to(torch.int32), logprobs.float()


# ---- in 64 bits -------------------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "share":
        return None  # whole numbers
    return _exact_sample(state) if case["op"] == "sample" else _exact_attention(state)


def _exact_attention(state):
    """Request by request, over all that its own table names."""
    case, page = state["case"], state["case"]["page"]
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    group, starts, lens = heads // kv_heads, state["starts"].tolist(), state["lens"].tolist()
    kind = torch.int8 if state["codes"] == "int8" else torch.float8_e4m3fn
    out = torch.zeros(starts[-1], heads, dim, dtype=torch.float64, device="cuda")
    lse = torch.full((starts[-1], heads), -math.inf, dtype=torch.float64, device="cuda")
    for i, slot in enumerate(state["slots"].tolist()):
        length, a, b = lens[slot], starts[i], starts[i + 1]
        pages = state["table"][slot, : -(-length // page)].long()
        for h in range(kv_heads):
            def values(name):
                code = state[name][0, pages, h].view(kind).double().reshape(-1, dim)[:length]
                return code * state[name + "_scale"][0, pages, h].double().reshape(-1).repeat_interleave(_BLOCK)[:length, None]

            mine = slice(h * group, (h + 1) * group)
            q = state["q"][a:b, mine].double().reshape(-1, dim)
            s = q @ values("k").t() / math.sqrt(dim)
            if case["op"] == "shared":
                place = torch.arange(length - (b - a), length, device="cuda").repeat_interleave(group)
                s[torch.arange(length, device="cuda")[None] > place[:, None]] = -math.inf
            lse[a:b, mine] = torch.logsumexp(s, 1).view(b - a, group)
            out[a:b, mine] = (torch.softmax(s, 1) @ values("v")).view(b - a, group, dim)
    return {"out": out, "lse": lse}


def _exact_sample(state):
    """Row by row: the tokens from the likeliest on until a setting ends them, then the winner among them."""
    logprobs = []
    settings = zip(*[state[name].tolist() for name in ("temperature", "top_k", "top_p", "min_p")])
    for row, noise, (temperature, top_k, top_p, min_p) in zip(state["logits"], state["noise"], settings):
        x = row.double()
        order = torch.argsort(x, descending=True, stable=True)
        if temperature > 0:
            held = order[:top_k] if top_k else order
            w = torch.exp((x[held] - x[order[0]]) / temperature)
            keep = max(1, int((w >= min_p).sum()))
            if top_p < 1:
                before = torch.cumsum(w, 0) - w
                keep = min(keep, max(1, int((before < top_p * w.sum()).sum())))
            token = held[torch.argmax(w[:keep] / noise.double()[held[:keep]])]
        else:
            token = order[0]
        logprobs.append(x[token] - torch.logsumexp(x, 0))
    return {"tokens": None, "logprobs": torch.stack(logprobs)}
