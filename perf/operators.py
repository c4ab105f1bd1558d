"""What a generator asks of the 8-bit key-value cache beside the index, as cases that can be timed.

A program that answers from retrieved passages keeps their keys and values as
8-bit codes in pages, with one scale for every 16 tokens and head, and makes
the same few calls in every step of its decoding loop:

* ``append``: quantise the new tokens' keys and values into their pages;
* ``attend``: causal attention of the new tokens over the cache;
* ``pages``: share a passage's pages with the requests that retrieved it and
  give each room for its own tokens (``branch``), or move the pages in use to
  the front of the pool (``compact``);
* ``verify``: accept or reject drafted tokens by the target's probabilities.

Every case has a plain form in float32 (``own = False``), elementary torch
operations on padded batches, beside the calls of the library (``own = True``).
A cache's pages lie in shuffled order, as they do after some time of service.
The lengths of a batch are the same for every seed, in another order.
"""
import math

import torch

own = False

_BLOCK = 16  # tokens that share a scale
_QMAX = {"int8": 127.0, "e4m3": 448.0}
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    def append(name, seqs, new, length, kv_heads=8, heads=32, dim=128, page=64, codes="int8", type="bf16"):
        return {"name": name, "op": "append", "seqs": seqs, "new": new, "length": length, "kv_heads": kv_heads,
                "heads": heads, "dim": dim, "page": page, "codes": codes, "type": type}

    def attend(name, seqs, new, length, heads=32, kv_heads=8, dim=128, page=64, codes="int8", type="bf16", window=0,
               idle=0):
        return {"name": name, "op": "attend", "seqs": seqs, "new": new, "length": length, "heads": heads,
                "kv_heads": kv_heads, "dim": dim, "page": page, "codes": codes, "type": type, "window": window,
                "idle": idle}

    def pages(name, kind, seqs, length, pool, layers, share=4, new=1, kv_heads=8, dim=128, page=64):
        return {"name": name, "op": "pages", "kind": kind, "seqs": seqs, "length": length, "pool": pool,
                "layers": layers, "share": share, "new": new, "kv_heads": kv_heads, "dim": dim, "page": page}

    def verify(name, seqs, drafts, vocab, type="fp32", text=False):
        return {"name": name, "op": "verify", "seqs": seqs, "drafts": drafts, "vocab": vocab, "type": type,
                "text": text}

    return [
        # one decoding step of a busy server: a token for each of 64 sequences
        append("append-step", 64, 1, 4000),
        # the prompts of a few requests with their passages, of different lengths
        append("append-prompts", 5, 5000, 0, codes="e4m3", type="fp16"),
        # one interactive request with a short prompt: latency
        attend("attend-one", 1, 1, 1031),
        # a decoding step of a server, lengths from a few hundred tokens on, some slots of the batch idle
        attend("attend-batch", 128, 1, 4096, codes="e4m3", idle=6),
        # one request over a long collection of passages
        attend("attend-long", 1, 1, 200_001, heads=64),
        # drafted tokens of a batch scored at once, an odd group, a narrow head, a sliding window
        attend("attend-drafts", 24, 5, 8190, heads=40, dim=64, type="fp16", window=4096),
        # the second half of two long prompts
        attend("attend-prompt", 2, 2048, 6000, codes="e4m3"),
        # four passages forked to sixteen requests, each given room for one token
        pages("branch-16", "branch", 16, 700, 1024, 2),
        # a burst: 256 requests over 8 long contexts, each with the tokens of its question
        pages("branch-256", "branch", 256, 16_000, 8192, 4, share=32, new=40),
        # a pool of 4 GB, a third of it in use, packed to the front before its end is given back
        pages("compact-4gb", "compact", 70, 2000, 4096, 8, share=1),
        # a passage's own words as drafts of a few sequences
        verify("verify-text", 4, 6, 32_000, text=True),
        # a batch with a small model's drafts
        verify("verify-batch", 256, 7, 128_000, type="bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "pages", "verify"])
    kv_heads, dim, page = rng.choice([1, 2, 4, 8, 8]), rng.choice([64, 128, 128, 128, 256]), rng.choice([16, 32, 64, 64, 128])
    codes, type_ = rng.choice(["int8", "e4m3"]), rng.choice(["bf16", "bf16", "fp16"])
    group = rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
    if op == "append":
        seqs = _log_uniform(rng, 1, 256)
        new = 1 if rng.random() < 0.5 else _log_uniform(rng, 2, max(3, 12_000 // seqs))
        return {"op": op, "seqs": seqs, "new": new, "length": rng.choice([0, _log_uniform(rng, 1, 8000 // (1 + seqs // 16))]),
                "kv_heads": kv_heads, "heads": kv_heads * group, "dim": dim, "page": page, "codes": codes,
                "type": rng.choice(["bf16", "bf16", "fp16", "fp32"])}
    if op == "attend":
        case = {"op": op, "heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim, "page": page, "codes": codes,
                "type": type_}
        if rng.random() < 0.3:  # (part of) a prompt
            new, seqs = _log_uniform(rng, 17, 2048), rng.choice([1, 1, 2, 3])
            if new * case["heads"] > 65_536:
                case["heads"] = kv_heads * max(1, 65_536 // (new * kv_heads))
            length = _log_uniform(rng, new, max(new + 1, 7000 // seqs))
        else:
            new, seqs = rng.choice([1, 1, 1, 2, 4, 5, 8]), _log_uniform(rng, 1, 160)
            length = _log_uniform(rng, 20, min(200_000, 3_000_000 // (seqs * kv_heads * dim // 64)))
        return {**case, "seqs": seqs, "new": new, "length": max(new, length),
                "window": rng.choice([0, 0, 0, _log_uniform(rng, 16, 8192)]), "idle": seqs // 20}
    if op == "pages":
        kind = rng.choice(["branch", "branch", "compact"])
        seqs = _log_uniform(rng, 2, 256)
        share = rng.choice([1, 2, 4, 16])
        length = _log_uniform(rng, 20, 16_000)
        layers = rng.choice([1, 2, 4])
        most = min(16_384, 6_000_000_000 // (layers * 2 * kv_heads * page * dim))
        length = min(length, page * (most // 3) // (1 + seqs // share))
        new = rng.choice([1, 1, 9, 33])
        need = (1 + seqs // share) * (1 + length // page) + seqs * (2 + new // page)
        if kind == "compact":
            need = min(most, need * rng.randint(1, 3))
        return {"op": op, "kind": kind, "seqs": seqs, "length": max(20, length), "pool": need + rng.randrange(64, 1024),
                "layers": layers, "share": share, "new": new, "kv_heads": kv_heads, "dim": dim, "page": page}
    seqs, vocab = _log_uniform(rng, 1, 256), _log_uniform(rng, 1000, 130_000)
    return {"op": op, "seqs": seqs, "drafts": rng.randint(1, min(7, max(1, 250_000_000 // (seqs * vocab)))), "vocab": vocab,
            "type": rng.choice(["fp32", "bf16", "fp16"]), "text": rng.random() < 0.4}


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


def _lengths(case):
    """(tokens that a sequence holds with its new ones, its new ones), in the order of _new_counts."""
    counts = _new_counts(case)
    if case["op"] == "append":
        held = _spread(case["seqs"], case["length"], 0) if case["length"] else [0] * case["seqs"]
        return [(h + c, c) for h, c in zip(held, counts)]
    held = _spread(case["seqs"], case["length"], 0)
    both = [(max(h, c), c) for h, c in zip(held, counts)]
    return [(0, c) if i < case["idle"] else (h, c) for i, (h, c) in enumerate(both)]


def _seen(length, i, window):
    """Tokens that a query at place i sees."""
    return 0 if i < 0 else min(i + 1, window) if window else i + 1


def work(case):
    op = case["op"]
    if op == "verify":  # the target's row and the noise of the place that is drawn, and the drafting model's after a rejection
        size = {"fp32": 4, "bf16": 2, "fp16": 2}[case["type"]]
        row = case["vocab"] * (size + 4 + (0 if case["text"] else 0.8 * size))
        return {"bytes": case["seqs"] * row, "flops": 0}
    heads, dim = case["kv_heads"], case["dim"]
    block = heads * (_BLOCK * dim + 4)  # codes and scales of a block, keys or values
    if op == "append":
        size = 4 if case["type"] == "fp32" else 2
        total = 0
        for length, new in _lengths(case):
            first = length - new
            part = first % _BLOCK
            total += 2 * new * heads * dim * (size + 1) + 2 * heads * 4 * ((length - 1) // _BLOCK - first // _BLOCK + 1)
            total += 2 * heads * dim * part  # codes that may have to take a larger scale: read
        return {"bytes": total, "flops": 0}
    if op == "attend":
        size, pairs, read = 2, 0, 0
        for length, new in _lengths(case):
            seen = [_seen(length, length - new + i, case["window"]) for i in range(new)]
            pairs += sum(seen)
            start = max(0, length - new - case["window"] + 1) if case["window"] else 0
            read += 2 * block * (-(-length // _BLOCK) - start // _BLOCK) if length else 0
            read += new * case["heads"] * (2 * size * dim + 4)
        return {"bytes": read, "flops": 4 * dim * case["heads"] * pairs}
    used = _page_lengths(case)
    if case["kind"] == "branch":  # tables, counts, and the part of a page that each request takes for itself
        total = 0
        for parent, children in used:
            total += children * (3 * 4 * -(-parent // case["page"]))
            total += children * 2 * 2 * case["layers"] * block * -(-(parent % case["page"]) // _BLOCK)
        return {"bytes": total, "flops": 0}
    live = sum(-(-n // case["page"]) for n, _ in used)
    moved = live * (1 - live / case["pool"])  # pages of a shuffled pool that lie behind its first `live`
    return {"bytes": 2 * moved * 2 * case["layers"] * block * (case["page"] // _BLOCK), "flops": 0}


def _page_lengths(case):
    """(length, requests that share it) of each cached context."""
    n = max(1, case["seqs"] // case["share"])
    lengths = _spread(n, case["length"], 1)
    return [(length, case["seqs"] // n + (i < case["seqs"] % n)) for i, length in enumerate(lengths)]


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


def _pool(case, pages, layers, codes, g):
    shape = (layers, pages, case["kv_heads"], case["page"], case["dim"])
    scales = (layers, pages, case["kv_heads"], case["page"] // _BLOCK)
    return {"k": _codes(shape, codes, g), "v": _codes(shape, codes, g), "k_scale": _scales(scales, codes, g),
            "v_scale": _scales(scales, codes, g), "codes": codes}


def _tables(lengths, page, pages, slots, width, g):
    """Tables of sequences in the given slots over pages in shuffled order: (table, lens, refs)."""
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((slots, width), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(slots, dtype=torch.int32, device="cuda")
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    at = 0
    for slot, length in lengths:
        n = -(-length // page)
        table[slot, :n] = order[at: at + n]
        lens[slot] = length
        at += n
    refs[order[:at].long()] = 1
    return table, lens, refs


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op == "verify":
        return _prepare_verify(case, g)
    if op == "pages":
        return _prepare_pages(case, g)
    shuffle = torch.randperm(case["seqs"], device="cuda", generator=g).tolist()
    both = [_lengths(case)[i] for i in shuffle]
    page = case["page"]
    slots = case["seqs"] + 3
    slot = torch.randperm(slots, device="cuda", generator=g)[: case["seqs"]].tolist()
    need = sum(-(-length // page) for length, _ in both)
    pages = need + 5
    width = max(-(-length // page) for length, _ in both) + 2
    table, lens, refs = _tables([(s, length) for s, (length, _) in zip(slot, both)], page, pages, slots, width, g)
    starts = [0]
    for _, new in both:
        starts.append(starts[-1] + new)
    total = starts[-1]
    state = {"case": dict(case), **_pool(case, pages, 1, case["codes"], g), "table": table, "lens": lens, "refs": refs,
             "slots": _ints(slot), "starts": _ints(starts), "most_new": max(new for _, new in both),
             "most": max(max(length for length, _ in both), 1)}
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    dtype = _TYPES[case["type"]]
    # queries, keys and values as one projection gives them: a row of them all for each token
    rows = torch.randn(total, heads + 2 * kv_heads, dim, dtype=torch.float32, device="cuda", generator=g).to(dtype)
    if op == "append":
        # a few channels of the keys are much larger than the others
        rows[:, heads: heads + kv_heads, :: dim // 4] *= 4
        state["new_k"], state["new_v"] = rows[:, heads: heads + kv_heads], rows[:, heads + kv_heads:]
    else:
        state["q"] = rows[:, :heads] * 2
    return state


def _prepare_pages(case, g):
    used = _page_lengths(case)
    page, pool = case["page"], case["pool"]
    parents = len(used)
    width = -(-(max(n for n, _ in used) + case["new"]) // page) + 1
    if case["kind"] == "branch":
        slots = parents + case["seqs"]
        table, lens, refs = _tables([(i, n) for i, (n, _) in enumerate(used)], page, pool, slots, width, g)
        source = [i for i, (_, children) in enumerate(used) for _ in range(children)]
        child = (torch.randperm(case["seqs"], device="cuda", generator=g) + parents).to(torch.int32)
        more = {"source": _ints(source), "child": child, "counts": _ints([case["new"]] * case["seqs"])}
    else:
        table, lens, refs = _tables([(i, n) for i, (n, _) in enumerate(used)], page, pool, parents, width, g)
        # the requests that share the first context hold its pages too
        refs[table[0, : -(-used[0][0] // page)].long()] += 1
        table = torch.cat([table, table[:1]])
        lens = torch.cat([lens, lens[:1]])
        more = {"table0": table.clone(), "refs0": refs.clone()}
    return {"case": dict(case), **_pool(case, pool, case["layers"], "int8", g), "table": table, "lens": lens, "refs": refs,
            **more}


def _prepare_verify(case, g):
    n, t, vocab, dtype = case["seqs"], case["drafts"], case["vocab"], _TYPES[case["type"]]
    top = torch.randint(vocab, (n, t + 1, 1), device="cuda", generator=g)
    logits = torch.randn(n, t + 1, vocab, dtype=torch.float32, device="cuda", generator=g).mul_(2)
    gain = math.log(vocab) + 2  # the likeliest token gets about three quarters of the target's mass
    here = logits.scatter_add(2, top, torch.full_like(top, 1, dtype=torch.float32).mul_(gain + 1.1))
    target = torch.softmax(here, dim=2).to(dtype)
    noise = torch.empty(n, vocab, dtype=torch.float32, device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    state = {"case": dict(case), "target": target, "noise": noise, "draft": None,
             "uniforms": torch.rand(n, t, device="cuda", generator=g),
             "lens": torch.randint(max(1, t - 2), t + 1, (n,), device="cuda", generator=g).to(torch.int32)}
    if case["text"]:
        state["drafts"] = top[:, :t, 0].to(torch.int32).contiguous()
        return state
    logits = logits[:, :t] + 0.7 * torch.randn(n, t, vocab, dtype=torch.float32, device="cuda", generator=g)
    logits.scatter_add_(2, top[:, :t], torch.full_like(top[:, :t], 1, dtype=torch.float32).mul_(gain + 1.5))
    draft = torch.softmax(logits, dim=2).to(dtype)
    race = torch.empty(n, t, vocab, dtype=torch.float32, device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    state["draft"], state["drafts"] = draft, (draft.float() / race).argmax(2).to(torch.int32)
    return state


# ---- one pass ---------------------------------------------------------------

def _cache(state):
    import paper_2607_16973_gb300 as tq

    if "cache" not in state:  # the handle that a program keeps
        state["cache"] = tq.KVCache.from_tensors(state["k"], state["v"], state["k_scale"], state["v_scale"],
                                                 state["table"], state["lens"], state["refs"], codes=state["codes"])
    return state["cache"]


def run(state):
    op = state["case"]["op"]
    if op == "append":
        if own:
            _cache(state).append(0, state["slots"], state["starts"], state["new_k"], state["new_v"])
        else:
            _plain_append(state, state["k"][0], state["k_scale"][0], state["new_k"])
            _plain_append(state, state["v"][0], state["v_scale"][0], state["new_v"])
        kind = torch.float8_e4m3fn if state["codes"] == "e4m3" else torch.int8
        return {"k": state["k"].view(kind), "v": state["v"].view(kind), "k_scale": state["k_scale"],
                "v_scale": state["v_scale"]}
    if op == "attend":
        if own:
            out, lse = _cache(state).attention(0, state["slots"], state["starts"], state["q"],
                                               window=state["case"]["window"], return_lse=True)
        else:
            out, lse = _plain_attention(state)
        return {"out": out, "lse": lse}
    if op == "verify":
        if own:
            import paper_2607_16973_gb300 as tq

            tokens, accepted = tq.verify_drafts(state["target"], state["drafts"], state["uniforms"], state["noise"],
                                                draft_probs=state["draft"], draft_lens=state["lens"])
        else:
            tokens, accepted = _plain_verify(state)
        return {"tokens": tokens, "accepted": accepted}
    if state["case"]["kind"] == "branch":
        if own:
            cache = _cache(state)
            cache.fork(state["child"], state["source"])
            cache.extend(state["child"], state["counts"])
        else:
            _plain_fork(state)
            _plain_extend(state)
    else:  # a pool that has become sparse again
        state["table"].copy_(state["table0"])
        state["refs"].copy_(state["refs0"])
        if own:
            _cache(state).compact()
        else:
            _plain_compact(state)
    return {name: state[name] for name in ("table", "lens", "refs", "k", "v", "k_scale", "v_scale")}


# ---- the plain forms --------------------------------------------------------

def _values(raw, codes):
    return raw.view(torch.int8 if codes == "int8" else torch.float8_e4m3fn).float()


def _round(y, codes):
    """float32 values in the codes' range to codes."""
    y = torch.nan_to_num(y.clamp(-_QMAX[codes], _QMAX[codes]), nan=0.0)
    return y.round().to(torch.int8).view(torch.uint8) if codes == "int8" else y.to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_append(state, pool, scale, new):
    codes, page = state["codes"], state["case"]["page"]
    per_page = page // _BLOCK
    starts, slots = state["starts"].long(), state["slots"].long()
    total = new.shape[0]
    token = torch.arange(total, device=new.device)
    seq = torch.searchsorted(starts, token, right=True) - 1
    first = state["lens"].long()[slots] - (starts[1:] - starts[:-1])  # tokens held before
    place = first[seq] + token - starts[seq]
    where = state["table"].long()[slots[seq], place // page]  # the page of each new token
    block = where * per_page + place % page // _BLOCK
    heads = scale.shape[1]
    flat = scale.permute(0, 2, 1).reshape(-1, heads)  # [pages * blocks, heads]
    x = new.float()
    size = torch.where(x.isfinite(), x.abs(), torch.zeros_like(x)).amax(2)
    largest = torch.zeros_like(flat).scatter_reduce_(0, block[:, None].expand(-1, heads), size, "amax")
    fresh = largest / torch.full((), _QMAX[codes], device=new.device)
    # the block that was part full: its codes take the larger of the two scales
    part = first % _BLOCK
    half = state["table"].long()[slots, (first // page).clamp(max=state["table"].shape[1] - 1)].clamp(min=0)
    some = (part > 0)[:, None] & (starts[1:] > starts[:-1])[:, None]
    old_block = half * per_page + first % page // _BLOCK
    old = torch.where(some, flat[old_block], torch.zeros_like(flat[old_block]))
    now = torch.maximum(old, fresh[old_block])
    ratio = torch.where(now > old, old / now, torch.ones_like(old))
    lines = pool.view(-1, heads, per_page, _BLOCK, pool.shape[3])
    held = lines[half, :, first % page // _BLOCK]  # [seqs, heads, 16, dim]
    again = _round(_values(held, codes) * ratio[:, :, None, None], codes)
    keep = torch.arange(_BLOCK, device=new.device)[None, :] < part[:, None]
    keep = (keep[:, None, :] & some[:, :, None]).expand(held.shape[:3])
    at = keep.nonzero(as_tuple=True)
    lines[half[at[0]], at[1], (first % page // _BLOCK)[at[0]], at[2]] = again[at]
    fresh = fresh.scatter_reduce(0, old_block[:, None].expand(-1, heads), old, "amax")
    used = fresh[block]  # [tokens, heads]
    y = torch.where(used[:, :, None] > 0, x / used[:, :, None], torch.zeros_like(x))
    lines[where, :, place % page // _BLOCK, place % _BLOCK] = _round(y, codes)
    scale[where, :, place % page // _BLOCK] = used


def _plain_attention(state):
    case, codes, page = state["case"], state["codes"], state["case"]["page"]
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    slots, starts = state["slots"].long(), state["starts"].long()
    n, most_new, width = slots.numel(), state["most_new"], -(-state["most"] // page)
    where = state["table"].long()[slots, :width].clamp(min=0)

    def read(pool, scale):
        x = _values(pool[where], codes).view(n, width, kv_heads, page // _BLOCK, _BLOCK * dim)
        x = x * scale[where][..., None]
        return x.view(n, width, kv_heads, page, dim).transpose(1, 2).reshape(n, kv_heads, width * page, dim)

    counts = starts[1:] - starts[:-1]
    row = torch.arange(most_new, device=slots.device)
    here = (starts[:-1, None] + row).clamp(max=state["q"].shape[0] - 1)
    q = state["q"][here].float().view(n, most_new, kv_heads, heads // kv_heads, dim).permute(0, 2, 3, 1, 4)
    q = q.reshape(n, kv_heads, -1, dim)
    s = torch.matmul(q, read(state["k"][0], state["k_scale"][0]).transpose(2, 3)) * (1 / math.sqrt(dim))
    s = s.view(n, kv_heads, heads // kv_heads, most_new, width * page)
    lens = state["lens"].long()[slots]
    at = (lens - counts)[:, None] + row  # place of each row
    token = torch.arange(width * page, device=slots.device)
    seen = token <= at[:, :, None]
    if case["window"]:
        seen &= token > at[:, :, None] - case["window"]
    s = s.masked_fill(~seen[:, None, None], float("-inf"))
    top = s.amax(4, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    p = torch.exp(s - top)
    total = p.sum(4, keepdim=True)
    v = read(state["v"][0], state["v_scale"][0])
    o = torch.matmul(p.view(n, kv_heads, -1, width * page), v).view(n, kv_heads, heads // kv_heads, most_new, dim)
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + torch.log(total))[..., 0]
    real = (row < counts[:, None]).nonzero(as_tuple=True)
    o = o.permute(0, 3, 1, 2, 4).reshape(n, most_new, heads, dim)[real]
    return o.to(state["q"].dtype), lse.permute(0, 3, 1, 2).reshape(n, most_new, heads)[real]


def _plain_fork(state):
    table, lens, refs = state["table"], state["lens"], state["refs"]
    child, source = state["child"].long(), state["source"].long()
    page = state["case"]["page"]
    place = torch.arange(table.shape[1], device=table.device)
    old, new = table[child], table[source]
    held = place < -(-lens[child] // page)[:, None]
    refs.index_add_(0, old[held].long(), torch.full_like(old[held], -1))
    given = place < -(-lens[source] // page)[:, None]
    refs.index_add_(0, new[given].long(), torch.ones_like(new[given]))
    table[child] = torch.where(given, new, torch.where(held, torch.full_like(old, -1), old))
    lens[child] = lens[source]


def _plain_extend(state):
    table, lens, refs, page = state["table"], state["lens"], state["refs"], state["case"]["page"]
    slots, counts = state["child"].long(), state["counts"]
    held, after = -(-lens[slots] // page), -(-(lens[slots] + counts) // page)
    last = table[slots, (held - 1).clamp(min=0).long()].long().clamp(min=0)
    # a part-full page that others hold too is taken along as a copy
    copied = (counts > 0) & (lens[slots] % page > 0) & (refs[last] > 1)
    first = held - copied.int()
    wanted = (after - first).long()
    free = (refs == 0).nonzero()[:, 0][: int(wanted.sum())].to(torch.int32)
    before = torch.cumsum(wanted, 0) - wanted
    place = torch.arange(table.shape[1], device=table.device)
    here = (place >= first[:, None]) & (place < after[:, None])
    index = before[:, None] + place - first[:, None]
    table[slots] = torch.where(here, free[index.clamp(0, max(free.numel() - 1, 0))], table[slots])
    refs[free.long()] = 1
    refs.index_add_(0, last[copied], torch.full_like(last[copied], -1, dtype=torch.int32))
    to = table[slots, (held - 1).clamp(min=0).long()].long()
    blocks = -(-(lens[slots] % page) // _BLOCK)
    block = torch.arange(page // _BLOCK, device=table.device)
    some = (copied[:, None] & (block < blocks[:, None])).nonzero(as_tuple=True)
    for name in ("k", "v", "k_scale", "v_scale"):
        x = state[name]
        x = x.view(*x.shape[:3], page // _BLOCK, -1)
        x[:, to[some[0]], :, some[1]] = x[:, last[some[0]], :, some[1]]
    lens[slots] += counts


def _plain_compact(state):
    table, refs = state["table"], state["refs"]
    used = refs > 0
    live = int(used.sum())
    place = torch.arange(refs.numel(), device=refs.device)
    old, new = (used & (place >= live)).nonzero()[:, 0], (~used & (place < live)).nonzero()[:, 0]
    for name in ("k", "v", "k_scale", "v_scale"):
        state[name][:, new] = state[name][:, old]
    name = place.to(torch.int32)
    name[old] = new.to(torch.int32)
    refs[new] = refs[old]
    refs[old] = 0
    table.copy_(torch.where(table >= 0, name[table.long().clamp(min=0)], table))


def _plain_verify(state):
    target, drafts, noise, draft = state["target"], state["drafts"].long(), state["noise"], state["draft"]
    n, t = drafts.shape
    p = target[:, :t].gather(2, drafts[:, :, None])[..., 0].float()
    q = torch.ones_like(p) if draft is None else draft.gather(2, drafts[:, :, None])[..., 0].float()
    place = torch.arange(t + 1, device=p.device)
    lens = state["lens"].long()[:, None]
    good = (state["uniforms"] * q < p) & (place[:t] < lens)
    accepted = good.to(torch.int64).cumprod(1).sum(1)
    row = target[torch.arange(n, device=p.device), accepted].float()
    last = accepted.clamp(max=t - 1)
    if draft is None:
        rest = row.scatter(1, drafts.gather(1, last[:, None]), 0.0)
    else:
        rest = (row - draft[torch.arange(n, device=p.device), last].float()).clamp(min=0)
    rest = torch.where((rest > 0).any(1, keepdim=True), rest, row)
    weight = torch.where((accepted < lens[:, 0])[:, None], rest, row)
    token = (weight / noise).argmax(1)
    padded = torch.cat([drafts, torch.zeros_like(drafts[:, :1])], 1)
    tokens = torch.where(place < accepted[:, None], padded, torch.full_like(padded, -1))
    tokens = torch.where(place == accepted[:, None], token[:, None], tokens)
    return tokens.to(torch.int32), accepted.to(torch.int32)


# ---- in 64 bits -------------------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "verify":
        return None  # tokens and counts: whole numbers
    return {"append": _exact_append, "attend": _exact_attention, "pages": _exact_pages}[case["op"]](state)


def _decoded(state, name, slot, length):
    """Tokens 0 .. length - 1 of one slot, float64 [length, heads, dim]."""
    page = state["case"]["page"]
    pages = state["table"][slot, : -(-length // page)].tolist()
    raw = torch.cat([state[name][0, p].transpose(0, 1) for p in pages])[:length]
    scale = torch.cat([state[name + "_scale"][0, p].t().repeat_interleave(_BLOCK, 0) for p in pages])[:length]
    kind = torch.int8 if state["codes"] == "int8" else torch.float8_e4m3fn
    return raw.view(kind).double() * scale.double()[:, :, None]


def _exact_attention(state):
    case = state["case"]
    group, scale = case["heads"] // case["kv_heads"], 1 / math.sqrt(case["dim"])
    starts, outs, lses = state["starts"].tolist(), [], []
    for i, slot in enumerate(state["slots"].tolist()):
        q = state["q"][starts[i]: starts[i + 1]].double()
        new, length = q.shape[0], int(state["lens"][slot])
        out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
        if length:
            k, v = _decoded(state, "k", slot, length), _decoded(state, "v", slot, length)
            at = torch.arange(length - new, length, device=q.device)[:, None]
            token = torch.arange(length, device=q.device)[None]
            hidden = token > at
            if case["window"]:
                hidden |= at - token >= case["window"]
            empty = hidden.all(1)
            for h in range(case["heads"]):
                s = (q[:, h] @ k[:, h // group].t() * scale).masked_fill(hidden, -math.inf)
                lse[:, h] = torch.logsumexp(s, 1)
                p = torch.softmax(s, 1)
                p[empty] = 0
                out[:, h] = p @ v[:, h // group]
        outs.append(out)
        lses.append(lse)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _exact_append(state):
    """Scales, and for e4m3 codes their values; the codes of int8 are whole numbers."""
    case, page, codes = state["case"], state["case"]["page"], state["codes"]
    result = {}
    for name in ("k", "v"):
        scale = state[name + "_scale"].double()
        value = state[name].view(torch.float8_e4m3fn).double() if codes == "e4m3" else None
        starts, lens = state["starts"].tolist(), state["lens"].tolist()
        for i, slot in enumerate(state["slots"].tolist()):
            x = state["new_" + name][starts[i]: starts[i + 1]].double()
            begin, pages = lens[slot] - x.shape[0], state["table"][slot].tolist()
            at = begin
            while at < lens[slot]:
                end = min(lens[slot], at // _BLOCK * _BLOCK + _BLOCK)
                p, b, first = pages[at // page], at % page // _BLOCK, at % _BLOCK
                new = x[at - begin: end - begin]
                s = new.abs().amax((0, 2)) / _QMAX[codes]
                if first:
                    s = torch.maximum(s, scale[0, p, :, b])
                if value is not None:
                    line = slice(b * _BLOCK, b * _BLOCK + first)
                    held = value[0, p, :, line] * (scale[0, p, :, b] / s)[:, None, None]
                    value[0, p, :, line] = held.float().to(torch.float8_e4m3fn).double()
                    y = (new / s[None, :, None]).transpose(0, 1)
                    value[0, p, :, at % page: at % page + end - at] = y.float().to(torch.float8_e4m3fn).double()
                scale[0, p, :, b] = s
                at = end
        result[name + "_scale"] = scale
        result[name] = value
    return result


def _exact_pages(state):
    """The scales' places after the moves, page by page."""
    case, page = state["case"], state["case"]["page"]
    refs = state["refs"].tolist()
    scales = {name: state[name].double() for name in ("k_scale", "v_scale")}
    if case["kind"] == "branch":
        lens = state["lens"].tolist()
        free, moves = [p for p, r in enumerate(refs) if r == 0], []
        sources, holders = state["source"].tolist(), {}
        for s in sources:
            holders[s] = holders.get(s, 0) + 1
        for s in sources:
            n, fill = lens[s], lens[s] % page
            if fill:
                moves.append((int(state["table"][s, n // page]), free.pop(0), -(-fill // _BLOCK)))
            free = free[(n + case["new"] + page - 1) // page - (n + page - 1) // page:]
        for x in scales.values():
            for old, new, blocks in moves:
                x[:, new, :, :blocks] = x[:, old, :, :blocks]
    else:
        live = [p for p, r in enumerate(refs) if r > 0]
        holes = [p for p, r in enumerate(refs) if r == 0 and p < len(live)]
        tail = [p for p in live if p >= len(live)]
        for x in scales.values():
            for old, new in zip(tail, holes):
                x[:, new] = x[:, old]
    return {"table": None, "lens": None, "refs": None, "k": None, "v": None, **scales}
