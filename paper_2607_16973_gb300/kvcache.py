"""The 8-bit key-value cache of the generator behind the index, the verification
of its drafts and the sampling of its tokens: tq_kv_*, tq_verify_drafts and
tq_sample of include/tq.h.

A retrieved passage is prompted once, its keys and values stay in pages of
8-bit codes (one scale for every 16 tokens and head), and each request that
retrieves it forks those pages.  One decoding step of a batch is

    cache.extend(slots, counts)                        # room for the new tokens
    for layer in ...:
        cache.append(layer, slots, starts, k, v)       # their keys and values
        o = cache.attention(layer, slots, starts, q)   # causal, over all that is held
    tokens, accepted = tq.verify_drafts(...)           # where some were drafts
    cache.truncate(slots, lens)                        # rejected ones go

Where requests of a batch were forked from one passage and stand side by side,

    plan = cache.share(slots, starts)                                # once a step
    o = cache.shared_attention(layer, slots, starts, plan, q, groups)

reads what they share once for all of them; `cross_attention` lets queries from
elsewhere see all that a slot holds; `sample_tokens` draws from logits.

All that with slots, counts and lengths on the device: nothing in it waits for the host,
and the same calls can be captured into a CUDA graph.  `check()` reports what a
call could not carry out.
"""
from __future__ import annotations

import ctypes as C
import functools

from . import _dev_ptr, _on_stream, _stream_handle, _torch, _used_on
from ._lib import KV_CODES, KvCacheStruct, check, load

BLOCK = 16  # tokens that share a scale
INT_MAX = 2**31 - 1  # (a wider window hides no more; ctypes would take its low 32 bits)

# A decoding step makes these calls once per layer on a few tokens, and their
# host side is then what it waits for: the checks below take the short way where
# everything is in order and leave it to _dev_ptr to say what is not.


@functools.lru_cache(maxsize=1)
def _types():
    torch = _torch()
    return {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


def _ptr(t, name: str, dtype) -> int:
    if t.dtype is dtype and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    return _dev_ptr(t, name, dtype)


@functools.lru_cache(maxsize=1)
def _current_raw_stream():
    """Handle of the current stream: without the Stream object that
    torch.cuda.current_stream makes, where torch offers that."""
    c = _torch()._C
    raw, device = getattr(c, "_cuda_getCurrentRawStream", None), getattr(c, "_cuda_getDevice", None)
    return (lambda: raw(device())) if raw and device else (lambda: _stream_handle(None))


def _stream(stream) -> int:
    return _current_raw_stream()() if stream is None else int(stream.cuda_stream)


def _empty(shape, dtype, device, stream):
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with _on_stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _used(stream, *tensors) -> None:
    if stream is not None:
        for t in tensors:
            _used_on(t, stream)


def _rows(t, name: str, heads: int, dim: int, types):
    """Rows [tokens, heads, dim] with any strides but the last: (pointer, type,
    token stride, head stride, tokens)."""
    kind = types.get(t.dtype)
    if kind is None or not t.is_cuda:
        _dev_ptr(t, name, tuple(types), contiguous=False)
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        raise ValueError(f"{name} must be [tokens, {heads}, {dim}], got {tuple(shape)}")
    s0, s1, s2 = t.stride()
    if s2 != 1 and t.numel():
        raise ValueError(f"{name}: the elements of a row must lie side by side")
    return t.data_ptr(), kind, s0, s1, shape[0]


def _checked(c):
    """Reference to a cache's struct; raises TQError where the calls would refuse it."""
    check(load().tq_kv_compact_workspace(C.byref(c), C.byref(C.c_size_t())))
    return C.byref(c)


class KVCache:
    """Keys and values of sequences in slots, as 8-bit codes in pages.

    pages, slots, max_pages (pages of one slot's table), page_tokens (a power of
    two from 16 to 256), layers, kv_heads, head_dim (64, 128 or 256); codes:
    "int8" or "e4m3".  The tensors are attributes: k, v (uint8), k_scale,
    v_scale, table, lens, refs, status; `from_tensors` makes a cache of given
    ones.  Work on a cache belongs on one stream at a time, except that
    attention only reads it."""

    def __init__(self, pages: int, slots: int, max_pages: int, kv_heads: int, head_dim: int, page_tokens: int = 64,
                 layers: int = 1, codes: str = "int8", device="cuda"):
        torch = _torch()
        if min(pages, slots, max_pages, kv_heads, head_dim, page_tokens // BLOCK, layers) < 1:
            raise ValueError("pages, slots, max_pages, kv_heads, head_dim and layers must be positive, "
                             "page_tokens at least 16")
        if codes not in KV_CODES:
            raise ValueError(f"codes must be one of {sorted(KV_CODES)}, got {codes!r}")
        # the library's own checks of the sizes, before any memory is taken (addresses that nothing is read from)
        _checked(KvCacheStruct(*[BLOCK] * 8, pages, slots, max_pages, layers, kv_heads, head_dim, page_tokens,
                               KV_CODES[codes]))
        shape = (layers, pages, kv_heads, page_tokens, head_dim)
        scales = (layers, pages, kv_heads, page_tokens // BLOCK)
        i32 = torch.int32
        self._set(torch.zeros(shape, dtype=torch.uint8, device=device),
                  torch.zeros(shape, dtype=torch.uint8, device=device), torch.zeros(scales, device=device),
                  torch.zeros(scales, device=device), torch.full((slots, max_pages), -1, dtype=i32, device=device),
                  torch.zeros(slots, dtype=i32, device=device), torch.zeros(pages, dtype=i32, device=device), codes)

    @classmethod
    def from_tensors(cls, k, v, k_scale, v_scale, table, lens, refs, codes: str = "int8") -> "KVCache":
        """A cache of tensors that the caller keeps (not copied): k, v uint8
        [layers, pages, kv_heads, page_tokens, head_dim], scales float32
        [layers, pages, kv_heads, page_tokens / 16], table int32 [slots,
        max_pages], lens int32 [slots], refs int32 [pages]."""
        self = cls.__new__(cls)
        self._set(k, v, k_scale, v_scale, table, lens, refs, codes)
        return self

    def _set(self, k, v, k_scale, v_scale, table, lens, refs, codes):
        torch = _torch()
        if codes not in KV_CODES:
            raise ValueError(f"codes must be one of {sorted(KV_CODES)}, got {codes!r}")
        if k.dim() != 5 or k.shape != v.shape:
            raise ValueError("k and v must both be [layers, pages, kv_heads, page_tokens, head_dim]")
        layers, pages, kv_heads, page_tokens, head_dim = k.shape
        scales = (layers, pages, kv_heads, page_tokens // BLOCK)
        if tuple(k_scale.shape) != scales or tuple(v_scale.shape) != scales:
            raise ValueError(f"k_scale and v_scale must be {scales}")
        if table.dim() != 2 or lens.shape != (table.shape[0],) or refs.shape != (pages,):
            raise ValueError("table must be [slots, max_pages], lens [slots], refs [pages]")
        u8, f32, i32 = torch.uint8, torch.float32, torch.int32
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.table, self.lens, self.refs, self.codes = table, lens, refs, codes
        self.status = torch.zeros(1, dtype=i32, device=k.device)
        self._c = KvCacheStruct(
            _dev_ptr(k, "k", u8), _dev_ptr(v, "v", u8), _dev_ptr(k_scale, "k_scale", f32),
            _dev_ptr(v_scale, "v_scale", f32), _dev_ptr(table, "table", i32), _dev_ptr(lens, "lens", i32),
            _dev_ptr(refs, "refs", i32), _dev_ptr(self.status, "status"), pages, table.shape[0], table.shape[1],
            layers, kv_heads, head_dim, page_tokens, KV_CODES[codes])
        self._handle = _checked(self._c)
        self._needs = {}  # workspace bytes by call and sizes
        self._heads, self._dim, self._device = kv_heads, head_dim, k.device
        self._lib, self._i32, self._f32, self._u8 = load(), i32, f32, u8
        self._query_types = {torch.bfloat16: 0, torch.float16: 1}
        self._types = _types()
        self._own = (k, v, k_scale, v_scale, table, lens, refs, self.status)
        self._streams = set()  # that the cache has been used on by name

    def _used(self, stream, *tensors) -> None:
        """Keeps the memory of what a call works on until work queued on `stream` is done."""
        if stream is not None:
            if stream.cuda_stream not in self._streams:  # (once is enough for as long as they live)
                self._streams.add(stream.cuda_stream)
                _used(stream, *self._own)
            _used(stream, *tensors)

    def _entries(self, a, b, name_a: str, name_b: str, stream, extra: int = 0):
        """Two int32 arrays of as many entries (the second `extra` more)."""
        i32, n = self._i32, a.numel()
        if a.dim() != 1 or b.dim() != 1 or b.numel() != n + extra:
            raise ValueError(f"{name_a} must be [n] and {name_b} [n{' + 1' if extra else ''}]")
        self._used(stream, a, b)
        return _ptr(a, name_a, i32), _ptr(b, name_b, i32), n

    def _need(self, fn: str, *sizes) -> int:
        need = self._needs.get((fn, sizes))
        if need is None:
            out = C.c_size_t()
            check(getattr(self._lib, fn)(self._handle, *sizes, C.byref(out)))
            if len(self._needs) >= 4096:
                self._needs.clear()
            need = self._needs[fn, sizes] = max(out.value, 16)
        return need

    def _workspace(self, workspace, stream, fn: str, *sizes):
        if workspace is None:
            need = self._need(fn, *sizes)
            workspace = _empty(need, self._u8, self._device, stream)
            return workspace, workspace.data_ptr(), need
        self._used(stream, workspace)
        return workspace, _dev_ptr(workspace, "workspace"), workspace.numel() * workspace.element_size()

    def append(self, layer: int, slots, starts, k, v, stream=None) -> None:
        """tq_kv_append: the last tokens of the sequences in `slots` (int32 [n]),
        sequence i's at starts[i] .. starts[i+1] - 1 (int32 [n + 1]) of k and v
        ([tokens, kv_heads, head_dim], bfloat16, float16 or float32, any strides
        but the last)."""
        ps, pt, n = self._entries(slots, starts, "slots", "starts", stream, 1)
        kp, kt, k0, k1, total = _rows(k, "k", self._heads, self._dim, self._types)
        vp, vt, v0, v1, tokens = _rows(v, "v", self._heads, self._dim, self._types)
        if kt != vt or tokens != total:
            raise ValueError("k and v must have one type and shape")
        self._used(stream, k, v)
        check(self._lib.tq_kv_append(self._handle, layer, ps, pt, n, kp, vp, kt, total, k0, k1, v0, v1,
                                     _stream(stream)))

    def attention_workspace(self, n: int, total: int, heads: int) -> int:
        """tq_kv_attend_workspace: device bytes for up to `total` queries of up to n sequences and `heads` heads."""
        return self._need("tq_kv_attend_workspace", n, total, heads)

    def attention(self, layer: int, slots, starts, q, scale: float | None = None, window: int = 0, out=None,
                  lse=None, return_lse: bool = False, workspace=None, stream=None):
        """tq_kv_attend: causal attention of the last tokens of the sequences over
        the cache; q [tokens, heads, head_dim] bfloat16 or float16 (any strides but
        the last), heads a multiple of kv_heads; scale 1 / sqrt(head_dim) by
        default; window 0, or the tokens that a query sees.  Returns out
        [tokens, heads, head_dim], or (out, lse float32 [tokens, heads]) with
        `return_lse`."""
        head, tail, result = self._attend(slots, starts, q, out, lse, return_lse, workspace, stream,
                                          "tq_kv_attend_workspace")
        check(self._lib.tq_kv_attend(self._handle, layer, *head, self._dim ** -0.5 if scale is None else scale,
                                     min(window, INT_MAX), *tail))
        return result

    def _attend(self, slots, starts, q, out, lse, return_lse, workspace, stream, need: str):
        """What the attention calls have in common: arguments up to the queries' strides, those from `out` on, results."""
        ps, pt, n = self._entries(slots, starts, "slots", "starts", stream, 1)
        if q.dim() != 3:
            raise ValueError(f"q must be [tokens, heads, {self._dim}]")
        heads, dim = q.shape[1], self._dim
        qp, qt, q0, q1, total = _rows(q, "q", heads, dim, self._query_types)
        self._used(stream, q, out, lse)
        if out is None:
            out = _empty((total, heads, dim), q.dtype, q.device, stream)
            op = out.data_ptr()
        else:
            if out.shape != (total, heads, dim):
                raise ValueError(f"out must be {(total, heads, dim)}")
            op = _ptr(out, "out", q.dtype)
        lp = None
        if lse is not None:
            if lse.shape != (total, heads):
                raise ValueError(f"lse must be {(total, heads)}")
            lp = _ptr(lse, "lse", self._f32)
        elif return_lse:
            lse = _empty((total, heads), self._f32, q.device, stream)
            lp = lse.data_ptr()
        workspace, wp, wb = self._workspace(workspace, stream, need, n, total, heads)
        return ((ps, pt, n, qp, qt, total, heads, q0, q1), (op, lp, wp, wb, _stream(stream)),
                (out, lse) if return_lse else out)

    def cross_attention(self, layer: int, slots, starts, q, scale: float | None = None, out=None, lse=None,
                        return_lse: bool = False, workspace=None, stream=None):
        """tq_kv_cross: attention of queries over all tokens that the slots hold,
        whatever the queries' number and place (a reader over encoded passages);
        arguments, workspace (`attention_workspace`) and results as for
        `attention`."""
        head, tail, result = self._attend(slots, starts, q, out, lse, return_lse, workspace, stream,
                                          "tq_kv_attend_workspace")
        check(self._lib.tq_kv_cross(self._handle, layer, *head, self._dim ** -0.5 if scale is None else scale, *tail))
        return result

    def share(self, slots, starts, plan=None, stream=None):
        """tq_kv_share: which neighbouring requests hold the same first pages:
        plan int32 [3, n], for each request its group's first request, how many
        there are, and the tokens that they share before their new ones."""
        ps, pt, n = self._entries(slots, starts, "slots", "starts", stream, 1)
        self._used(stream, plan)
        if plan is None:
            plan = _empty((3, n), self._i32, self._device, stream)
        elif plan.shape != (3, n):
            raise ValueError(f"plan must be {(3, n)}")
        check(self._lib.tq_kv_share(self._handle, ps, pt, n, _ptr(plan, "plan", self._i32), _stream(stream)))
        return plan

    def shared_attention_workspace(self, n: int, total: int, heads: int) -> int:
        """tq_kv_attend_shared_workspace: device bytes for up to `total` queries of up to n requests and `heads` heads."""
        return self._need("tq_kv_attend_shared_workspace", n, total, heads)

    def shared_attention(self, layer: int, slots, starts, plan, q, groups: int | None = None,
                         scale: float | None = None, out=None, lse=None, return_lse: bool = False, workspace=None,
                         stream=None):
        """tq_kv_attend_shared: `attention` (without a window) where the tokens that
        the requests of a group share are read once for all its queries; `plan`
        from `share`.  groups: groups and single requests of the plan, which the
        choice of a kernel goes by (None: taken as n, right for a few requests of a
        group; many over a long passage are several times faster with the number)."""
        if plan.shape != (3, slots.numel()):
            raise ValueError(f"plan must be {(3, slots.numel())}")
        self._used(stream, plan)
        plan = _ptr(plan, "plan", self._i32)
        head, tail, result = self._attend(slots, starts, q, out, lse, return_lse, workspace, stream,
                                          "tq_kv_attend_shared_workspace")
        ps, pt, n, *queries = head
        check(self._lib.tq_kv_attend_shared(self._handle, layer, ps, pt, plan, n, n if groups is None else groups,
                                            *queries, self._dim ** -0.5 if scale is None else scale, *tail))
        return result

    def fork(self, dst, src, stream=None) -> None:
        """tq_kv_fork: slots dst hold what slots src hold, in the same pages."""
        pd, ps, n = self._entries(dst, src, "dst", "src", stream)
        check(self._lib.tq_kv_fork(self._handle, pd, ps, n, _stream(stream)))

    def extend(self, slots, counts, workspace=None, stream=None) -> None:
        """tq_kv_extend: room for counts[i] more tokens in slots[i]; a shared last
        page that is part full is replaced by a copy."""
        ps, pc, n = self._entries(slots, counts, "slots", "counts", stream)
        workspace, wp, wb = self._workspace(workspace, stream, "tq_kv_extend_workspace", n)
        check(self._lib.tq_kv_extend(self._handle, ps, pc, n, wp, wb, _stream(stream)))

    def truncate(self, slots, lens, stream=None) -> None:
        """tq_kv_truncate: slots[i] keeps its first lens[i] tokens (0: none)."""
        ps, pl, n = self._entries(slots, lens, "slots", "lens", stream)
        check(self._lib.tq_kv_truncate(self._handle, ps, pl, n, _stream(stream)))

    def compact(self, workspace=None, stream=None):
        """tq_kv_compact: moves the pages in use to the front of the pool; returns
        how many there are (int32 [1] on the device)."""
        workspace, wp, wb = self._workspace(workspace, stream, "tq_kv_compact_workspace")
        self._used(stream)
        used = _empty(1, _torch().int32, self.k.device, stream)
        check(self._lib.tq_kv_compact(self._handle, used.data_ptr(), wp, wb, _stream(stream)))
        return used

    def check(self, stream=None) -> None:
        """tq_kv_check: waits for the stream; raises TQError if a call since the
        last check found too few free pages (TQ_ENOMEM) or left entries out
        (TQ_EINVAL)."""
        check(self._lib.tq_kv_check(self._handle, _stream(stream)))


def verify_drafts(target_probs, drafts, uniforms, noise, draft_probs=None, draft_lens=None, tokens=None, accepted=None,
                  workspace=None, stream=None):
    """tq_verify_drafts: drafted tokens against the target's probabilities.

    target_probs [n, t + 1, vocab] and draft_probs [n, t, vocab] (None: drafts
    proposed with certainty, such as a retrieved passage's own words) float32,
    bfloat16 or float16; drafts int32 [n, t]; draft_lens int32 [n] (None: t for
    all); uniforms float32 [n, t] in [0, 1); noise float32 [n, vocab],
    exponentially distributed.  Returns (tokens int32 [n, t + 1]: the accepted
    drafts, the token drawn behind them, then -1; accepted int32 [n])."""
    torch = _torch()
    types = _types()
    if target_probs.dim() != 3:
        raise ValueError("target_probs must be [n, t + 1, vocab]")
    n, t, vocab = target_probs.shape
    t -= 1
    dtype, i32, f32, dev = target_probs.dtype, torch.int32, torch.float32, target_probs.device

    def ptr(x, name, kind, *shape):
        if x is None:
            return None
        if x.shape != shape:
            raise ValueError(f"{name} must be {shape}, got {tuple(x.shape)}")
        return _ptr(x, name, kind)

    args = (target_probs.data_ptr(), ptr(draft_probs, "draft_probs", dtype, n, t, vocab), types.get(dtype),
            ptr(drafts, "drafts", i32, n, t), ptr(draft_lens, "draft_lens", i32, n),
            ptr(uniforms, "uniforms", f32, n, t), ptr(noise, "noise", f32, n, vocab), n, t, vocab)
    if not target_probs.is_cuda or dtype not in types or not target_probs.is_contiguous():
        _dev_ptr(target_probs, "target_probs", tuple(types))
    _used(stream, target_probs, draft_probs, drafts, draft_lens, uniforms, noise, tokens, accepted, workspace)
    if tokens is None:
        tokens = _empty((n, t + 1), i32, dev, stream)
    if accepted is None:
        accepted = _empty(n, i32, dev, stream)
    if workspace is None:
        workspace = _empty(_verify_need(n, vocab), torch.uint8, dev, stream)
    check(load().tq_verify_drafts(*args, ptr(tokens, "tokens", i32, n, t + 1), ptr(accepted, "accepted", i32, n),
                                  _dev_ptr(workspace, "workspace"), workspace.numel() * workspace.element_size(),
                                  _stream(stream)))
    return tokens, accepted


@functools.lru_cache(maxsize=4096)
def _verify_need(n: int, vocab: int) -> int:
    need = C.c_size_t()
    check(load().tq_verify_drafts_workspace(n, vocab, C.byref(need)))
    return max(need.value, 16)


def sample_tokens(logits, noise, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None, logprobs=None,
                  return_logprobs=False, workspace=None, stream=None):
    """tq_sample: the next token of each row of logits, from given random numbers.

    logits [n, vocab] float32, bfloat16 or float16 and noise float32 [n, vocab],
    exponentially distributed, with any row stride; temperature, top_p, min_p float32
    [n] and top_k int32 [n] on the device, or None: off (temperature 1).  Returns
    tokens int32 [n], or (tokens, logprobs float32 [n]: at temperature 1, over all
    tokens) with `return_logprobs`."""
    torch = _torch()
    types, i32, f32, dev = _types(), torch.int32, torch.float32, logits.device
    if logits.dim() != 2 or noise.shape != logits.shape:
        raise ValueError("logits and noise must both be [n, vocab]")
    n, vocab = logits.shape
    for t, name, kinds in ((logits, "logits", tuple(types)), (noise, "noise", (f32,))):
        if t.dtype not in kinds or not t.is_cuda:
            _dev_ptr(t, name, kinds, contiguous=False)
        if t.stride(1) != 1 and vocab > 1:
            raise ValueError(f"{name}: the elements of a row must lie side by side")

    def ptr(x, name, kind):
        if x is None:
            return None
        if x.shape != (n,):
            raise ValueError(f"{name} must be {(n,)}, got {tuple(x.shape)}")
        return _ptr(x, name, kind)

    settings = (ptr(temperature, "temperature", f32), ptr(top_k, "top_k", i32), ptr(top_p, "top_p", f32),
                ptr(min_p, "min_p", f32))
    _used(stream, logits, noise, temperature, top_k, top_p, min_p, tokens, logprobs, workspace)
    if tokens is None:
        tokens = _empty(n, i32, dev, stream)
    if logprobs is None and return_logprobs:
        logprobs = _empty(n, f32, dev, stream)
    if workspace is None:
        workspace = _empty(_sample_need(n, vocab), torch.uint8, dev, stream)
    # (one row has no next one: a view of it may say any stride)
    step, noise_step = (logits.stride(0), noise.stride(0)) if n > 1 else (vocab, vocab)
    check(load().tq_sample(logits.data_ptr(), types[logits.dtype], step, noise.data_ptr(), noise_step, n, vocab,
                           *settings, ptr(tokens, "tokens", i32), ptr(logprobs, "logprobs", f32), _dev_ptr(workspace, "workspace"),
                           workspace.numel() * workspace.element_size(), _stream(stream)))
    return (tokens, logprobs) if return_logprobs else tokens


@functools.lru_cache(maxsize=4096)
def _sample_need(n: int, vocab: int) -> int:
    need = C.c_size_t()
    check(load().tq_sample_workspace(n, vocab, C.byref(need)))
    return max(need.value, 16)
