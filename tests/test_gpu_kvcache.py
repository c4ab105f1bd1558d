"""The 8-bit key-value cache on the GPU against plain forms in 64 bits:
quantising appends, attention, pages."""
import math

import numpy as np
import pytest

import kvref

pytestmark = pytest.mark.gpu

STALE = 0x7F  # what unwritten slots hold here: NaN as e4m3, 127 as int8


class Case:
    """A cache of sequences in shuffled slots and pages, on the host and on the GPU."""

    def __init__(self, tq, lens, new, *, kv_heads=2, dim=128, page=64, codes="int8", seed=0, spare_pages=3, layers=2):
        import torch
        rng = np.random.default_rng(seed)
        self.tq, self.torch, self.rng, self.codes, self.page = tq, torch, rng, codes, page
        n = len(lens)
        need = [-(-x // page) for x in lens]
        pages, slots = sum(need) + spare_pages, n + 2
        self.slots = rng.permutation(slots)[:n].astype(np.int32)
        order = rng.permutation(pages).astype(np.int32)
        self.table = np.full((slots, max(need + [1]) + 1), -1, np.int32)
        self.lens = np.zeros(slots, np.int32)
        self.refs = np.zeros(pages, np.int32)
        at = 0
        for slot, x, m in zip(self.slots, lens, need):
            self.table[slot, :m] = order[at: at + m]
            self.refs[order[at: at + m]] = 1
            self.lens[slot] = x
            at += m
        shape = (layers, pages, kv_heads, page, dim)
        self.pool = {name: np.full(shape, STALE, np.uint8) for name in "kv"}
        self.scale = {name: np.full(shape[:3] + (page // 16,), np.nan, np.float32) for name in "kv"}
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.layer = layers - 1

    def fill(self, spread=0.3):
        """Random codes for the tokens held, in the last layer."""
        rng, page = self.rng, self.page
        for slot in self.slots:
            for t in range(0, int(self.lens[slot]), 16):
                p, b, m = self.table[slot, t // page], t % page // 16, min(16, int(self.lens[slot]) - t)
                for name in "kv":
                    x = rng.standard_normal((self.pool["k"].shape[2], m, self.pool["k"].shape[4]))
                    c = kvref.to_codes(np.clip(x * (36 if self.codes == "int8" else 127), -127, 127), self.codes)
                    self.pool[name][self.layer, p, :, b * 16: b * 16 + m] = c
                    self.scale[name][self.layer, p, :, b] = np.exp(rng.normal(0, spread, c.shape[0])) / (
                        36 if self.codes == "int8" else 127)
        return self

    def device(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x)).cuda()

    def cache(self):
        d = self.device
        return self.tq.KVCache.from_tensors(d(self.pool["k"]), d(self.pool["v"]), d(self.scale["k"]), d(self.scale["v"]),
                                            d(self.table), d(self.lens), d(self.refs), codes=self.codes)

    def queries(self, heads, type, width=2.0):
        x = self.rng.standard_normal((int(self.starts[-1]), heads, self.pool["k"].shape[4])) * width
        return self.device(x.astype(np.float32)).to(getattr(self.torch, type))

    def expected(self, q, window=0, scale=None):
        scale = 1 / math.sqrt(q.shape[2]) if scale is None else scale
        parts = []
        for i, slot in enumerate(self.slots):
            n = int(self.lens[slot])
            k, v = (kvref.read(self.pool[x][self.layer], self.scale[x][self.layer], self.table, slot, n, self.codes)
                    for x in "kv")
            parts.append(kvref.attention(k, v, q[self.starts[i]: self.starts[i + 1]], scale, window))
        return [np.concatenate(x) for x in zip(*parts)]


def check_attention(case, q, window=0, scale=None, **kw):
    cache = case.cache()
    out, lse = cache.attention(case.layer, case.device(case.slots), case.device(case.starts), q, window=window,
                               scale=scale, return_lse=True, **kw)
    cache.check()
    compare(case, q, out, lse, window, scale)
    return cache


def compare(case, q, out, lse, window=0, scale=None):
    """Bounds: a weight is held in at least 8 significant bits (relative error
    2^-9), its exponent is off by the error of its score and of the running
    maximum (2 x error); the result is rounded once more, to its type."""
    ref, ref_lse, size, error = case.expected(q.double().cpu().numpy(), window, scale)
    half_ulp = 2.0 ** -9 if q.dtype == case.torch.bfloat16 else 2.0 ** -12
    assert out.dtype == q.dtype and out.shape == q.shape
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    bound = (2.0 ** -9 + 4 * error[..., None] + 1e-6) * size + half_ulp * np.abs(ref) + 2.0 ** -24
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) / bound)
    seen = np.isfinite(ref_lse)
    assert np.array_equal(seen, np.isfinite(got_lse)) and (got_lse[~seen] == -np.inf).all()
    assert (np.abs(got_lse - ref_lse)[seen] <= (2 * error + 2.0 ** -21 * np.abs(ref_lse) + 2e-6)[seen]).all()
    assert not got[~seen].any()


LENGTHS = [
    ([1], [1]),
    ([0, 1, 15, 16, 17, 31, 33], [1] * 7),                     # an empty sequence among them
    ([700, 64, 65, 1300, 128], [1] * 5),
    ([40, 3, 200, 0], [5, 3, 8, 2]),                           # drafts; a sequence that only has them; an empty one
    ([150, 40], [33, 40]),                                     # (part of) a prompt
    ([300, 10, 140], [140, 10, 129]),
]


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,new", LENGTHS)
@pytest.mark.parametrize("dim,group,type", [(128, 4, "bfloat16"), (64, 5, "float16"), (256, 1, "bfloat16"),
                                            (128, 16, "float16")])
def test_attention(cuda_lib, codes, lens, new, dim, group, type):
    case = Case(cuda_lib, lens, new, dim=dim, codes=codes, seed=len(lens) + dim).fill()
    check_attention(case, case.queries(2 * group, type))


@pytest.mark.parametrize("page", [16, 32, 128, 256])
@pytest.mark.parametrize("kv_heads,group", [(1, 8), (3, 7)])
def test_attention_page_sizes(cuda_lib, page, kv_heads, group):
    case = Case(cuda_lib, [500, 16, 257, 90], [1, 1, 4, 70], page=page, kv_heads=kv_heads, seed=page).fill()
    check_attention(case, case.queries(kv_heads * group, "bfloat16"))


@pytest.mark.parametrize("window", [1, 16, 37, 128, 5000])
@pytest.mark.parametrize("new", [[1, 1, 1], [6, 3, 2], [150, 100, 20]])
def test_attention_window(cuda_lib, window, new):
    case = Case(cuda_lib, [400, 129, 20], new, codes="e4m3", seed=window).fill()
    check_attention(case, case.queries(8, "bfloat16"), window=window)


@pytest.mark.parametrize("spread,scale,width", [(0.3, 4.0, 2.0), (5.0, None, 2.0), (0.3, -1.0, 1.0), (0.3, 0.0, 1.0),
                                                (0.3, 1e-5, 1e4), (0.3, 1e-4, 6e-6)])
@pytest.mark.parametrize("new", [1, 40])
def test_attention_ranges(cuda_lib, spread, scale, width, new):
    """Peaked, flat and reversed weights, blocks whose scales differ by e^10, queries close to fp16's ends."""
    case = Case(cuda_lib, [300, 90], [new, new], seed=3).fill(spread)
    check_attention(case, case.queries(8, "float16", width), scale=scale)


def test_attention_zero_blocks(cuda_lib):
    """Blocks of zero scale: all keys and values zero, as an append of zeros leaves them."""
    case = Case(cuda_lib, [100, 200], [1, 50], seed=4).fill()
    for name in "kv":
        for slot in case.slots:
            p = case.table[slot, 0]
            case.pool[name][case.layer, p, :, 16:48] = 0
            case.scale[name][case.layer, p, :, 1:3] = 0
    check_attention(case, case.queries(8, "bfloat16"))


@pytest.mark.parametrize("new", [1, 20, 130])
def test_attention_strides_and_streams(cuda_lib, new):
    """Queries as a slice of a projection, head-major and off the 16-byte grid; work on a side stream; kept buffers."""
    import torch
    case = Case(cuda_lib, [300, 150], [new, new], seed=5).fill()
    q = case.queries(8, "bfloat16")
    total = q.shape[0]
    fused = torch.zeros(total, 12, 128, dtype=q.dtype, device="cuda")
    fused[:, 2:10] = q
    major = q.transpose(0, 1).contiguous().transpose(0, 1)
    odd = torch.zeros(total * 8 * 128 + 3, dtype=q.dtype, device="cuda")[3:].view(total, 8, 128)
    odd.copy_(q)
    want = None
    for x in (q, fused[:, 2:10], major, odd):
        cache = case.cache()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        args = (case.layer, case.device(case.slots), case.device(case.starts), x)
        torch.cuda.synchronize()
        out, lse = cache.attention(*args, return_lse=True, stream=side)
        side.synchronize()
        if want is None:
            want = out.clone()
            compare(case, q, out, lse)
        assert torch.equal(out, want)
        ws = torch.full((cache.attention_workspace(2, total, 8),), 0xFF, dtype=torch.uint8, device="cuda")
        buf = torch.empty_like(out)
        got = cache.attention(*args, out=buf, workspace=ws)
        assert got is buf and torch.equal(buf, want)


def test_attention_many_sequences(cuda_lib):
    """More sequences than a warp probes at once, some without new tokens."""
    rng = np.random.default_rng(6)
    lens = rng.integers(1, 70, 300).tolist()
    new = [int(min(x, rng.integers(0, 3))) for x in lens]
    case = Case(cuda_lib, lens, new, kv_heads=1, dim=64, page=16, seed=6).fill()
    check_attention(case, case.queries(4, "float16"))


@pytest.mark.parametrize("new", [1, 64])
def test_attention_long(cuda_lib, new):
    """A length that is split over many blocks; scores that grow with the place, so that the running maximum moves."""
    case = Case(cuda_lib, [9000], [new], kv_heads=1, dim=64, seed=7).fill(0.0)
    rise = np.linspace(0.2, 2.0, case.scale["k"].shape[1]).astype(np.float32)
    pages = case.table[case.slots[0]]
    for i, p in enumerate(pages[pages >= 0]):
        case.scale["k"][case.layer, p] *= rise[i]
    check_attention(case, case.queries(2, "float16"))


def test_attention_offsets_beyond_32_bits(cuda_lib):
    """Pages whose codes lie more than 2^32 bytes into the pool: appended to, attended to, moved."""
    import torch
    page, dim, heads = 64, 128, 8
    pages = (1 << 32) // (page * dim * heads) + 40
    cache = cuda_lib.KVCache(pages, 2, 4, heads, dim, page)
    cache.refs.fill_(1)
    cache.refs[-5:] = 0
    slots = torch.tensor([1], dtype=torch.int32, device="cuda")
    counts = torch.tensor([100], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 100], dtype=torch.int32, device="cuda")
    cache.extend(slots, counts)
    assert cache.table[1, :2].tolist() == [pages - 5, pages - 4]
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v, q = (torch.randn(100, heads, dim, device="cuda", generator=g).to(torch.bfloat16) for _ in range(3))
    cache.append(0, slots, starts, k, v)
    out = cache.attention(0, slots, starts, q)
    cache.check()

    def plain():
        kk, vv = (torch.cat([(c[0, p].view(torch.int8).double() * s[0, p].double().repeat_interleave(16, 1)[..., None])
                             for p in cache.table[1, :2].tolist()], 1)[:, :100]
                  for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        s = torch.einsum("thd,hjd->htj", q.double(), kk) / math.sqrt(dim)
        s.masked_fill_(torch.ones(100, 100, device="cuda").triu(1).bool(), -math.inf)
        return torch.einsum("htj,hjd->thd", torch.softmax(s, 2), vv)

    assert (out.double() - plain()).abs().max() < 0.03  # 2^-8 of values up to 4, and the codes are the same on both sides
    assert (plain() - torch.cumsum(v.double(), 0)).abs().max() > 0.1  # (a plain form that looks at the keys)
    cache.refs.fill_(0)
    cache.refs[[0, pages - 5, pages - 4]] = 1
    used = cache.compact()
    assert used.item() == 3 and cache.table[1, :2].tolist() == [1, 2]
    assert torch.equal(cache.attention(0, slots, starts, q), out)


def test_attention_deterministic(cuda_lib):
    case = Case(cuda_lib, [5000, 3000, 17], [1, 40, 1], seed=8).fill()
    q = case.queries(8, "bfloat16")
    cache = case.cache()
    args = (case.layer, case.device(case.slots), case.device(case.starts), q)
    a = cache.attention(*args, return_lse=True)
    for _ in range(5):
        b = cache.attention(*args, return_lse=True)
        assert case.torch.equal(a[0], b[0]) and case.torch.equal(a[1], b[1])


def test_attention_leaves_out_bad_entries(cuda_lib):
    """A slot or a page that does not exist gives zeros for its queries, the others are served, check() says so."""
    case = Case(cuda_lib, [100, 90, 80], [1, 1, 1], seed=9).fill()
    q = case.queries(8, "bfloat16")
    good = case.cache().attention(case.layer, case.device(case.slots), case.device(case.starts), q)
    for what in ("slot", "length", "page"):
        cache = case.cache()
        slots = case.slots.copy()
        if what == "slot":
            slots[1] = 99
        elif what == "length":
            cache.lens[int(slots[1])] = 1 << 20
        else:
            cache.table[int(slots[1]), 0] = 1 << 20
        out = cache.attention(case.layer, case.device(slots), case.device(case.starts), q)
        with pytest.raises(cuda_lib.TQError, match="TQ_EINVAL"):
            cache.check()
        cache.check()
        assert case.torch.equal(out[0], good[0]) and case.torch.equal(out[2], good[2])


# ---- append -----------------------------------------------------------------

def run_append(case, new_k, new_v, cache=None):
    cache = cache or case.cache()
    cache.append(case.layer, case.device(case.slots), case.device(case.starts), new_k, new_v)
    cache.check()
    return cache


def check_append(case, cache, new_k, new_v):
    """Codes and scales are the definition's, bit for bit; slots that hold no token keep what they had."""
    for name, x in (("k", new_k), ("v", new_v)):
        pool, scale = case.pool[name][case.layer].copy(), case.scale[name][case.layer].copy()
        kvref.append(pool, scale, case.table, case.lens, case.slots, case.starts, x.float().cpu().numpy(), case.codes)
        got, got_scale = getattr(cache, name).cpu().numpy(), getattr(cache, name + "_scale").cpu().numpy()
        assert np.array_equal(got_scale[case.layer], scale, equal_nan=True)
        if case.codes == "e4m3":  # (zero has two codes)
            got, pool = np.where(got == 128, 0, got), np.where(pool == 128, 0, pool)
        assert np.array_equal(got[case.layer], pool)
        assert (got[: case.layer] == STALE).all()


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("type", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 32)])
@pytest.mark.parametrize("lens,new", [([1], [1]), ([16, 17, 31, 48, 5], [1, 1, 2, 16, 5]), ([200, 33, 3], [150, 17, 0])])
def test_append(cuda_lib, codes, type, dim, page, lens, new):
    import torch
    case = Case(cuda_lib, lens, new, dim=dim, page=page, codes=codes, seed=dim + len(lens)).fill()
    total = sum(new)
    k, v = (case.device(case.rng.standard_normal((total, 2, dim)).astype(np.float32) * w).to(getattr(torch, type))
            for w in (1.5, 0.2))
    check_append(case, run_append(case, k, v), k, v)


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
@pytest.mark.parametrize("type", ["float32", "bfloat16"])
def test_append_values(cuda_lib, codes, type):
    """NaN, infinities, zeros, subnormals, values at rounding boundaries."""
    import torch
    case = Case(cuda_lib, [96], [96], codes=codes, seed=1)
    x = case.rng.standard_normal((96, 2, 128)).astype(np.float32)
    x[0, 0, :3] = [np.nan, np.inf, -np.inf]     # the block's finite values set its scale
    x[16:32] = 0                                 # nothing but zeros
    x[32:48, 0] = np.nan                         # nothing finite
    x[32:48, 1] = np.inf
    x[48:64] *= np.float32(1e-39)                # subnormal values and scales
    x[64:80] *= np.float32(5e37)
    x[80:96] = (case.rng.integers(-254, 255, (16, 2, 128)) / 2).astype(np.float32)  # halves: ties
    x[80] = 127
    k = case.device(x).to(getattr(torch, type))
    check_append(case, run_append(case, k, k), k, k)
    cache = run_append(case, k, k)
    assert torch.isfinite(cache.k_scale[case.layer, case.table[case.slots[0]][:2].tolist()][:, :, :2]).all()


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_append_token_by_token(cuda_lib, codes):
    """A block's scale grows with its tokens and its older codes follow; the result stays within the rounding
    of every rescaling: a half step of each scale that the block went through."""
    import torch
    case = Case(cuda_lib, [40], [40], codes=codes, seed=2)
    x = case.rng.standard_normal((40, 2, 128)).astype(np.float32) * np.linspace(0.1, 3, 40, dtype=np.float32)[:, None, None]
    cache = case.cache()
    slots = case.device(case.slots)
    starts = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for t in range(40):
        cache.lens[int(case.slots[0])] = t + 1
        part = case.device(x[t: t + 1])
        cache.append(case.layer, slots, starts, part, part)
    cache.check()
    pool, scale = case.pool["k"][case.layer].copy(), case.scale["k"][case.layer].copy()
    lens = case.lens.copy()
    for t in range(40):
        lens[case.slots[0]] = t + 1
        kvref.append(pool, scale, case.table, lens, case.slots, [0, 1], x[t: t + 1], codes)
    got = kvref.read(cache.k[case.layer].cpu().numpy(), cache.k_scale[case.layer].cpu().numpy(), case.table,
                     case.slots[0], 40, codes)
    assert np.array_equal(got, kvref.read(pool, scale, case.table, case.slots[0], 40, codes))
    if codes == "int8":  # at most 16 roundings of half a step, at scales up to the last
        last = np.repeat(scale[case.table[case.slots[0], 0]].T, 16, 0)[:40]
        assert (np.abs(got - x) <= 8 * last[:, :, None]).all()


def test_append_strides(cuda_lib):
    """Keys and values as slices of one projection, head-major, and off the 16-byte grid; a head stride of 0."""
    import torch
    case = Case(cuda_lib, [30, 77], [30, 20], seed=3).fill()
    k, v = (case.device(case.rng.standard_normal((50, 2, 128)).astype(np.float32)).to(torch.bfloat16) for _ in range(2))
    fused = torch.zeros(50, 9, 128, dtype=torch.bfloat16, device="cuda")
    fused[:, 5:7], fused[:, 7:] = k, v
    odd = torch.zeros(50 * 2 * 128 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(50, 2, 128)
    odd.copy_(v)
    for kk, vv in ((k, v), (fused[:, 5:7], fused[:, 7:]), (k.transpose(0, 1).contiguous().transpose(0, 1), odd)):
        check_append(case, run_append(case, kk, vv), k, v)
    one = k[:, :1].expand(50, 2, 128)
    check_append(case, run_append(case, one, one), one, one)


def test_append_leaves_out_bad_entries(cuda_lib):
    import torch
    case = Case(cuda_lib, [30, 40, 50], [10, 10, 10], seed=4).fill()
    k = case.device(case.rng.standard_normal((30, 2, 128)).astype(np.float32)).to(torch.bfloat16)
    good = run_append(case, k, k)
    bad = int(case.slots[1])
    for what in ("slot", "length", "page"):
        cache, slots = case.cache(), case.slots.copy()
        if what == "slot":
            slots[1] = -1
        elif what == "length":
            cache.lens[bad] = 5
        else:
            cache.table[bad, 0] = -1
        cache.append(case.layer, case.device(slots), case.device(case.starts), k, k)
        with pytest.raises(cuda_lib.TQError, match="TQ_EINVAL"):
            cache.check()
        keep = [int(p) for s in (0, 2) for p in case.table[case.slots[s]] if p >= 0]
        lost = int(case.table[bad, 0])
        assert torch.equal(cache.k[:, keep], good.k[:, keep])
        assert (cache.k[:, lost].cpu().numpy() == case.pool["k"][:, lost]).all()


# ---- pages ------------------------------------------------------------------

class Model:
    """The cache's bookkeeping in plain Python; a page's content is a list of stamps, one for each token."""

    def __init__(self, pages, slots, max_pages, page):
        self.refs, self.page, self.max_pages = [0] * pages, page, max_pages
        self.table, self.lens = [[-1] * max_pages for _ in range(slots)], [0] * slots
        self.data = np.zeros((pages, page), np.int64)

    def count(self, n):
        return -(-n // self.page)

    def fork(self, dst, src):
        for d, s in zip(dst, src):
            self.truncate([d], [0])
            for p in range(self.count(self.lens[s])):
                self.table[d][p] = self.table[s][p]
                self.refs[self.table[s][p]] += 1
            self.lens[d] = self.lens[s]

    def truncate(self, slots, lens):
        for s, n in zip(slots, lens):
            for p in range(self.count(n), self.count(self.lens[s])):
                self.refs[self.table[s][p]] -= 1
                self.table[s][p] = -1
            self.lens[s] = n

    def extend(self, slots, counts):
        free = [p for p, r in enumerate(self.refs) if r == 0]
        plan = []
        for s, c in zip(slots, counts):
            n = self.lens[s]
            last = self.table[s][n // self.page] if n % self.page else -1
            copy = c > 0 and last >= 0 and self.refs[last] > 1
            take = self.count(n + c) - self.count(n) + copy
            if n + c > self.max_pages * self.page:
                return False
            plan.append((s, c, n, last if copy else -1, take))
        if sum(x[4] for x in plan) > len(free):
            return False
        for s, c, n, last, take in plan:
            first = self.count(n) - (last >= 0)
            for i in range(take):
                self.table[s][first + i] = free.pop(0)
                self.refs[self.table[s][first + i]] = 1
            if last >= 0:
                self.refs[last] -= 1
                used = -(-(n % self.page) // 16) * 16
                self.data[self.table[s][first], :used] = self.data[last, :used]
            self.lens[s] += c
        return True

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] == 0]
        tail = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        name = dict(zip(tail, holes))
        for old, new in name.items():
            self.refs[new], self.refs[old] = self.refs[old], 0
            self.data[new] = self.data[old]
        self.table = [[name.get(p, p) for p in row] for row in self.table]
        return live


@pytest.mark.parametrize("seed,page,pages,layers,heads,dim", [(0, 16, 60, 1, 1, 64), (1, 64, 40, 2, 3, 128),
                                                              (2, 32, 17_000, 1, 1, 64)])
def test_pages_against_a_model(cuda_lib, seed, page, pages, layers, heads, dim):
    """A random sequence of forks, extends, truncates and compactions; every token carries a stamp in each layer,
    head, and K and V."""
    import torch
    rng = np.random.default_rng(seed)
    slots, max_pages = 9, pages // 5 if pages < 1000 else 3000
    model = Model(pages, slots, max_pages, page)
    cache = cuda_lib.KVCache(pages, slots, max_pages, heads, dim, page, layers=layers)
    lane = torch.arange(layers * heads, device="cuda").view(layers, 1, heads, 1, 1)
    i32 = lambda x: torch.tensor([int(v) for v in x], dtype=torch.int32, device="cuda")  # noqa: E731
    stamp = 0
    for step in range(60):
        what = rng.choice(["extend", "extend", "extend", "fork", "truncate", "compact"])
        some = rng.permutation(slots)[: rng.integers(1, 5)]
        if what == "extend":
            counts = rng.integers(0, page * max_pages // 6, len(some)) * (rng.random(len(some)) < 0.8)
            before = [model.lens[s] for s in some]
            done = model.extend(some, counts)
            cache.extend(i32(some), i32(counts))
            if done:
                cache.check()
                for s, n, c in zip(some, before, counts):  # stamp the new tokens
                    for t in range(n, n + int(c), max(1, int(c) // 40)):
                        stamp = (stamp + 1) % 120
                        p = model.table[s][t // page]
                        model.data[p, t % page] = stamp
                        cache.k[:, p, :, t % page] = (lane[:, 0, :, 0] + stamp).to(torch.uint8)
                        cache.v[:, p, :, t % page] = (lane[:, 0, :, 0] + stamp + 100).to(torch.uint8)
                        cache.k_scale[:, p, :, t % page // 16] = float(stamp)
                        cache.v_scale[:, p, :, t % page // 16] = float(stamp) + 0.5
            else:
                with pytest.raises(cuda_lib.TQError):
                    cache.check()
        elif what == "fork":
            half = len(some) // 2
            model.fork(some[:half], some[half: 2 * half])
            cache.fork(i32(some[:half]), i32(some[half: 2 * half]))
        elif what == "truncate":
            lens = [int(rng.integers(0, model.lens[s] + 1)) if rng.random() < 0.7 else 0 for s in some]
            model.truncate(some, lens)
            cache.truncate(i32(some), i32(lens))
        else:
            live = model.compact()
            assert cache.compact().item() == live
        cache.check()
        assert cache.table.tolist() == model.table and cache.lens.tolist() == model.lens
        assert cache.refs.tolist() == model.refs
        for s in range(slots):
            n = model.lens[s]
            at = np.arange(n)
            rows = np.asarray(model.table[s])[at // page] if n else np.zeros(0, int)
            want = torch.from_numpy(model.data[rows, at % page]).cuda()
            known = want > 0
            rows, at = torch.from_numpy(rows).cuda()[known], torch.from_numpy(at % page).cuda()[known]
            want = want[known]
            got = cache.k[:, rows, :, at]  # [tokens, layers, heads, dim]
            assert torch.equal(got, (lane.view(1, layers, heads, 1) + want.view(-1, 1, 1, 1)).to(torch.uint8).expand_as(got))
            got = cache.v[:, rows, :, at]
            assert torch.equal(got, (lane.view(1, layers, heads, 1) + want.view(-1, 1, 1, 1) + 100).to(torch.uint8).expand_as(got))


def test_copied_blocks_keep_their_scales(cuda_lib):
    import torch
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = cuda_lib.KVCache(8, 3, 4, 2, 64, 64, layers=3)
    cache.extend(i32(0), i32(100))
    for i, x in enumerate((cache.k, cache.v, cache.k_scale, cache.v_scale)):
        x.copy_((torch.arange(x.numel(), device="cuda") % 251 + i).view(x.shape).to(x.dtype))
    held = [x.clone() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    cache.fork(i32(1, 2), i32(0, 0))
    cache.extend(i32(2, 1), i32(1, 30))
    cache.check()
    assert cache.table[:, :3].tolist() == [[0, 1, -1], [0, 3, 4], [0, 2, -1]]
    assert cache.refs.tolist() == [3, 1, 1, 1, 1, 0, 0, 0] and cache.lens.tolist() == [100, 130, 101]
    for now, was, blocks in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), held, (48, 48, 3, 3)):
        for p in (2, 3):
            assert torch.equal(now[:, p, :, :blocks], was[:, 1, :, :blocks])
            assert torch.equal(now[:, p, :, blocks:], was[:, p, :, blocks:])
        assert torch.equal(now[:, :2], was[:, :2]) and torch.equal(now[:, 4:], was[:, 4:])


def test_pages_refuse_bad_entries(cuda_lib):
    """extend changes nothing at all; fork and truncate leave the bad entries out and carry out the others."""
    import torch
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = cuda_lib.KVCache(10, 6, 4, 1, 64, 16)
    cache.extend(i32(0, 1, 2), i32(20, 5, 40))
    cache.check()

    def state():
        return [x.tolist() for x in (cache.table, cache.lens, cache.refs)]

    before = state()
    for slots, counts, error in (((3, 3), (1, 1), "EINVAL"), ((3, 6), (1, 1), "EINVAL"), ((-1,), (1,), "EINVAL"),
                                 ((3,), (-1,), "EINVAL"), ((3, 2), (1, 30), "EINVAL"), ((3, 4), (64, 1), "ENOMEM"),
                                 ((3,), (2**31 - 1,), "EINVAL")):
        cache.extend(i32(*slots), i32(*counts))
        with pytest.raises(cuda_lib.TQError, match=error):
            cache.check()
        assert state() == before
    cache.fork(i32(3, 4, 4, 0, 5), i32(1, 0, 1, 2, 9))  # 4 twice; 0 is a source too; 9 does not exist
    with pytest.raises(cuda_lib.TQError, match="EINVAL"):
        cache.check()
    assert cache.lens.tolist() == [20, 5, 40, 5, 0, 0]
    assert cache.table[3].tolist() == cache.table[1].tolist() and sum(cache.refs.tolist()) == 2 + 1 + 3 + 1
    cache.truncate(i32(0, 2, 2, 1, 3), i32(1, 0, 0, 6, 0))  # 2 twice; 1 is shorter
    with pytest.raises(cuda_lib.TQError, match="EINVAL"):
        cache.check()
    assert cache.lens.tolist() == [1, 5, 40, 0, 0, 0] and sum(cache.refs.tolist()) == 1 + 1 + 3


def test_nothing_to_do(cuda_lib):
    import torch
    cache = cuda_lib.KVCache(4, 2, 2, 2, 64)
    none, zero = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache.extend(none, none)
    cache.fork(none, none)
    cache.truncate(none, none)
    cache.append(0, none, zero, rows, rows)
    assert cache.attention(0, none, zero, rows).shape == rows.shape
    assert cache.compact().item() == 0
    cache.check()


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_a_decoding_loop_in_a_graph(cuda_lib, codes):
    """extend, append, attention, truncate captured once and replayed: as many steps by hand give the same."""
    import torch
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    def fresh():
        cache = cuda_lib.KVCache(40, 4, 8, 2, 64, 16, codes=codes)
        cache.extend(i32(0), i32(37))
        g = torch.Generator(device="cuda").manual_seed(1)
        x = torch.randn(37, 2, 64, device="cuda", generator=g).to(torch.bfloat16)
        cache.append(0, i32(0), i32(0, 37), x, x)
        cache.fork(i32(1, 2), i32(0, 0))
        return cache

    slots, counts, starts = i32(1, 2, 0), i32(3, 1, 2), i32(0, 3, 4, 6)
    kv, q = (torch.randn(6, h, 64, device="cuda", dtype=torch.bfloat16) for h in (2, 4))

    def step(cache, keep):
        cache.extend(slots, counts)
        cache.append(0, slots, starts, kv, kv)
        o = cache.attention(0, slots, starts, q)
        torch.sub(cache.lens[slots.long()], 1, out=keep)
        cache.truncate(slots, keep)
        return o

    a, keep = fresh(), i32(0, 0, 0)
    for _ in range(4):
        want = step(a, keep)
    a.check()
    b = fresh()
    side = torch.cuda.Stream()
    warm, warm_keep = fresh(), i32(0, 0, 0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(warm, warm_keep)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(b, keep)
    for _ in range(4):
        graph.replay()
    b.check()
    assert torch.equal(got, want)
    for x, y in ((a.table, b.table), (a.lens, b.lens), (a.refs, b.refs), (a.k, b.k), (a.v_scale, b.v_scale)):
        assert torch.equal(x, y)
