"""Refusals of cross attention, shared attention, its plan and of sampling: checked
before any CUDA call, so they run without a GPU."""
import ctypes as C

import pytest

from paper_2607_16973_gb300 import _lib
from test_kvcache_host import ATTEND, BAD_CACHES, P, cache, lib, refused  # noqa: F401  (a fixture)

BIG = 1 << 40


@pytest.mark.parametrize("kw,match", BAD_CACHES)
def test_every_call_checks_the_cache(lib, kw, match):
    c, need = cache(**kw), C.c_size_t()
    refused(lib, lib.tq_kv_cross(c, 0, P, P, 1, P, 0, 1, 4, 512, 128, 1.0, P, P, P, BIG, None), match)
    refused(lib, lib.tq_kv_share(c, P, P, 1, P, None), match)
    refused(lib, lib.tq_kv_attend_shared_workspace(c, 1, 1, 4, C.byref(need)), match)
    refused(lib, lib.tq_kv_attend_shared(c, 0, P, P, P, 1, 1, P, 0, 1, 4, 512, 128, 1.0, P, P, P, BIG, None), match)


CALLS = [
    (dict(layer=2), "layer"), (dict(n=9), "n="), (dict(n=0), "no sequence"), (dict(type=2), "type"), (dict(heads=6), "heads"),
    (dict(heads=0), "heads"), (dict(total=-1), "total"), (dict(total=2 ** 29), "too many"), (dict(scale=float("nan")), "scale"),
    (dict(scale=float("inf")), "scale"), (dict(slots=None), "NULL"), (dict(starts=P + 2), "4-byte"), (dict(q=None), "NULL q"),
    (dict(q=P + 1), "q must be aligned"), (dict(q0=-1), "strides of q"), (dict(q1=2 ** 31), "strides of q"),
    (dict(out=None), "out"), (dict(out=P + 8), "out"), (dict(lse=P + 2), "lse"), (dict(ws=None), "workspace"),
    (dict(ws=P + 8), "workspace"), (dict(bytes=16), "needed")]


@pytest.mark.parametrize("kw,match", CALLS)
def test_attention_refusals(lib, kw, match):
    a = {**ATTEND, **kw}
    tail = a["q"], a["type"], a["total"], a["heads"], a["q0"], a["q1"], a["scale"], a["out"], a["lse"], a["ws"], a["bytes"], None
    refused(lib, lib.tq_kv_cross(cache(), a["layer"], a["slots"], a["starts"], a["n"], *tail), match)
    refused(lib, lib.tq_kv_attend_shared(cache(), a["layer"], a["slots"], a["starts"], P, a["n"], 1, *tail), match)


@pytest.mark.parametrize("plan,groups,match", [(None, 1, "plan"), (P + 2, 1, "plan"), (P, 0, "groups"), (P, 3, "groups")])
def test_plans_that_are_refused(lib, plan, groups, match):
    refused(lib, lib.tq_kv_attend_shared(cache(), 0, P, P, plan, 2, groups, P, 0, 2, 4, 512, 128, 1.0, P, P, P, BIG, None), match)


@pytest.mark.parametrize("kw,match", [(dict(n=-1), "n="), (dict(n=9), "n="), (dict(slots=None), "NULL"), (dict(starts=P + 1), "4-byte"),
                                      (dict(plan=None), "plan"), (dict(plan=P + 2), "plan")])
def test_share_refusals(lib, kw, match):
    a = {**dict(slots=P, starts=P, n=2, plan=P), **kw}
    refused(lib, lib.tq_kv_share(cache(), a["slots"], a["starts"], a["n"], a["plan"], None), match)


def test_nothing_to_do(lib):
    assert lib.tq_kv_share(cache(), None, None, 0, None, None) == 0
    assert lib.tq_kv_cross(cache(), 0, None, None, 0, None, 0, 0, 4, 512, 128, 1.0, None, None, None, 0, None) == 0
    assert lib.tq_kv_attend_shared(cache(), 0, None, None, None, 0, 0, None, 0, 0, 4, 512, 128, 1.0, None, None, None, 0, None) == 0
    assert lib.tq_sample(None, 0, 0, None, 0, 0, 10, None, None, None, None, None, None, None, 0, None) == 0


SAMPLE = dict(logits=P, type=0, ls=100, noise=P, ns=100, n=2, vocab=100, t=P, k=P, p=P, m=P, tokens=P, logprobs=P, ws=P, bytes=BIG)


@pytest.mark.parametrize("kw,match", [
    (dict(n=-1), "n="), (dict(n=65536), "n="), (dict(vocab=0), "vocab"), (dict(vocab=2 ** 24 + 1), "vocab"), (dict(type=3), "type"),
    (dict(ls=-1), "strides"), (dict(ns=2 ** 31), "strides"), (dict(logits=None), "NULL"), (dict(noise=None), "NULL"),
    (dict(tokens=None), "NULL"), (dict(logits=P + 1), "aligned"), (dict(type=2, logits=P + 2), "aligned"),
    (dict(noise=P + 2), "4-byte"), (dict(t=P + 1), "4-byte"), (dict(k=P + 1), "4-byte"), (dict(p=P + 2), "4-byte"),
    (dict(m=P + 3), "4-byte"), (dict(tokens=P + 2), "4-byte"), (dict(logprobs=P + 2), "4-byte"), (dict(ws=None), "workspace"),
    (dict(ws=P + 4), "workspace")])
def test_sample_refusals(lib, kw, match):
    a = {**SAMPLE, **kw}
    refused(lib, lib.tq_sample(a["logits"], a["type"], a["ls"], a["noise"], a["ns"], a["n"], a["vocab"], a["t"], a["k"], a["p"],
                               a["m"], a["tokens"], a["logprobs"], a["ws"], a["bytes"], None), match)


def test_workspaces_grow_with_the_call(lib):
    def need(fn, *a):
        out = C.c_size_t()
        assert getattr(lib, fn)(*a, C.byref(out)) == 0
        return out.value

    for dim in (64, 128, 256):
        c = cache(head_dim=dim, slots=65536)
        last = 0
        for n, total, heads in ((1, 1, 4), (1, 40, 4), (3, 40, 8), (40, 40, 32), (40, 4000, 32), (300, 4000, 64)):
            now = need("tq_kv_attend_shared_workspace", c, n, total, heads)
            assert now >= last
            last = now
    sizes = [need("tq_sample_workspace", n, v) for n, v in ((0, 1), (1, 1), (1, 5000), (7, 5000), (7, 300_000), (65535, 300_000))]
    assert sizes == sorted(sizes)


def test_python_refusals():
    torch = pytest.importorskip("torch")
    import paper_2607_16973_gb300 as tq
    x = torch.zeros(2, 10)
    with pytest.raises(TypeError, match="CUDA"):
        tq.sample_tokens(x, x)
    with pytest.raises(ValueError, match="vocab"):
        tq.sample_tokens(x, x[:1])
    with pytest.raises(ValueError, match="vocab"):
        tq.sample_tokens(x[0], x[0])
