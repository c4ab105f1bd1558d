"""Refusals of the key-value cache's calls and of draft verification: checked
before any CUDA call, so they run without a GPU."""
import ctypes as C

import numpy as np
import pytest

import kvref
import paper_2607_16973_gb300 as tq
from paper_2607_16973_gb300 import _lib
from paper_2607_16973_gb300.build import build

P = 1 << 20  # an address nothing is read from
GOOD = dict(k=P, v=P, k_scale=P, v_scale=P, table=P, lens=P, refs=P, status=P, pages=100, slots=8, max_pages=10,
            layers=2, kv_heads=4, head_dim=128, page_tokens=64, codes=0)


@pytest.fixture(scope="module")
def lib():
    build()
    return tq.load()


def cache(**kw):
    return C.byref(_lib.KvCacheStruct(**{**GOOD, **kw}))


def refused(lib, status, match):
    assert status == _lib.TQ_EINVAL, status
    assert match in lib.tq_last_error().decode(), lib.tq_last_error()


BAD_CACHES = [(dict(head_dim=96), "head_dim"), (dict(page_tokens=48), "page_tokens"), (dict(page_tokens=8), "page_tokens"),
              (dict(page_tokens=512), "page_tokens"), (dict(codes=2), "codes"), (dict(layers=0), "layers"),
              (dict(kv_heads=0), "kv_heads"), (dict(slots=0), "slots"), (dict(slots=65537), "slots"),
              (dict(pages=0), "pages"), (dict(pages=2**31 - 1), "pages"), (dict(max_pages=0), "max_pages"),
              (dict(max_pages=2**25), "max_pages"), (dict(v=None), "NULL"), (dict(status=None), "NULL"),
              (dict(k=P + 8), "16-byte"), (dict(lens=P + 2), "4-byte")]


@pytest.mark.parametrize("kw,match", BAD_CACHES)
def test_every_call_checks_the_cache(lib, kw, match):
    c, need = cache(**kw), C.c_size_t()
    refused(lib, lib.tq_kv_append(c, 0, P, P, 1, P, P, 0, 1, 512, 128, 512, 128, None), match)
    refused(lib, lib.tq_kv_attend_workspace(c, 1, 1, 4, C.byref(need)), match)
    refused(lib, lib.tq_kv_attend(c, 0, P, P, 1, P, 0, 1, 4, 512, 128, 1.0, 0, P, P, P, 1 << 40, None), match)
    refused(lib, lib.tq_kv_fork(c, P, P, 1, None), match)
    refused(lib, lib.tq_kv_extend_workspace(c, 1, C.byref(need)), match)
    refused(lib, lib.tq_kv_extend(c, P, P, 1, P, 1 << 40, None), match)
    refused(lib, lib.tq_kv_truncate(c, P, P, 1, None), match)
    refused(lib, lib.tq_kv_compact_workspace(c, C.byref(need)), match)
    refused(lib, lib.tq_kv_compact(c, P, P, 1 << 40, None), match)
    refused(lib, lib.tq_kv_check(c, None), match)


def test_null_cache(lib):
    assert lib.tq_kv_check(None, None) == _lib.TQ_EINVAL


APPEND = dict(layer=0, slots=P, starts=P, n=1, k=P, v=P, type=0, total=1, k0=512, k1=128, v0=512, v1=128)


@pytest.mark.parametrize("kw,match", [
    (dict(layer=2), "layer"), (dict(layer=-1), "layer"), (dict(n=-1), "n="), (dict(n=9), "n="), (dict(type=3), "type"),
    (dict(total=-1), "total"), (dict(total=2**31 - 1), "total"), (dict(slots=None), "NULL"), (dict(starts=P + 1), "4-byte"),
    (dict(k=None), "NULL k"), (dict(v=None), "NULL v"), (dict(k=P + 1), "k must be aligned"),
    (dict(type=2, v=P + 2), "v must be aligned"), (dict(k0=-1), "strides of k"), (dict(v1=2**31), "strides of v")])
def test_append_refusals(lib, kw, match):
    a = {**APPEND, **kw}
    refused(lib, lib.tq_kv_append(cache(), a["layer"], a["slots"], a["starts"], a["n"], a["k"], a["v"], a["type"],
                                  a["total"], a["k0"], a["k1"], a["v0"], a["v1"], None), match)


ATTEND = dict(layer=0, slots=P, starts=P, n=1, q=P, type=0, total=1, heads=8, q0=1024, q1=128, scale=1.0, window=0,
              out=P, lse=P, ws=P, bytes=1 << 40)


@pytest.mark.parametrize("kw,match", [
    (dict(layer=2), "layer"), (dict(n=9), "n="), (dict(n=0), "no sequence"), (dict(type=2), "type"), (dict(heads=6), "heads"),
    (dict(heads=0), "heads"), (dict(total=-1), "total"), (dict(scale=float("nan")), "scale"),
    (dict(scale=float("inf")), "scale"), (dict(window=-1), "window"), (dict(q=None), "NULL q"), (dict(q=P + 1), "aligned"),
    (dict(q0=-1), "strides"), (dict(out=None), "out"), (dict(out=P + 2), "out"), (dict(lse=P + 2), "lse"),
    (dict(ws=None), "workspace"), (dict(ws=P + 8), "workspace"), (dict(bytes=0), "workspace")])
def test_attend_refusals(lib, kw, match):
    a = {**ATTEND, **kw}
    refused(lib, lib.tq_kv_attend(cache(), a["layer"], a["slots"], a["starts"], a["n"], a["q"], a["type"], a["total"],
                                  a["heads"], a["q0"], a["q1"], a["scale"], a["window"], a["out"], a["lse"], a["ws"],
                                  a["bytes"], None), match)


def test_page_refusals(lib):
    c = cache()
    for call in (lib.tq_kv_fork, lib.tq_kv_truncate):
        refused(lib, call(c, P, P, 9, None), "n=")
        refused(lib, call(c, None, P, 1, None), "NULL")
        refused(lib, call(c, P, P + 2, 1, None), "4-byte")
    refused(lib, lib.tq_kv_extend(c, P, P, -1, P, 1 << 40, None), "n=")
    refused(lib, lib.tq_kv_extend(c, P, None, 1, P, 1 << 40, None), "NULL")
    refused(lib, lib.tq_kv_extend(c, P, P, 1, None, 1 << 40, None), "workspace")
    refused(lib, lib.tq_kv_extend(c, P, P, 1, P, 16, None), "needed")
    refused(lib, lib.tq_kv_extend_workspace(c, 1, None), "NULL")
    refused(lib, lib.tq_kv_compact(c, P + 1, P, 1 << 40, None), "used")
    refused(lib, lib.tq_kv_compact(c, None, P, 16, None), "needed")


def test_nothing_to_do_touches_no_gpu(lib):
    c = cache()
    assert lib.tq_kv_append(c, 0, None, None, 0, None, None, 0, 0, 0, 0, 0, 0, None) == 0
    assert lib.tq_kv_attend(c, 0, None, None, 0, None, 0, 0, 8, 0, 0, 1.0, 0, None, None, None, 0, None) == 0
    assert lib.tq_kv_fork(c, None, None, 0, None) == 0
    assert lib.tq_kv_extend(c, None, None, 0, None, 0, None) == 0
    assert lib.tq_kv_truncate(c, None, None, 0, None) == 0
    assert lib.tq_verify_drafts(None, None, 2, None, None, None, None, 0, 3, 100, None, None, None, 0, None) == 0


VERIFY = dict(target=P, draft=P, type=2, drafts=P, lens=P, uniforms=P, noise=P, n=1, t=3, vocab=100, tokens=P, accepted=P,
              ws=P, bytes=1 << 40)


@pytest.mark.parametrize("kw,match", [
    (dict(n=-1), "n="), (dict(n=65536), "n="), (dict(t=-1), "t="), (dict(t=65), "t="), (dict(vocab=0), "vocab"),
    (dict(vocab=2**24 + 1), "vocab"), (dict(type=3), "type"), (dict(target=None), "NULL"), (dict(drafts=None), "NULL"),
    (dict(uniforms=None), "NULL"), (dict(noise=None), "NULL"), (dict(tokens=None), "NULL"), (dict(accepted=None), "NULL"),
    (dict(target=P + 2), "aligned"), (dict(draft=P + 1), "aligned"), (dict(noise=P + 2), "4-byte"),
    (dict(lens=P + 1), "4-byte"), (dict(ws=None), "workspace"), (dict(ws=P + 4), "workspace"), (dict(bytes=8), "needed")])
def test_verify_refusals(lib, kw, match):
    a = {**VERIFY, **kw}
    refused(lib, lib.tq_verify_drafts(a["target"], a["draft"], a["type"], a["drafts"], a["lens"], a["uniforms"], a["noise"],
                                      a["n"], a["t"], a["vocab"], a["tokens"], a["accepted"], a["ws"], a["bytes"], None),
            match)


def test_python_checks():
    torch = pytest.importorskip("torch")
    z = lambda *s, dtype=torch.uint8: torch.zeros(s, dtype=dtype)  # noqa: E731
    i32 = torch.int32
    with pytest.raises(TypeError, match="CUDA"):
        tq.KVCache.from_tensors(z(1, 2, 1, 16, 64), z(1, 2, 1, 16, 64), z(1, 2, 1, 1, dtype=torch.float32),
                                z(1, 2, 1, 1, dtype=torch.float32), z(1, 2, dtype=i32), z(1, dtype=i32), z(2, dtype=i32))
    with pytest.raises(ValueError, match="codes"):
        tq.KVCache(2, 1, 2, 1, 64, 16, codes="int4", device="cpu")
    with pytest.raises(ValueError, match="positive"):
        tq.KVCache(2, 1, 2, 1, 64, 8, device="cpu")
    with pytest.raises(ValueError, match="k_scale"):
        tq.KVCache.from_tensors(z(1, 2, 1, 16, 64), z(1, 2, 1, 16, 64), z(1, 2), z(1, 2), z(1, 2), z(1), z(2))
    with pytest.raises(ValueError, match="drafts"):
        tq.verify_drafts(z(2, 4, 10), z(2, 2, dtype=i32), z(2, 3), z(2, 10))
    with pytest.raises(TypeError, match="CUDA"):
        tq.verify_drafts(z(2, 4, 10, dtype=torch.float32), z(2, 3, dtype=i32), z(2, 3), z(2, 10))


def test_plain_e4m3_codes():
    """The plain form's table and rounding: every code comes back, neighbours split at their middle, ties go to even."""
    finite = np.array([b for b in range(256) if b & 127 != 127], np.uint8)
    v = kvref.E4M3[finite]
    assert np.array_equal(kvref.to_codes(v, "e4m3"), finite)
    assert v.max() == 448 and np.abs(v[v != 0]).min() == 2.0 ** -9
    up = np.arange(0, 126, dtype=np.uint8)
    middle = (kvref.E4M3[up] + kvref.E4M3[up + 1]) / 2
    assert np.array_equal(kvref.to_codes(middle, "e4m3"), np.where(up % 2 == 0, up, up + 1))
    torch = pytest.importorskip("torch")
    x = torch.linspace(-448, 448, 100_001)
    assert np.array_equal(kvref.to_codes(x.numpy(), "e4m3"), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
