"""A cache of sizes that the library does not take is refused when it is made, before its memory is taken."""
import pytest

import paper_2607_16973_gb300 as tq
from paper_2607_16973_gb300.build import build

GOOD = dict(pages=1 << 30, slots=8, max_pages=10, kv_heads=8, head_dim=128, page_tokens=64)  # (128 TB: not to be allocated)


@pytest.mark.parametrize("kw,match", [
    (dict(head_dim=96), "head_dim"), (dict(head_dim=512), "head_dim"), (dict(page_tokens=48), "page_tokens"),
    (dict(page_tokens=512), "page_tokens"), (dict(kv_heads=1025), "kv_heads"), (dict(layers=1025), "layers"),
    (dict(slots=65537), "slots"), (dict(pages=2**31 - 1), "pages"), (dict(max_pages=2**25), "max_pages")])
def test_sizes(kw, match):
    pytest.importorskip("torch")
    build()
    with pytest.raises(tq.TQError, match=match) as e:
        tq.KVCache(**{**GOOD, **kw}, device="cpu")
    assert "TQ_EINVAL" in str(e.value)


def test_codes():
    pytest.importorskip("torch")
    with pytest.raises(ValueError, match="codes"):
        tq.KVCache(**GOOD, codes="int4", device="cpu")


@pytest.mark.gpu
def test_given_tensors(cuda_lib):
    import torch
    z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    u8, f32 = torch.uint8, torch.float32
    for page, dim, match in ((48, 64, "page_tokens"), (16, 96, "head_dim")):
        with pytest.raises(cuda_lib.TQError, match=match):
            cuda_lib.KVCache.from_tensors(z(1, 2, 1, page, dim, dtype=u8), z(1, 2, 1, page, dim, dtype=u8),
                                          z(1, 2, 1, page // 16, dtype=f32), z(1, 2, 1, page // 16, dtype=f32), z(1, 2),
                                          z(1), z(2))
