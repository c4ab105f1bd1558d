"""Memory of what a call on another stream works on: buffers and caches that are
let go of while the stream still has the call in front of it keep their memory
until it is done."""
import pytest

pytestmark = pytest.mark.gpu

SLEEP = 400_000_000  # cycles, about 0.2 s: what stands in front of the call


def i32(*x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def fresh(torch, shape, dtype):
    """(address, tensor) of memory of this size class that no one else has: what is freed is what comes next."""
    a = torch.empty(shape, dtype=dtype, device="cuda").data_ptr()
    b = torch.empty(shape, dtype=dtype, device="cuda")
    assert b.data_ptr() == a
    return a, b


def busy(torch):
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(SLEEP)
    return side


def check(torch, side, made):
    """made: (address, shape, dtype) of tensors that were let go of."""
    assert not side.query()  # (the sleep is not over, or this shows nothing)
    again = [torch.empty(shape, dtype=dtype, device="cuda") for _, shape, dtype in made]
    assert not {a for a, _, _ in made} & {x.data_ptr() for x in again}
    torch.cuda.synchronize()


def test_buffers_of_attention(cuda_lib):
    import torch
    cache = cuda_lib.KVCache(8, 1, 4, 2, 64)
    cache.extend(i32(0), i32(100))
    q = torch.randn(100, 8, 64, device="cuda").to(torch.bfloat16)
    slots, starts = i32(0), i32(0, 100)
    size = cache.attention_workspace(1, 100, 8)
    shapes = [((100, 8, 64), torch.bfloat16), ((100, 8), torch.float32), ((size,), torch.uint8)]
    cache.attention(0, slots, starts, q, return_lse=True)  # (a kernel's first launch waits for the GPU)
    made = [fresh(torch, *s) for s in shapes]
    side = busy(torch)
    cache.attention(0, slots, starts, q, out=made[0][1], lse=made[1][1], workspace=made[2][1], stream=side)
    made = [(a, *s) for (a, _), s in zip(made, shapes)]
    check(torch, side, made)


def test_buffers_of_verification(cuda_lib):
    import torch
    n, t, vocab = 3, 2, 5000
    target = torch.softmax(torch.randn(n, t + 1, vocab, device="cuda"), 2)
    args = target, torch.zeros(n, t, dtype=torch.int32, device="cuda"), torch.rand(n, t, device="cuda"), \
        torch.ones(n, vocab, device="cuda")
    shapes = [((n, t + 1), torch.int32), ((n,), torch.int32), ((1 << 21,), torch.uint8)]
    cuda_lib.verify_drafts(*args)
    made = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype in shapes]
    side = busy(torch)
    cuda_lib.verify_drafts(*args, tokens=made[0], accepted=made[1], workspace=made[2], stream=side)
    gone = [(x.data_ptr(), *s) for x, s in zip(made, shapes)]
    del made
    check(torch, side, gone)


def test_a_cache(cuda_lib):
    import torch
    cache = cuda_lib.KVCache(64, 2, 40, 2, 64)
    shapes = [(tuple(x.shape), x.dtype) for x in (cache.k, cache.v, cache.k_scale, cache.table)]
    gone = [(x.data_ptr(), *s) for x, s in zip((cache.k, cache.v, cache.k_scale, cache.table), shapes)]
    slots, counts = i32(0), i32(700)
    cache.extend(slots, counts)
    cache.truncate(slots, i32(0))
    side = busy(torch)
    cache.extend(slots, counts, stream=side)
    del cache
    check(torch, side, gone)
