"""Verification of drafted tokens on the GPU against the plain form: tokens and
counts are equal, whatever way a row is split."""
import numpy as np
import pytest

import kvref

pytestmark = pytest.mark.gpu


def make(torch, n, t, vocab, type, seed, text=False):
    rng = np.random.default_rng(seed)

    def soft(x):
        x = np.exp(x - x.max(-1, keepdims=True))
        return x / x.sum(-1, keepdims=True)

    logits = rng.standard_normal((n, t + 1, vocab)) * 2
    target = torch.from_numpy(soft(logits).astype(np.float32)).to(getattr(torch, type))
    draft = None if text else torch.from_numpy(
        soft(logits[:, :t] + rng.standard_normal((n, t, vocab))).astype(np.float32)).to(getattr(torch, type))
    drafts = (logits[:, :t] if text else logits[:, :t] + rng.standard_normal((n, t, vocab))).argmax(-1).astype(np.int32)
    uniforms = rng.random((n, t), dtype=np.float32)
    if text:
        uniforms *= 0.3
    return (target, torch.from_numpy(drafts), torch.from_numpy(uniforms),
            torch.from_numpy(rng.exponential(size=(n, vocab)).astype(np.float32) + np.float32(1e-30)), draft)


def run(tq, target, drafts, uniforms, noise, draft=None, lens=None):
    d = lambda x: None if x is None else x.cuda()  # noqa: E731
    tokens, accepted = tq.verify_drafts(d(target), d(drafts), d(uniforms), d(noise), draft_probs=d(draft),
                                        draft_lens=d(lens))
    f = lambda x: None if x is None else x.float().numpy()  # noqa: E731
    want = kvref.verify(f(target), drafts.numpy(), uniforms.numpy(), noise.numpy(), f(draft),
                        None if lens is None else lens.numpy())
    assert np.array_equal(accepted.cpu().numpy(), want[1])
    assert np.array_equal(tokens.cpu().numpy(), want[0])
    return want


@pytest.mark.parametrize("type", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("text", [False, True])
@pytest.mark.parametrize("n,t,vocab", [(1, 1, 1), (1, 4, 2), (3, 5, 31), (2, 3, 2049), (40, 7, 1003), (1, 2, 50_001),
                                       (1300, 1, 65), (2, 0, 300), (2, 33, 70), (2, 64, 33)])
def test_verify(cuda_lib, type, text, n, t, vocab):
    import torch
    run(cuda_lib, *make(torch, n, t, vocab, type, n + vocab, text))


def test_lengths(cuda_lib):
    import torch
    args = make(torch, 30, 6, 500, "float32", 3, True)
    lens = torch.arange(30, dtype=torch.int32) % 7
    _, accepted = run(cuda_lib, *args, lens=lens)
    assert (accepted == lens.numpy()).any() and (accepted < lens.numpy()).any() and (accepted == 0).any()


def test_edges(cuda_lib):
    """Equal rows (nothing is left after a rejection), ties, a draft the target gives nothing, tokens out of range."""
    import torch
    n, t, vocab = 6, 2, 3000
    target = torch.zeros(n, t + 1, vocab)
    target[:, :, 10], target[:, :, 2000], target[:, :, 2999] = 0.5, 0.25, 0.25
    draft = target[:, :t].clone()
    draft[0] = 0
    draft[0, :, 5] = 1.0                                   # never accepted; all of the target is left
    drafts = torch.tensor([[5, 5], [10, 10], [7, 10], [-1, 10], [vocab, 3], [2000, 2999]], dtype=torch.int32)
    uniforms = torch.full((n, t), 0.99)
    noise = torch.ones(n, vocab)                           # equal racers: the lowest token
    noise[5, 10] = 2.0                                     # ties at 2000, 2999 and 10 itself
    tokens, accepted = run(cuda_lib, target, drafts, uniforms, noise, draft)
    assert tokens[0].tolist() == [10, -1, -1] and accepted.tolist()[:2] == [0, 2]
    assert tokens[2].tolist() == [10, -1, -1]              # p = q everywhere: the draw is from p itself
    assert tokens[5].tolist() == [2000, 2999, 10]
    run(cuda_lib, target, drafts, uniforms, noise)         # the same drafts, proposed with certainty
    one = torch.zeros(1, 2, 4)
    one[:, :, 2] = 1.0                                     # certain to be accepted: u < 1
    tokens, _ = run(cuda_lib, one, torch.tensor([[2]], dtype=torch.int32), torch.tensor([[0.9999999]]), torch.ones(1, 4))
    assert tokens[0].tolist() == [2, 2]


def test_distribution(cuda_lib):
    """Accepted drafts and draws together follow the target's row: 200,000 trials over eight tokens, each frequency
    within five standard deviations."""
    import torch
    n, vocab = 50_000, 8
    g = torch.Generator().manual_seed(5)
    p = torch.tensor([0.3, 0.05, 0.2, 0.15, 0.1, 0.1, 0.06, 0.04])
    q = torch.tensor([0.05, 0.3, 0.1, 0.15, 0.2, 0.02, 0.08, 0.1])
    counts = torch.zeros(vocab)
    for _ in range(4):
        drafts = torch.multinomial(q, n, replacement=True, generator=g).to(torch.int32)[:, None]
        tokens, _ = cuda_lib.verify_drafts(p.expand(n, 2, vocab).contiguous().cuda(), drafts.cuda(),
                                           torch.rand(n, 1, generator=g).cuda(),
                                           torch.empty(n, vocab).exponential_(generator=g).clamp_(min=1e-30).cuda(),
                                           draft_probs=q.expand(n, 1, vocab).contiguous().cuda())
        counts += torch.bincount(tokens[:, 0].cpu().long(), minlength=vocab)
    trials = 4 * n
    assert ((counts - trials * p).abs() <= 5 * (trials * p * (1 - p)).sqrt()).all()


def test_kept_buffers_and_streams(cuda_lib):
    import torch
    target, drafts, uniforms, noise, draft = (x.cuda() for x in make(torch, 5, 3, 9000, "float32", 9))
    want = cuda_lib.verify_drafts(target, drafts, uniforms, noise, draft_probs=draft)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ws = torch.full((1 << 16,), 0xFF, dtype=torch.uint8, device="cuda")
    tokens, accepted = torch.empty_like(want[0]), torch.empty_like(want[1])
    torch.cuda.synchronize()
    got = cuda_lib.verify_drafts(target, drafts, uniforms, noise, draft_probs=draft, tokens=tokens, accepted=accepted,
                                 workspace=ws, stream=side)
    side.synchronize()
    assert got[0] is tokens and torch.equal(tokens, want[0]) and torch.equal(accepted, want[1])
