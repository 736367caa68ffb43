"""Scores of the most rows, and of logits beyond 2^32 elements: rows come out bit for bit as they
do in a call on few of them (at the same addresses)."""
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu
from rows_common import TYPES

pytestmark = pytest.mark.gpu


def bits_of(t):
    return t.contiguous().view(torch.int32 if t.dtype.itemsize == 4 else torch.int16)


@pytest.mark.parametrize("n,vocab,dtype,k", [
    (1 << 20, 33, "f32", 5), (1 << 20, 260, "bf16", 3), (33000, 131073, "bf16", 5),
    (17000, 262145, "f16", 3)])
def test_rows_of_a_large_call(n, vocab, dtype, k):
    announce(f"scores of {n}x{vocab} {dtype}")
    dev = need_gpu()
    gen = torch.Generator(device=dev).manual_seed(n)
    z = torch.empty(n, vocab, dtype=TYPES[dtype], device=dev)
    step = 1 << 24
    for i in range(0, z.numel(), step):
        z.view(-1)[i:i + step].normal_(0.0, 3.0, generator=gen)
    tokens = torch.randint(-1, vocab, (n,), generator=gen, device=dev, dtype=torch.int32)
    dlogp, dentropy = (torch.randn(n, generator=gen, device=dev) for _ in range(2))
    plan = tk.ScorePlan(n, vocab, k, dtype=TYPES[dtype], check=True)
    logp, entropy, idx, val = plan.execute(z, tokens)
    logp2, entropy2, stats = plan.forward(z, tokens)
    grad = plan.backward(z, tokens, stats, dlogp=dlogp, dentropy=dentropy)
    for at in (0, n // 2 - 3, n - 7):
        few = slice(at, at + 7)
        some = tk.ScorePlan(7, vocab, k, dtype=TYPES[dtype], check=True)
        want = some.execute(z[few], tokens[few])
        for a, b in zip((logp, entropy, idx, val), want):
            assert torch.equal(bits_of(a[few]), bits_of(b)), at
        l2, e2, s2 = some.forward(z[few], tokens[few])
        for a, b in zip((logp2, entropy2, stats), (l2, e2, s2)):
            assert torch.equal(bits_of(a[few]), bits_of(b)), at
        g = some.backward(z[few], tokens[few], s2, dlogp=dlogp[few], dentropy=dentropy[few])
        assert torch.equal(bits_of(grad[few]), bits_of(g)), at
    # in every row: a token among the alternatives has their log-probability, the first is the
    # greatest word, and the gradient of a row without a token is 0
    live = tokens >= 0
    hit = idx == tokens[:, None]
    assert torch.equal(val[hit & live[:, None]], logp[hit.any(1) & live])
    for i in range(0, n, 1 << 13):
        part = slice(i, i + (1 << 13))
        first = z[part].float().max(1).values
        at = idx[part, :1].long().clamp(min=0)
        assert torch.equal(z[part].float().gather(1, at)[:, 0][live[part]], first[live[part]])
        assert not bool(grad[part][~live[part]].any())
