"""A verification's workspace chooses among the call's own rows, tokens and
words: with counters that something else has written the results are
unspecified, but lie in their ranges, and a bind puts it right."""
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [700, 40001])
@pytest.mark.parametrize("word", [1, 64, 65, 1000, 2 ** 31 - 1, -1])
def test_written_counters(vocab, word):
    dev = need_gpu()
    gen = torch.Generator(device=dev).manual_seed(vocab)
    batch, draft = 6, 5
    target = torch.randn(batch, draft + 1, vocab, generator=gen, device=dev)
    drafts = target[:, :draft].contiguous()
    tokens = torch.randint(0, vocab, (batch, draft), generator=gen, device=dev, dtype=torch.int32)
    tokens[2, 3] = 2 ** 31 - 1
    tokens[3, 1] = -5
    inputs = (target, drafts, tokens, torch.rand(batch, draft, generator=gen, device=dev),
              torch.empty(batch, vocab, device=dev).exponential_(generator=gen))
    length = torch.tensor([5, 0, 5, 3, 1, 4], dtype=torch.int32, device=dev)
    plan = tk.VerifyPlan(batch, draft, vocab, dtype=torch.float32)
    want = [w.clone() for w in plan.execute(*inputs, length=length)]
    (ws,) = plan._ws.values()
    announce(f"verify with counters at {word}, {vocab} words")
    ws.view(torch.int32).fill_(word)
    accepted = torch.full((batch,), -2, dtype=torch.int32, device=dev)
    out = torch.full((batch, draft + 1), -2, dtype=torch.int32, device=dev)
    plan.execute(*inputs, length=length, accepted_out=accepted, tokens_out=out)
    torch.cuda.synchronize()
    assert bool(((accepted == -2) | ((accepted >= 0) & (accepted <= length))).all())
    given = torch.nn.functional.pad(tokens, (0, 1), value=-1)
    assert bool(((out == given) | ((out >= -2) & (out < vocab))).all())
    plan._ready(ws, None)
    got = plan.execute(*inputs, length=length)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
