"""Row operators in a HIP graph: a captured chain (top logits, distillation
step, verification) replayed with new inputs, eager work and synchronizations in
between gives what the same calls give eagerly, bit for bit."""
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,vocab,k,batch,draft", [(24, 32000, 16, 3, 4), (300, 5003, 64, 70, 6),
                                                      (5, 150001, 100, 2, 3)])
def test_replays_match_eager_calls(rows, vocab, k, batch, draft):
    dev = need_gpu()
    gen = torch.Generator(device=dev).manual_seed(vocab)

    def inputs():
        t = torch.randn(rows, vocab, generator=gen, device=dev) * 3
        z = t + torch.randn(rows, vocab, generator=gen, device=dev)
        target = torch.randn(batch, draft + 1, vocab, generator=gen, device=dev) * 3
        drafts = target[:, :draft] + torch.randn(batch, draft, vocab, generator=gen, device=dev)
        race = torch.empty(batch, draft, vocab, device=dev).exponential_(generator=gen)
        tokens = (drafts.softmax(-1) / race).argmax(-1).to(torch.int32)
        return [t, z, target, drafts, tokens, torch.rand(batch, draft, generator=gen, device=dev),
                torch.empty(batch, vocab, device=dev).exponential_(generator=gen)]

    top = tk.TopLogitsPlan(rows, vocab, k, dtype=torch.float32)
    distill = tk.DistillPlan(rows, vocab, k, dtype=torch.float32)
    verify = tk.VerifyPlan(batch, draft, vocab, dtype=torch.float32)

    def chain(x):
        idx, val, tail = top.execute(x[0])
        loss, stats = distill.forward(x[1], idx, val, tail=tail)
        back = distill.backward(x[1], idx, val, stats, tail=tail)
        step = distill.step(x[1], idx, val, tail=tail)
        return [idx, val, tail, loss, back, *step, *verify.execute(*x[2:])]

    fixed = inputs()
    announce(f"graph {rows}x{vocab}")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(fixed)   # workspaces of this stream
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = chain(fixed)
    for _ in range(4):
        new = inputs()
        want = [w.clone() for w in chain(new)]      # eager, on the ordinary stream
        for a, b in zip(fixed, new):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(captured, want)):
            assert torch.equal(a, b), i
