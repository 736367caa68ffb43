"""Graphs of row operators that were captured without an eager call on the
capture stream: each has its own cleared workspace, whatever is replayed first,
between or at the same time."""
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu

pytestmark = pytest.mark.gpu


def same(got, want):
    return all(torch.equal(a, b) for a, b in zip(got, want))


def verify_inputs(gen, batch, draft, vocab):
    dev = need_gpu()
    target = torch.randn(batch, draft + 1, vocab, generator=gen, device=dev) * 3
    drafts = target[:, :draft] + torch.randn(batch, draft, vocab, generator=gen, device=dev)
    race = torch.empty(batch, draft, vocab, device=dev).exponential_(generator=gen)
    tokens = (drafts.softmax(-1) / race).argmax(-1).to(torch.int32)
    return [target, drafts, tokens, torch.rand(batch, draft, generator=gen, device=dev),
            torch.empty(batch, vocab, device=dev).exponential_(generator=gen)]


@pytest.mark.parametrize("vocab", [5003, 40001])
def test_two_graphs_of_one_verification_plan(vocab):
    dev = need_gpu()
    gen = torch.Generator(device=dev).manual_seed(vocab)
    draft = 4
    plan = tk.VerifyPlan(40, draft, vocab, dtype=torch.float32)
    fixed = {b: verify_inputs(gen, b, draft, vocab) for b in (40, 3)}
    announce(f"two graphs of one verification plan, {vocab} words")
    plan.execute(*fixed[3])        # eager, on the ordinary stream; the captures use another
    torch.cuda.synchronize()
    graphs, outs = {}, {}
    for b in (40, 3):              # both on torch's own capture stream
        graphs[b] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[b]):
            outs[b] = plan.execute(*fixed[b])
    streams = {b: torch.cuda.Stream() for b in graphs}
    for turn in range(4):
        want = {}
        for b in (40, 3):
            for a, x in zip(fixed[b], verify_inputs(gen, b, draft, vocab)):
                a.copy_(x)
            want[b] = [w.clone() for w in plan.execute(*fixed[b])]
        torch.cuda.synchronize()
        for b in (3, 40):          # the one that was captured last first
            graphs[b].replay()
            if turn % 2:
                plan.execute(*fixed[40])
            torch.cuda.synchronize()
            assert same(outs[b], want[b]), (turn, b)
            for o in outs[b]:
                o.zero_()
        torch.cuda.synchronize()
        for _ in range(3):         # both at the same time
            for b in (40, 3):
                with torch.cuda.stream(streams[b]):
                    graphs[b].replay()
        torch.cuda.synchronize()
        for b in (40, 3):
            assert same(outs[b], want[b]), (turn, b)


def test_two_graphs_of_plans_over_long_rows():
    """Selections in parts and losses in chunks: their scratch is the graph's own."""
    dev = need_gpu()
    gen = torch.Generator(device=dev).manual_seed(5)
    vocab, k = 140001, 100
    announce("two graphs over long rows")
    top = tk.TopLogitsPlan(24, vocab, k, dtype=torch.float32)
    distill = tk.DistillPlan(24, vocab, k, dtype=torch.float32)

    def chain(t, z):
        idx, val, tail = top.execute(t)
        loss, stats = distill.forward(z, idx, val, tail=tail)
        return [idx, val, tail, loss, stats, *distill.step(z, idx, val, tail=tail)]

    def inputs(n):
        t = torch.randn(n, vocab, generator=gen, device=dev) * 3
        return [t, t + torch.randn(n, vocab, generator=gen, device=dev)]

    fixed = {n: inputs(n) for n in (24, 5)}
    chain(*fixed[5])
    torch.cuda.synchronize()
    graphs, outs = {}, {}
    for n in fixed:
        graphs[n] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[n]):
            outs[n] = chain(*fixed[n])
    streams = {n: torch.cuda.Stream() for n in graphs}
    for _ in range(3):
        want = {}
        for n in fixed:
            for a, x in zip(fixed[n], inputs(n)):
                a.copy_(x)
            want[n] = [w.clone() for w in chain(*fixed[n])]
        torch.cuda.synchronize()
        for n in (5, 24):
            with torch.cuda.stream(streams[n]):
                graphs[n].replay()
        torch.cuda.synchronize()
        for n in fixed:
            assert same(outs[n], want[n]), n


def test_graphs_with_workspaces_given():
    """A workspace that was readied before the capture serves its graph's replays,
    each of which leaves it ready; two such graphs run at the same time."""
    dev = need_gpu()
    gen = torch.Generator(device=dev).manual_seed(8)
    draft, vocab = 3, 32000
    plan = tk.VerifyPlan(24, draft, vocab, dtype=torch.float32)
    fixed = {b: verify_inputs(gen, b, draft, vocab) for b in (24, 2)}
    announce("graphs with workspaces given")
    plan.execute(*fixed[24])
    ws = {b: plan.workspace() for b in fixed}
    assert ws[24].data_ptr() != ws[2].data_ptr()
    torch.cuda.synchronize()
    graphs, outs, streams = {}, {}, {}
    for b in fixed:
        graphs[b], streams[b] = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graphs[b]):
            outs[b] = plan.execute(*fixed[b], ws=ws[b])
    for _ in range(4):
        want = {}
        for b in fixed:
            for a, x in zip(fixed[b], verify_inputs(gen, b, draft, vocab)):
                a.copy_(x)
            want[b] = [w.clone() for w in plan.execute(*fixed[b])]
            assert same(plan.execute(*fixed[b], ws=ws[b]), want[b])
        torch.cuda.synchronize()
        for _ in range(3):
            for b in fixed:
                with torch.cuda.stream(streams[b]):
                    graphs[b].replay()
        torch.cuda.synchronize()
        for b in fixed:
            assert same(outs[b], want[b]), b
