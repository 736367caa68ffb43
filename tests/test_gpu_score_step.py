"""Scores and embedding run together, as a training step uses them: lookup, readout (a torch
product), log-probability and entropy, the gradient of the logits, of the embedding, dense into
sparsification and as a list into the update; eagerly, captured, and on another stream."""
import numpy as np
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, check_selection, need_gpu
from oracle import score as oracle
from rows_common import EPS, STORE
from test_gpu_embed import bits_of, close, some_tokens
from test_gpu_score import check_gradient, check_scores

pytestmark = pytest.mark.gpu


class Step:
    def __init__(self, n, vocab, width, seed):
        dev = need_gpu()
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.n, self.vocab, self.width = n, vocab, width
        self.table = torch.randn(vocab, width, generator=gen, device=dev)
        self.readout = torch.randn(width, vocab, generator=gen, device=dev)
        self.tokens = torch.zeros(n, dtype=torch.int32, device=dev)
        self.targets = torch.zeros(n, dtype=torch.int32, device=dev)
        self.dlogp, self.dentropy = torch.zeros(n, device=dev), torch.zeros(n, device=dev)
        self.grad = torch.zeros(vocab, width, device=dev)
        self.embed = tk.EmbedPlan(n, vocab, width, scale=0.25)
        self.score = tk.ScorePlan(n, vocab, 5, dtype=torch.float32)
        stride = self.embed.most(n)
        self.idx = torch.zeros(1, stride, dtype=torch.int32, device=dev)
        self.val = torch.zeros(1, stride, device=dev)
        self.nnz = torch.zeros(1, dtype=torch.int32, device=dev)

    def new_inputs(self, rng):
        kinds = ["law", "uniform", "one", "few"]
        self.tokens.copy_(torch.as_tensor(
            some_tokens(rng, kinds[rng.integers(4)], self.n, self.vocab).astype(np.int32)))
        self.targets.copy_(torch.as_tensor(
            rng.integers(-1, self.vocab, self.n).astype(np.int32)))
        self.dlogp.copy_(torch.as_tensor(rng.normal(size=self.n)))
        self.dentropy.copy_(torch.as_tensor(rng.normal(size=self.n) * 0.1))

    def run(self, stream=None):
        x = self.embed.forward(self.table, self.tokens, stream=stream)
        with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(
                torch.cuda.current_stream()):
            z = x @ self.readout
        logp, entropy, stats = self.score.forward(z, self.targets, stream=stream)
        best = self.score.execute(z, self.targets, stream=stream)
        dz = self.score.backward(z, self.targets, stats, dlogp=self.dlogp,
                                 dentropy=self.dentropy, stream=stream)
        with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(
                torch.cuda.current_stream()):
            dx = dz @ self.readout.t()
        self.embed.backward(self.tokens, dx, grad_out=self.grad, stream=stream)
        tied = self.embed.backward(self.tokens, dx, add=self.table, stream=stream)
        self.embed.lists(self.tokens, dx, idx_out=self.idx[0], val_out=self.val[0],
                         nnz_out=self.nnz, stream=stream)
        return [x, z, logp, entropy, *best, dz, dx, self.grad, tied, self.nnz, self.idx, self.val]


def test_a_step_against_the_oracle():
    """Each operator on what the one before it gave."""
    rng = np.random.default_rng(31)
    s = Step(150, 700, 48, 31)
    announce("a step of scores and embedding")
    sparsify = tk.SparsifyPlan([s.grad.numel()], rho=0.02)
    residual = torch.zeros_like(s.grad)
    sparsify.bind([s.grad], [residual])
    for _ in range(3):
        s.new_inputs(rng)
        x, z, logp, entropy, _, _, words, _, dz, dx, grad, tied, nnz, idx, val = s.run()
        tokens, targets = s.tokens.cpu().numpy(), s.targets.cpu().numpy()
        rows = torch.where((s.tokens >= 0)[:, None], s.table[s.tokens.long().clamp(min=0)], 0.0)
        assert torch.equal(x, rows * 0.25)
        zs = z.double().cpu().numpy()
        scores = (logp.double().cpu().numpy(), entropy.double().cpu().numpy())
        g = dz.double().cpu().numpy()
        for r in range(s.n):
            want = oracle.score(zs[r], int(targets[r]), 5)
            check_scores((scores[0][r], scores[1][r]), zs[r], want, 1.0)
            assert (words[r].cpu().numpy() == want.words).all()
            check_gradient(g[r], zs[r], int(targets[r]), float(s.dlogp[r]), float(s.dentropy[r]),
                           1.0, "f32")
        want, size, counts = oracle.embed_sums(tokens, dx.double().cpu().numpy(), s.vocab, 0.25)
        close(grad.double().cpu().numpy(), want, size, counts, STORE["f32"])
        close(tied.double().cpu().numpy(), want, size, counts, STORE["f32"],
              add=s.table.double().cpu().numpy())
        # the list holds the dense gradient's rows, bit for bit
        m = int(nnz.item())
        assert m == int((counts > 0).sum()) * s.width
        assert torch.equal(grad.view(-1)[idx[0, :m].long()], val[0, :m])
        # the dense gradient is what sparsification takes
        before = (s.grad + residual).view(-1).cpu().numpy()
        sent, value = sparsify.execute()
        check_selection(before, sent.cpu().numpy(), value.cpu().numpy(),
                        residual.view(-1).cpu().numpy(), sparsify.k_total)


def equal(a, b):
    return all(torch.equal(bits_of(x), bits_of(y)) for x, y in zip(a, b))


@pytest.mark.parametrize("n,vocab,width", [(40, 5003, 24), (3, 40001, 8), (700, 900, 515)])
def test_captured_steps_replay(n, vocab, width):
    """Two graphs of one set of plans, captured without an eager call on their stream, replayed
    with new inputs between eager calls and at the same time; each replay gives what eager
    calls give, bit for bit."""
    rng = np.random.default_rng(vocab)
    steps = [Step(n, vocab, width, 1), Step(n, vocab, width, 2)]
    steps[1].embed, steps[1].score = steps[0].embed, steps[0].score
    announce(f"captured steps {n} {vocab} {width}")
    for s in steps:
        s.new_inputs(rng)
        s.run()             # (torch's own product wants an eager call before its capture)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in steps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(s.run())
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        want = []
        for s in steps:
            s.new_inputs(rng)
            s.idx.zero_()
            s.val.zero_()
            want.append([o.clone() for o in s.run()])
        torch.cuda.synchronize()
        for s in steps:
            s.idx.zero_()
            s.val.zero_()
        torch.cuda.synchronize()
        if turn % 2:
            graphs[1].replay()
            steps[0].run()
            graphs[0].replay()
        else:
            for g, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert equal(outs[i], want[i]), (turn, i)


def test_another_stream():
    rng = np.random.default_rng(33)
    s = Step(64, 3001, 40, 5)
    s.new_inputs(rng)
    torch.cuda.synchronize()
    want = [o.clone() for o in s.run()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for o in (s.grad, s.idx, s.val, s.nnz):
        o.zero_()
    side.wait_stream(torch.cuda.current_stream())
    got = s.run(stream=side)
    side.synchronize()
    assert equal(got[:13], want[:13])
    m = int(s.nnz.item())
    assert torch.equal(s.val[0, :m], want[14][0, :m]) and torch.equal(s.idx[0, :m], want[13][0, :m])


def test_a_policy_step_under_autograd():
    """Both operators as nodes of one autograd graph, against the same loss in 64 bits: a tied
    embedding, its gradient from the lookup and from the readout. Products of 32 and 300
    terms in binary32 lose at most 300 units of the sum of magnitudes each, which passes three of
    them and the scores' own (rows of 300 words: 100 units of numbers below 20)."""
    rng = np.random.default_rng(34)
    dev = need_gpu()
    vocab, width, n = 300, 32, 50
    table = (rng.normal(size=(vocab, width)) * 0.5).astype(np.float32)
    tokens = some_tokens(rng, "law", n, vocab)
    targets = rng.integers(0, vocab, n)
    advantage = rng.normal(size=n)

    w = torch.from_numpy(table).to(dev).requires_grad_()
    ep = tk.EmbedPlan(n, vocab, width, scale=2.0)
    sp = tk.ScorePlan(n, vocab, dtype=torch.float32, temperature=1.25)
    x = ep.lookup(w, torch.as_tensor(tokens, dtype=torch.int32, device=dev))
    logp, entropy = sp.score(x @ w.t(), torch.as_tensor(targets, dtype=torch.int32, device=dev))
    (-(logp * torch.as_tensor(advantage, dtype=torch.float32, device=dev)).sum()
     - 0.05 * entropy.sum()).backward()

    w64 = torch.from_numpy(table).double().requires_grad_()
    t = torch.as_tensor(tokens)
    x64 = torch.where((t >= 0)[:, None], w64[t.clamp(min=0)], 0.0) * 2.0
    lp = torch.log_softmax(x64 @ w64.t() / 1.25, 1)
    loss = -(lp[torch.arange(n), torch.as_tensor(targets)] * torch.as_tensor(advantage)).sum()
    (loss + 0.05 * (lp.exp() * lp).sum()).backward()
    scale = float(w64.grad.abs().max())
    assert (w.grad.double().cpu() - w64.grad).abs().max() <= 3 * 300 * 20 * EPS * scale
