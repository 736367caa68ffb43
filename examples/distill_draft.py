"""Distils a small draft model from a teacher with top-k sparsified gradients,
and measures it by how many of its drafted tokens the teacher accepts.

Teacher and student are linear readouts of the same hidden states (the student
sees the first few coordinates only). One training step is

  teacher logits -> TopLogitsPlan   (idx, val) lists and the others' log-mass
  student logits -> DistillPlan     loss and gradient of the logits
  readout gradient -> SparsifyPlan  exact top-k with error feedback
                   -> UpdatePlan    momentum SGD on the sent entries

and every few steps the student drafts tokens that VerifyPlan checks against
the teacher. Run: python examples/distill_draft.py
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2010_10458_amd as tk  # noqa: E402


def acceptance(teacher, student, hidden, narrow, draft, gen):
    """Mean number of accepted tokens of `draft`, over the sequences that the
    hidden states make in groups of draft + 1."""
    dev, words = hidden.device, teacher.shape[1]
    batch = hidden.shape[0] // (draft + 1)
    h = hidden[: batch * (draft + 1)]
    target = (h @ teacher).to(torch.bfloat16).view(batch, draft + 1, words)
    drafts = (h[:, :narrow] @ student).to(torch.bfloat16).view(batch, draft + 1, words)[:, :draft]
    race = torch.empty(batch, draft, words, device=dev).exponential_(generator=gen)
    tokens = (drafts.float().softmax(-1) / race).argmax(-1).to(torch.int32)
    plan = tk.VerifyPlan(batch, draft, words, dtype=torch.bfloat16, check=True)
    accepted, _, _ = plan.execute(
        target, drafts, tokens, torch.rand(batch, draft, generator=gen, device=dev),
        torch.empty(batch, words, device=dev).exponential_(generator=gen))
    return accepted.float().mean().item()


def train(steps=200, rows=512, words=4096, wide=64, narrow=56, k=64, rho=0.05, temperature=2.0,
          lr=1e-2, draft=4, seed=0, report=print):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    teacher = torch.randn(wide, words, generator=gen, device=dev) * (3.0 / wide ** 0.5)
    student = torch.zeros(narrow, words, device=dev)
    momentum, residual = torch.zeros_like(student), torch.zeros_like(student)
    grad = torch.empty_like(student)

    top = tk.TopLogitsPlan(rows, words, k, dtype=torch.bfloat16, temperature=temperature,
                           val_dtype=torch.float16)
    distill = tk.DistillPlan(rows, words, k, dtype=torch.bfloat16, temperature=temperature,
                             val_dtype=torch.float16)
    sparsify = tk.SparsifyPlan([student.numel()], rho=rho).bind([grad], [residual])
    update = tk.UpdatePlan([student.numel()], P=1, stride=sparsify.k_total)
    update.bind([student], [momentum])

    test = torch.randn(rows, wide, generator=gen, device=dev)
    losses, accepted = [], [acceptance(teacher, student, test, narrow, draft, gen)]
    for step in range(steps):
        hidden = torch.randn(rows, wide, generator=gen, device=dev)
        idx, val, tail = top.execute((hidden @ teacher).to(torch.bfloat16))
        logits = (hidden[:, :narrow] @ student).to(torch.bfloat16)
        loss, d_logits = distill.step(logits, idx, val, tail=tail, grad_out=logits)
        grad.copy_(hidden[:, :narrow].t() @ d_logits.float())
        sent, value = sparsify.execute()
        update.execute(sent, value, lr=lr, mu=0.9)
        losses.append(loss.mean().item())
        if (step + 1) % 50 == 0 or step + 1 == steps:
            accepted.append(acceptance(teacher, student, test, narrow, draft, gen))
            report(f"step {step + 1}: loss {losses[-1]:.4f}, accepted {accepted[-1]:.2f} of {draft}")
    return losses, accepted


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--words", type=int, default=4096)
    ap.add_argument("--rho", type=float, default=0.05)
    a = ap.parse_args()
    train(steps=a.steps, words=a.words, rho=a.rho)
