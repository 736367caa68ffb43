"""One plan called by two host threads on one stream: a call's launches follow one
another, whichever workspace they share (stand-ins for tensors and for the library's
calls; no GPU)."""
import threading
import time

import pytest
import torch

import paper_2010_10458_amd as tk
from test_rows_devices import OnGpu, current_gpu_is_the_first  # noqa: F401 (a fixture)

INT, HALF = torch.int32, torch.float16


def top():
    p = tk.TopLogitsPlan(4, 100, 8, dtype=torch.float32)
    return p, "_execute", lambda: p.execute(
        OnGpu((4, 100)), idx_out=OnGpu((4, 8), INT), val_out=OnGpu((4, 8)), tail_out=OnGpu((4,)))


def distill(which):
    p = tk.DistillPlan(4, 100, 8, dtype=torch.float32)
    out = dict(stats_out=OnGpu((4, 4))) if which == "forward" else dict(grad_out=OnGpu((4, 100)))
    return p, "_" + which, lambda: getattr(p, which)(
        OnGpu((4, 100)), OnGpu((4, 8), INT), OnGpu((4, 8)), loss_out=OnGpu((4,)), **out)


def verify():
    p = tk.VerifyPlan(2, 3, 50, dtype=torch.float32)
    return p, "_execute", lambda: p.execute(
        OnGpu((2, 4, 50)), OnGpu((2, 3, 50)), OnGpu((2, 3), INT), OnGpu((2, 3)), OnGpu((2, 50)),
        accepted_out=OnGpu((2,), INT), tokens_out=OnGpu((2, 4), INT), logp_out=OnGpu((2, 4)))


def score(which):
    p = tk.ScorePlan(4, 100, 8, dtype=torch.float32)
    out = (dict(idx_out=OnGpu((4, 8), INT), val_out=OnGpu((4, 8))) if which == "execute"
           else dict(stats_out=OnGpu((4, 4))))
    return p, "_forward", lambda: getattr(p, which)(
        OnGpu((4, 100)), OnGpu((4,), INT), logp_out=OnGpu((4,)), entropy_out=OnGpu((4,)), **out)


def embed(which):
    p = tk.EmbedPlan(6, 20, 8, dtype=torch.float32, out_dtype=HALF)
    out = (dict(grad_out=OnGpu((20, 8))) if which == "backward" else
           dict(idx_out=OnGpu((48,), INT), val_out=OnGpu((48,)), nnz_out=OnGpu((1,), INT)))
    return p, "_" + which, lambda: getattr(p, which)(OnGpu((6,), INT), OnGpu((6, 8), HALF), **out)


CALLS = {"top": top, "distill forward": lambda: distill("forward"),
         "distill step": lambda: distill("step"), "verify": verify,
         "score execute": lambda: score("execute"), "score forward": lambda: score("forward"),
         "embed backward": lambda: embed("backward"), "embed lists": lambda: embed("lists")}


@pytest.mark.parametrize("name", CALLS)
def test_calls_of_two_threads_take_turns(name, monkeypatch):
    plan, entry, run = CALLS[name]()
    plan.ws_bytes, plan._keeps = 4096, True     # (small rows need none)
    monkeypatch.setattr(plan, "_ready", lambda ws, stream: None, raising=False)
    kept = type(plan)._workspace
    monkeypatch.setattr(plan, "_workspace", lambda stream, dev: kept(plan, stream, "cpu"),
                        raising=False)
    under_way, together = [0], [0]

    def launches(*args):
        under_way[0] += 1
        together[0] = max(together[0], under_way[0])
        time.sleep(0.05)        # (the library's calls run without the interpreter's lock)
        under_way[0] -= 1
        return tk.OK

    monkeypatch.setattr(plan, entry, launches)
    errors = []

    def worker():
        try:
            run()
        except Exception as e:      # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=worker) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(30)
    assert not errors and not any(t.is_alive() for t in threads)
    assert len(plan._ws) == 1
    assert together[0] == 1
