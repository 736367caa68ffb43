"""The row operators' Python binding on the CPU: what it keeps between calls
and which tensors it takes (no call here reaches the GPU)."""
import pytest
import torch

import paper_2010_10458_amd as tk


@pytest.fixture
def capturing(monkeypatch):
    """Whether the current stream is being captured, as the binding sees it."""
    state = [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state[0])
    return state


def test_captured_calls_have_readied_workspaces_of_their_own(capturing, monkeypatch):
    """What is recorded has not run: a workspace that a capture made must not
    serve any other call, and each captured call records its own clearing."""
    plan = tk.VerifyPlan(4, 3, 500, dtype=torch.float16)
    cleared = []
    monkeypatch.setattr(plan, "_ready", lambda ws, stream: cleared.append((ws, stream)))
    capturing[0] = True
    first, second = plan._workspace(7, "cpu"), plan._workspace(7, "cpu")
    assert [c[1] for c in cleared] == [7, 7]
    assert cleared[0][0] is first and cleared[1][0] is second and first is not second
    capturing[0] = False
    eager = plan._workspace(7, "cpu")
    assert len(cleared) == 3 and cleared[2][0] is eager
    assert eager is not first and eager is not second
    assert plan._workspace(7, "cpu") is eager and len(cleared) == 3
    # an eager workspace of the same stream does not serve a capture either
    capturing[0] = True
    assert plan._workspace(7, "cpu") is not eager and len(cleared) == 4


@pytest.mark.parametrize("make", [
    lambda: tk.TopLogitsPlan(8, 200_000, 64, dtype=torch.float32),
    lambda: tk.DistillPlan(8, 200_000, 64, dtype=torch.float32)])
def test_captured_calls_of_long_rows_share_no_scratch(capturing, make):
    plan = make()
    assert plan.ws_bytes > 0
    eager = plan._workspace(7, "cpu")
    capturing[0] = True
    first, second = plan._workspace(7, "cpu"), plan._workspace(7, "cpu")
    assert len({t.data_ptr() for t in (eager, first, second)}) == 3
