"""A row operator's tensors and its stream are on one GPU: others are refused
before anything is allocated or launched (stand-ins for tensors; no GPU)."""
import types

import pytest
import torch

import paper_2010_10458_amd as tk


class OnGpu:
    """What the binding looks at of a contiguous tensor on a GPU."""
    is_cuda = True

    def __init__(self, shape, dtype=torch.float32, gpu=0):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", gpu)

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def stride(self, i):
        return self.shape[i + 1:].numel()

    def get_device(self):
        return self.device.index

    def data_ptr(self):
        return 1 << 20


@pytest.fixture(autouse=True)
def current_gpu_is_the_first(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 0, raising=False)


def top(gpu=0, out=0, stream=None, status=0):
    p = tk.TopLogitsPlan(4, 100, 8, dtype=torch.float32)
    return p.execute(OnGpu((4, 100), gpu=gpu), stream=stream,
                     idx_out=OnGpu((4, 8), torch.int32, gpu), val_out=OnGpu((4, 8), gpu=out),
                     tail_out=OnGpu((4,), gpu=gpu), status=OnGpu((1,), torch.int32, status))


def distill(call, gpu=0, stream=None, **other):
    p = tk.DistillPlan(4, 100, 8, dtype=torch.float32)
    kw = dict(logits=(4, 100), idx=(4, 8), val=(4, 8), tail=(4,), count=(4,), weight=(4,))
    if call == "backward":
        kw.update(stats=(4, 4), dloss=(4,), grad_out=(4, 100))
    if call == "step":
        kw.update(loss_out=(4,), grad_out=(4, 100))
    if call == "forward":
        kw.update(loss_out=(4,), stats_out=(4, 4))
    ints = ("idx", "count")
    return getattr(p, call)(stream=stream, **{
        k: OnGpu(v, torch.int32 if k in ints else torch.float32, other.get(k, gpu))
        for k, v in kw.items()})


def verify(gpu=0, stream=None, **other):
    p = tk.VerifyPlan(2, 3, 50, dtype=torch.float32)
    kw = dict(target=(2, 4, 50), drafts=(2, 3, 50), tokens=(2, 3), uniform=(2, 3), noise=(2, 50),
              length=(2,), accepted_out=(2,), tokens_out=(2, 4), logp_out=(2, 4))
    ints = ("tokens", "length", "accepted_out", "tokens_out")
    return p.execute(stream=stream, **{
        k: OnGpu(v, torch.int32 if k in ints else torch.float32, other.get(k, gpu))
        for k, v in kw.items()})


CALLS = [top, lambda **kw: distill("forward", **kw), lambda **kw: distill("backward", **kw),
         lambda **kw: distill("step", **kw), verify]


@pytest.mark.parametrize("call", CALLS)
def test_tensors_of_another_gpu_than_the_current_one(call):
    kw = dict(out=1, status=1) if call is top else {}
    with pytest.raises(ValueError, match="cuda:1.*stream is on cuda:0"):
        call(gpu=1, **kw)


@pytest.mark.parametrize("call", CALLS)
def test_a_stream_of_another_gpu(call):
    stream = types.SimpleNamespace(device_index=1, cuda_stream=0)
    with pytest.raises(ValueError, match="cuda:0.*stream is on cuda:1"):
        call(stream=stream)


@pytest.mark.parametrize("call,names", [
    ("forward", ("idx", "val", "tail", "count", "weight", "loss_out", "stats_out")),
    ("backward", ("idx", "val", "tail", "count", "weight", "stats", "dloss", "grad_out")),
    ("step", ("idx", "val", "tail", "count", "weight", "loss_out", "grad_out"))])
def test_one_tensor_on_another_gpu(call, names):
    for name in names:
        with pytest.raises(ValueError, match=name):
            distill(call, **{name: 1})


def test_one_tensor_of_the_other_calls_on_another_gpu():
    for name in ("drafts", "tokens", "uniform", "noise", "length", "accepted_out", "tokens_out",
                 "logp_out"):
        with pytest.raises(ValueError, match=name):
            verify(**{name: 1})
    with pytest.raises(ValueError, match="val_out"):
        top(out=1)
    with pytest.raises(ValueError, match="status"):
        top(status=1)


def test_a_given_workspace_of_another_size_type_or_gpu():
    p = tk.VerifyPlan(2, 3, 50, dtype=torch.float32)
    kw = dict(target=(2, 4, 50), drafts=(2, 3, 50), tokens=(2, 3), uniform=(2, 3), noise=(2, 50),
              accepted_out=(2,), tokens_out=(2, 4), logp_out=(2, 4))
    ints = ("tokens", "accepted_out", "tokens_out")
    args = {k: OnGpu(v, torch.int32 if k in ints else torch.float32) for k, v in kw.items()}
    for bad in (OnGpu((p.ws_bytes - 1,), torch.uint8), OnGpu((p.ws_bytes,), torch.int8),
                OnGpu((p.ws_bytes,), torch.uint8, gpu=1)):
        with pytest.raises(ValueError, match="ws"):
            p.execute(ws=bad, **args)


def test_no_workspace_is_readied_in_a_capture(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="before the capture"):
        tk.VerifyPlan(2, 3, 50, dtype=torch.float32).workspace()
