"""Operators on rows of logits over a vocabulary (include/tkef.h, "Rows of
logits"): a teacher's top logits as (idx, val) lists, distillation on such
lists, verification of drafted tokens, scores of given tokens. Like the rest of the
package this module only marshals arguments; the computation runs in the library's HIP
kernels.

    top = TopLogitsPlan(rows, vocab, k, dtype=torch.bfloat16, temperature=2.0)
    idx, val, tail = top.execute(teacher_logits)

    dp = DistillPlan(rows, vocab, k, dtype=torch.bfloat16, temperature=2.0)
    loss, grad = dp.step(student_logits, idx, val, tail=tail)      # or .loss() under autograd

    vp = VerifyPlan(batch, draft, vocab, dtype=torch.bfloat16)
    accepted, tokens, logp = vp.execute(target_logits, draft_logits, drafted, uniform, noise)

    sp = ScorePlan(rows, vocab, k=5, dtype=torch.bfloat16)
    logp, entropy, words, word_logp = sp.execute(logits, tokens)
    logp, entropy, stats = sp.forward(logits, tokens)              # or .score() under autograd
    grad = sp.backward(logits, tokens, stats, dlogp=dlogp, dentropy=dentropy)

A call's tensors are all on one GPU, that of the stream it runs on (the current
one, or the caller's `stream`).

Every call can be captured into a graph, with or without an eager call before
it. A captured call has a workspace of its own in the graph's memory, so graphs
of one plan may be replayed in any order, between eager calls, and at the same
time on several streams (graphs that were told to share one memory pool: as
that pool allows). Host threads may share a plan: its calls take turns.
"""
from __future__ import annotations

import ctypes
import threading
from typing import Optional, Tuple

import torch

from . import _check, _new_status, _raise_on_status, _val_format, lib

DTYPE_F32, DTYPE_F16, DTYPE_BF16 = 0, 1, 2
ROWS_MAX_ROWS = ROWS_MAX_VOCAB = 1 << 20
ROWS_MAX_K = 1024
SCORE_MAX_K = 64
VERIFY_MAX_DRAFT = 63
VERIFY_MAX_BATCH = 32768

_DTYPES = {torch.float32: DTYPE_F32, torch.float16: DTYPE_F16, torch.bfloat16: DTYPE_BF16}


def _dtype_code(dtype) -> int:
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError("logits are float32, float16 or bfloat16")
    return code


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return t.data_ptr() if t is not None else None


def _check_vector(t: Optional[torch.Tensor], n: int, dtype, what: str, gpu: int) -> None:
    """(get_device: 0.05 us less than a comparison of devices, which a small call
    makes six times)"""
    if t is not None and (t.dtype is not dtype or t.numel() != n or t.get_device() != gpu
                          or not t.is_contiguous()):
        raise ValueError(f"{what}: expected {n} contiguous {dtype} values on cuda:{gpu}")


def _launch_on(gpu: int, stream) -> Optional[int]:
    """Handle of the stream that a call on tensors of a GPU launches on: the
    caller's, or the current one."""
    if stream is not None:
        index, handle = stream.device_index, stream.cuda_stream
    else:
        # (0.4 us without building a Stream object)
        index = torch.cuda.current_device()
        handle = torch._C._cuda_getCurrentRawStream(index)
    if index != gpu:
        raise ValueError(f"the tensors are on cuda:{gpu}, the call's stream is on cuda:{index}")
    return handle or None


class _RowPlan:
    _destroy = ""
    _readied = False  # whether a workspace has to be readied
    _small = 1 << 20  # bytes of scratch that a plan keeps for a stream's later calls

    def __init__(self, rows: int, vocab: int, dtype, temperature: float, check: bool):
        self.rows, self.vocab = int(rows), int(vocab)
        self.dtype, self.temperature, self.check = dtype, float(temperature), bool(check)
        self._h = ctypes.c_void_p()
        self._free = getattr(lib(), self._destroy)
        self._ws = {}  # kept ones, one per stream: calls on two streams do not share one
        # From the choice of a workspace to the last launch that uses it: two threads on one
        # stream share its workspace, and the library's calls run without the interpreter's
        # lock, so the launches of one would come between those of the other.
        self._turn = threading.RLock()

    def __del__(self):
        if getattr(self, "_h", None) and self._h.value:
            self._free(self._h)
            self._h.value = None

    def _info(self, name: str) -> None:
        ws = ctypes.c_size_t()
        _check(name, getattr(lib(), name)(self._h, ctypes.byref(ws)))
        self.ws_bytes = ws.value
        self._keeps = self._readied or self.ws_bytes <= self._small

    def _workspace(self, stream: Optional[int], dev) -> Optional[torch.Tensor]:
        """The workspace of one call, on the current stream (the caller holds it
        until the call's launches are issued).

        One that is small, or has to be readied, is kept for the stream's later
        calls. Others are asked for at each call and are torch's again after it, in the
        stream's order: the lists of long rows can take as much memory as their
        logits. (A loss of a few long rows takes 0.5 us less with kept scratch.)

        A captured call gets one of its own from the graph's memory, and what
        readies it is recorded in front of the call: the graph then depends neither
        on work that ran, or did not, before its replay, nor on what other graphs and
        eager calls leave in a workspace of the plan. It is not kept for later
        calls, since nothing that is captured has run."""
        if not self.ws_bytes:
            return None
        if not self._keeps:
            return torch.empty_strided((self.ws_bytes,), (1,), dtype=torch.uint8, device=dev)
        # (the default stream cannot be captured; asking takes 0.4 us)
        captured = stream is not None and torch.cuda.is_current_stream_capturing()
        ws = None if captured else self._ws.get((stream, dev))
        if ws is None:
            ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
            self._ready(ws, stream)
            if not captured:
                self._ws[(stream, dev)] = ws
        return ws

    def _ready(self, ws: torch.Tensor, stream: Optional[int]) -> None:
        """Readies a new workspace on the stream that will use it (asynchronous)."""

    def _logits(self, x: torch.Tensor, what: str) -> Tuple[int, int]:
        """(rows, row stride) of a 2-D tensor of the plan's type whose rows are
        contiguous."""
        if x.dim() != 2 or x.dtype != self.dtype or not x.is_cuda:
            raise ValueError(f"{what}: expected a 2-D CUDA tensor of {self.dtype}")
        n, vocab = x.shape
        if vocab != self.vocab or n > self.rows:
            raise ValueError(f"{what}: the plan takes up to {self.rows} rows of {self.vocab}")
        if vocab > 1 and x.stride(1) != 1:
            raise ValueError(f"{what}: the words of a row must be contiguous")
        return n, (x.stride(0) if n > 1 else vocab)

    def _grad(self, logits, grad_out):
        if grad_out is None:
            grad_out = _out(None, tuple(logits.shape), self.dtype, logits.device, "grad_out")
            return grad_out, self.vocab
        elif grad_out.shape != logits.shape or grad_out.device != logits.device:
            raise ValueError("grad_out: expected the shape and device of the logits")
        return grad_out, self._logits(grad_out, "grad_out")[1]

    def _status_of(self, status, dev):
        if status is None:
            return (_new_status(dev), True) if self.check else (None, False)
        if status.dtype not in (torch.int32, torch.uint32) or status.numel() < 1 \
                or not status.is_cuda or status.device != dev:
            raise ValueError(f"status: expected an int32 CUDA tensor on {dev}")
        return status, False


def _on(stream):
    """Allocations of a call on `stream` come from that stream."""
    return torch.cuda.stream(stream) if stream is not None else _HERE


class _Here:
    def __enter__(self):
        return None

    def __exit__(self, *a):
        return None


_HERE = _Here()


def _out(t: Optional[torch.Tensor], shape: Tuple[int, ...], dtype, dev, what: str):
    """The caller's output, checked, or a new one (empty_strided: the cheapest of
    torch's allocating calls, 1.3 against 1.6 us, and a small call waits for three)."""
    if t is None:
        if len(shape) == 1:
            return torch.empty_strided(shape, (1,), dtype=dtype, device=dev)
        return torch.empty_strided(shape, (shape[1], 1), dtype=dtype, device=dev)
    n = 1
    for d in shape:
        n *= d
    _check_vector(t, n, dtype, what, dev.index)
    return t


class TopLogitsPlan(_RowPlan):
    """Each row's k greatest logits, as lists with ascending words, and the
    log-mass of the others (tkef_top_execute)."""

    _destroy = "tkef_top_plan_destroy"

    def __init__(self, rows: int, vocab: int, k: int, dtype=torch.bfloat16,
                 temperature: float = 1.0, val_dtype=torch.float32, check: bool = False):
        """rows: the most rows a call gives. check=True: every execute without
        a caller status word uses its own, synchronizes and raises
        TkefStatusError on any status bit."""
        super().__init__(rows, vocab, dtype, temperature, check)
        self.k, self.val_dtype = int(k), val_dtype
        _check("tkef_top_plan_create", lib().tkef_top_plan_create(
            self.rows, self.vocab, self.k, _dtype_code(dtype), _val_format(val_dtype),
            self.temperature, ctypes.byref(self._h)))
        self._info("tkef_top_plan_info")
        self._execute = lib().tkef_top_execute

    def execute(self, logits: torch.Tensor, idx_out: Optional[torch.Tensor] = None,
                val_out: Optional[torch.Tensor] = None,
                tail_out: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None, stream=None
                ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """Returns idx (n, k) int32, val (n, k) of val_dtype, tail (n,) float32."""
        n, ld = self._logits(logits, "logits")
        dev = logits.device
        h = _launch_on(dev.index, stream)
        with _on(stream):
            idx_out = _out(idx_out, (n, self.k), torch.int32, dev, "idx_out")
            val_out = _out(val_out, (n, self.k), self.val_dtype, dev, "val_out")
            tail_out = _out(tail_out, (n,), torch.float32, dev, "tail_out")
            status, own = self._status_of(status, dev)
            with self._turn:
                ws = self._workspace(h, dev)
                rc = self._execute(
                    self._h, logits.data_ptr(), ld, n, idx_out.data_ptr(), val_out.data_ptr(),
                    tail_out.data_ptr(), _ptr(ws), self.ws_bytes, _ptr(status), h)
        if rc:
            _check("tkef_top_execute", rc)
        if own:
            _raise_on_status("tkef_top_execute", status, stream)
        return idx_out, val_out, tail_out


class DistillPlan(_RowPlan):
    """Distillation of student logits on a teacher's top-logit lists
    (tkef_distill_forward / _backward / _step): the loss of each row and its
    gradient. Every call takes the lists idx (n, k) int32 ascending and val
    (n, k) of val_dtype, and optionally, one value per row: tail (float32, the
    log-mass of the teacher's other words), count (int32, used entries of a
    list) and weight (float32)."""

    _destroy = "tkef_distill_plan_destroy"

    def __init__(self, rows: int, vocab: int, k: int, dtype=torch.bfloat16,
                 temperature: float = 1.0, val_dtype=torch.float32, check: bool = False):
        super().__init__(rows, vocab, dtype, temperature, check)
        self.k, self.val_dtype = int(k), val_dtype
        _check("tkef_distill_plan_create", lib().tkef_distill_plan_create(
            self.rows, self.vocab, self.k, _dtype_code(dtype), _val_format(val_dtype),
            self.temperature, ctypes.byref(self._h)))
        self._info("tkef_distill_plan_info")
        L = lib()
        self._forward, self._backward, self._step = (
            L.tkef_distill_forward, L.tkef_distill_backward, L.tkef_distill_step)

    def _lists(self, n, idx, val, tail, count, weight, gpu):
        _check_vector(idx, n * self.k, torch.int32, "idx", gpu)
        _check_vector(val, n * self.k, self.val_dtype, "val", gpu)
        _check_vector(tail, n, torch.float32, "tail", gpu)
        _check_vector(count, n, torch.int32, "count", gpu)
        _check_vector(weight, n, torch.float32, "weight", gpu)
        return (idx.data_ptr(), val.data_ptr(), _ptr(tail), _ptr(count), _ptr(weight))

    def forward(self, logits: torch.Tensor, idx: torch.Tensor, val: torch.Tensor,
                tail: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
                weight: Optional[torch.Tensor] = None, loss_out: Optional[torch.Tensor] = None,
                stats_out: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None, stream=None
                ) -> Tuple[torch.Tensor, torch.Tensor]:
        """Returns loss (n,) float32 and stats (n, 4) float32, which backward takes."""
        n, ld = self._logits(logits, "logits")
        dev = logits.device
        lists = self._lists(n, idx, val, tail, count, weight, dev.index)
        h = _launch_on(dev.index, stream)
        with _on(stream):
            loss_out = _out(loss_out, (n,), torch.float32, dev, "loss_out")
            stats_out = _out(stats_out, (n, 4), torch.float32, dev, "stats_out")
            status, own = self._status_of(status, dev)
            with self._turn:
                ws = self._workspace(h, dev)
                rc = self._forward(
                    self._h, logits.data_ptr(), ld, n, *lists, loss_out.data_ptr(),
                    stats_out.data_ptr(), _ptr(ws), self.ws_bytes, _ptr(status), h)
        if rc:
            _check("tkef_distill_forward", rc)
        if own:
            _raise_on_status("tkef_distill_forward", status, stream)
        return loss_out, stats_out

    def backward(self, logits: torch.Tensor, idx: torch.Tensor, val: torch.Tensor,
                 stats: torch.Tensor, tail: Optional[torch.Tensor] = None,
                 count: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                 dloss: Optional[torch.Tensor] = None, grad_out: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Gradient of sum(dloss * loss) (dloss (n,) float32, default 1) in the
        logits' type. grad_out may be the logits themselves."""
        n, ld = self._logits(logits, "logits")
        dev = logits.device
        lists = self._lists(n, idx, val, tail, count, weight, dev.index)
        _check_vector(stats, n * 4, torch.float32, "stats", dev.index)
        _check_vector(dloss, n, torch.float32, "dloss", dev.index)
        h = _launch_on(dev.index, stream)
        with _on(stream):
            grad_out, gld = self._grad(logits, grad_out)
            status, own = self._status_of(status, dev)
        rc = self._backward(
            self._h, logits.data_ptr(), ld, n, *lists, stats.data_ptr(), _ptr(dloss),
            grad_out.data_ptr(), gld, None, 0, _ptr(status), h)
        if rc:
            _check("tkef_distill_backward", rc)
        if own:
            _raise_on_status("tkef_distill_backward", status, stream)
        return grad_out

    def step(self, logits: torch.Tensor, idx: torch.Tensor, val: torch.Tensor,
             tail: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
             weight: Optional[torch.Tensor] = None, loss_out: Optional[torch.Tensor] = None,
             grad_out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
             stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Loss (n,) float32 and the gradient of its sum, in one call.
        grad_out may be the logits themselves."""
        n, ld = self._logits(logits, "logits")
        dev = logits.device
        lists = self._lists(n, idx, val, tail, count, weight, dev.index)
        h = _launch_on(dev.index, stream)
        with _on(stream):
            loss_out = _out(loss_out, (n,), torch.float32, dev, "loss_out")
            grad_out, gld = self._grad(logits, grad_out)
            status, own = self._status_of(status, dev)
            with self._turn:
                ws = self._workspace(h, dev)
                rc = self._step(
                    self._h, logits.data_ptr(), ld, n, *lists, loss_out.data_ptr(),
                    grad_out.data_ptr(), gld, _ptr(ws), self.ws_bytes, _ptr(status), h)
        if rc:
            _check("tkef_distill_step", rc)
        if own:
            _raise_on_status("tkef_distill_step", status, stream)
        return loss_out, grad_out

    def loss(self, logits: torch.Tensor, idx: torch.Tensor, val: torch.Tensor,
             tail: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
             weight: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The loss (n,) as a node of torch's autograd graph: its backward
        pass is `backward` (gradients of the logits only)."""
        return _DistillLoss.apply(logits, self, idx, val, tail, count, weight)


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, plan, idx, val, tail, count, weight):
        loss, stats = plan.forward(logits, idx, val, tail=tail, count=count, weight=weight)
        ctx.plan = plan
        ctx.save_for_backward(logits, idx, val, stats, tail, count, weight)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        logits, idx, val, stats, tail, count, weight = ctx.saved_tensors
        grad = ctx.plan.backward(logits, idx, val, stats, tail=tail, count=count, weight=weight,
                                 dloss=dloss.to(torch.float32).contiguous())
        return grad, None, None, None, None, None, None


class VerifyPlan(_RowPlan):
    """Verification of drafted tokens against a target model's logits from
    given random numbers (tkef_verify_execute)."""

    _destroy = "tkef_verify_plan_destroy"
    _readied = True

    def __init__(self, batch: int, draft: int, vocab: int, dtype=torch.bfloat16,
                 temperature: float = 1.0, check: bool = False):
        """batch: the most sequences a call gives; draft: tokens per sequence."""
        super().__init__(batch, vocab, dtype, temperature, check)
        self.batch, self.draft = self.rows, int(draft)
        _check("tkef_verify_plan_create", lib().tkef_verify_plan_create(
            self.rows, self.draft, self.vocab, _dtype_code(dtype), self.temperature,
            ctypes.byref(self._h)))
        self._info("tkef_verify_plan_info")
        self._execute = lib().tkef_verify_execute

    def _ready(self, ws, stream):
        _check("tkef_verify_plan_bind", lib().tkef_verify_plan_bind(
            self._h, ws.data_ptr(), ws.numel(), stream))

    def workspace(self, stream=None) -> torch.Tensor:
        """A readied workspace for `execute(ws=...)` on the current GPU, cleared on
        `stream` (asynchronous). The caller keeps it for as long as calls, or graphs
        that captured one, may use it, and gives it to no two that may run at the same
        time. Without one a captured call clears its own at every replay, a launch
        more (64 sequences of 5 tokens: 32 us a replay, 26 with a workspace given)."""
        with _on(stream):
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("a workspace is readied before the capture that uses it")
            gpu = torch.cuda.current_device()
            ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=torch.device("cuda", gpu))
            self._ready(ws, _launch_on(gpu, stream))
        return ws

    def _block(self, x: torch.Tensor, places: int, what: str) -> Tuple[int, int]:
        if x.dim() != 3 or x.dtype != self.dtype or not x.is_cuda:
            raise ValueError(f"{what}: expected a 3-D CUDA tensor of {self.dtype}")
        if x.shape[1] != places or x.shape[2] != self.vocab or x.shape[0] > self.batch:
            raise ValueError(f"{what}: the plan takes up to {self.batch} x {places} x "
                             f"{self.vocab}")
        if self.vocab > 1 and x.stride(2) != 1:
            raise ValueError(f"{what}: the words of a row must be contiguous")
        return x.stride(0), (x.stride(1) if places > 1 else self.vocab)

    def execute(self, target: torch.Tensor, drafts: torch.Tensor, tokens: torch.Tensor,
                uniform: torch.Tensor, noise: torch.Tensor,
                length: Optional[torch.Tensor] = None,
                accepted_out: Optional[torch.Tensor] = None,
                tokens_out: Optional[torch.Tensor] = None,
                logp_out: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None, stream=None,
                ws: Optional[torch.Tensor] = None
                ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """target (b, draft + 1, vocab) and drafts (b, draft, vocab) logits,
        tokens (b, draft) int32, uniform (b, draft) float32 in [0, 1), noise
        (b, vocab) float32 from the exponential distribution, length (b,) int32.
        Returns accepted (b,) int32, tokens (b, draft + 1) int32 (accepted
        drafts, the token after them, then -1) and their log-probabilities
        under the target (b, draft + 1) float32. ws: a workspace of this plan
        (`workspace`); by default the plan has one for each stream, and a captured call
        its own."""
        tb, ti = self._block(target, self.draft + 1, "target")
        db, di = self._block(drafts, self.draft, "drafts")
        b = target.shape[0]
        dev = target.device
        if drafts.shape[0] != b or drafts.device != dev:
            raise ValueError("target and drafts differ in their number of sequences or device")
        _check_vector(tokens, b * self.draft, torch.int32, "tokens", dev.index)
        _check_vector(uniform, b * self.draft, torch.float32, "uniform", dev.index)
        _check_vector(length, b, torch.int32, "length", dev.index)
        if noise.dtype != torch.float32 or noise.device != dev or \
                noise.shape != (b, self.vocab) or (self.vocab > 1 and noise.stride(1) != 1):
            raise ValueError(f"noise: expected (batch, vocab) float32 values in rows on {dev}")
        h = _launch_on(dev.index, stream)
        with _on(stream):
            accepted_out = _out(accepted_out, (b,), torch.int32, dev, "accepted_out")
            tokens_out = _out(tokens_out, (b, self.draft + 1), torch.int32, dev, "tokens_out")
            logp_out = _out(logp_out, (b, self.draft + 1), torch.float32, dev, "logp_out")
            status, own = self._status_of(status, dev)
            with self._turn:
                if ws is None:
                    ws = self._workspace(h, dev)
                else:
                    _check_vector(ws, self.ws_bytes, torch.uint8, "ws", dev.index)
                rc = self._execute(
                    self._h, target.data_ptr(), tb, ti, drafts.data_ptr(), db, di, b,
                    tokens.data_ptr(), uniform.data_ptr(), noise.data_ptr(),
                    noise.stride(0) if b > 1 else self.vocab, _ptr(length), accepted_out.data_ptr(),
                    tokens_out.data_ptr(), logp_out.data_ptr(), _ptr(ws), self.ws_bytes,
                    _ptr(status), h)
        if rc:
            _check("tkef_verify_execute", rc)
        if own:
            _raise_on_status("tkef_verify_execute", status, stream)
        return accepted_out, tokens_out, logp_out


# ----------------------------------------------------------------------------
class ScorePlan(_RowPlan):
    """Scores of given tokens: each row's log-probability of its token, entropy,
    and k greatest words in descending order (tkef_score_forward), and the gradient of the
    first two (tkef_score_backward). tokens (n,) int32; a row with token -1 is not read, its
    results and gradient are 0."""

    _destroy = "tkef_score_plan_destroy"

    def __init__(self, rows: int, vocab: int, k: int = 0, dtype=torch.bfloat16,
                 temperature: float = 1.0, check: bool = False):
        """rows: the most rows a call gives; k: alternatives that `execute` returns (0 to
        SCORE_MAX_K)."""
        super().__init__(rows, vocab, dtype, temperature, check)
        self.k = int(k)
        _check("tkef_score_plan_create", lib().tkef_score_plan_create(
            self.rows, self.vocab, self.k, _dtype_code(dtype), self.temperature,
            ctypes.byref(self._h)))
        self._info("tkef_score_plan_info")
        self._forward, self._backward = lib().tkef_score_forward, lib().tkef_score_backward

    def execute(self, logits: torch.Tensor, tokens: torch.Tensor,
                logp_out: Optional[torch.Tensor] = None,
                entropy_out: Optional[torch.Tensor] = None,
                idx_out: Optional[torch.Tensor] = None, val_out: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None, stream=None
                ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
        """Returns logp (n,), entropy (n,), and the alternatives idx (n, k) int32 with
        their log-probabilities val (n, k); values are float32."""
        n, ld = self._logits(logits, "logits")
        dev = logits.device
        _check_vector(tokens, n, torch.int32, "tokens", dev.index)
        h = _launch_on(dev.index, stream)
        with _on(stream):
            logp_out = _out(logp_out, (n,), torch.float32, dev, "logp_out")
            entropy_out = _out(entropy_out, (n,), torch.float32, dev, "entropy_out")
            idx_out = _out(idx_out, (n, self.k), torch.int32, dev, "idx_out")
            val_out = _out(val_out, (n, self.k), torch.float32, dev, "val_out")
            status, own = self._status_of(status, dev)
            with self._turn:
                ws = self._workspace(h, dev)
                rc = self._forward(
                    self._h, logits.data_ptr(), ld, n, tokens.data_ptr(), logp_out.data_ptr(),
                    entropy_out.data_ptr(), idx_out.data_ptr() if self.k else None,
                    val_out.data_ptr() if self.k else None, None, _ptr(ws), self.ws_bytes,
                    _ptr(status), h)
        if rc:
            _check("tkef_score_forward", rc)
        if own:
            _raise_on_status("tkef_score_forward", status, stream)
        return logp_out, entropy_out, idx_out, val_out

    def forward(self, logits: torch.Tensor, tokens: torch.Tensor,
                logp_out: Optional[torch.Tensor] = None,
                entropy_out: Optional[torch.Tensor] = None,
                stats_out: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None, stream=None
                ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """Returns logp (n,) and entropy (n,) float32, and stats (n, 4) float32, which
        backward takes. No alternatives are looked for, whatever the plan's k."""
        n, ld = self._logits(logits, "logits")
        dev = logits.device
        _check_vector(tokens, n, torch.int32, "tokens", dev.index)
        h = _launch_on(dev.index, stream)
        with _on(stream):
            logp_out = _out(logp_out, (n,), torch.float32, dev, "logp_out")
            entropy_out = _out(entropy_out, (n,), torch.float32, dev, "entropy_out")
            stats_out = _out(stats_out, (n, 4), torch.float32, dev, "stats_out")
            status, own = self._status_of(status, dev)
            with self._turn:
                ws = self._workspace(h, dev)
                rc = self._forward(
                    self._h, logits.data_ptr(), ld, n, tokens.data_ptr(), logp_out.data_ptr(),
                    entropy_out.data_ptr(), None, None, stats_out.data_ptr(), _ptr(ws),
                    self.ws_bytes, _ptr(status), h)
        if rc:
            _check("tkef_score_forward", rc)
        if own:
            _raise_on_status("tkef_score_forward", status, stream)
        return logp_out, entropy_out, stats_out

    def backward(self, logits: torch.Tensor, tokens: torch.Tensor, stats: torch.Tensor,
                 dlogp: Optional[torch.Tensor] = None, dentropy: Optional[torch.Tensor] = None,
                 grad_out: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Gradient of sum(dlogp * logp + dentropy * entropy) in the logits' type (dlogp,
        dentropy (n,) float32; one of them may be None, 0). grad_out may be the logits
        themselves."""
        n, ld = self._logits(logits, "logits")
        dev = logits.device
        if dlogp is None and dentropy is None:
            raise ValueError("backward: expected dlogp or dentropy")
        _check_vector(tokens, n, torch.int32, "tokens", dev.index)
        _check_vector(stats, n * 4, torch.float32, "stats", dev.index)
        _check_vector(dlogp, n, torch.float32, "dlogp", dev.index)
        _check_vector(dentropy, n, torch.float32, "dentropy", dev.index)
        h = _launch_on(dev.index, stream)
        with _on(stream):
            grad_out, gld = self._grad(logits, grad_out)
            status, own = self._status_of(status, dev)
        rc = self._backward(
            self._h, logits.data_ptr(), ld, n, tokens.data_ptr(), stats.data_ptr(), _ptr(dlogp),
            _ptr(dentropy), grad_out.data_ptr(), gld, _ptr(status), h)
        if rc:
            _check("tkef_score_backward", rc)
        if own:
            _raise_on_status("tkef_score_backward", status, stream)
        return grad_out

    def score(self, logits: torch.Tensor, tokens: torch.Tensor
              ) -> Tuple[torch.Tensor, torch.Tensor]:
        """logp (n,) and entropy (n,) as outputs of a node of torch's autograd graph, whose
        backward pass is `backward`. (A training step that is captured into a graph: torch
        keeps a leaf's accumulation on the stream of the first graph that it is part of, so no
        eager result of the same leaves may be alive when the backward pass is captured.)"""
        return _Score.apply(logits, self, tokens)


class _Score(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, plan, tokens):
        logp, entropy, stats = plan.forward(logits, tokens)
        ctx.plan = plan
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(logits, tokens, stats)
        return logp, entropy

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dlogp, dentropy):
        if dlogp is None and dentropy is None:
            return None, None, None
        logits, tokens, stats = ctx.saved_tensors
        dlogp, dentropy = (d if d is None else d.to(torch.float32).contiguous()
                           for d in (dlogp, dentropy))
        return ctx.plan.backward(logits, tokens, stats, dlogp=dlogp, dentropy=dentropy), None, None


# ----------------------------------------------------------------------------
# one-shot calls: a plan, one execution, and TkefStatusError on any status bit
# (they synchronize), unless the caller gives a status word to check itself

def top_logits(logits: torch.Tensor, k: int, temperature: float = 1.0,
               val_dtype=torch.float32, status: Optional[torch.Tensor] = None):
    """(idx, val, tail) of each row's k greatest logits: TopLogitsPlan."""
    plan = TopLogitsPlan(max(1, logits.shape[0]), logits.shape[1], k, logits.dtype, temperature,
                         val_dtype, check=status is None)
    return plan.execute(logits, status=status)


def distill_step(logits: torch.Tensor, idx: torch.Tensor, val: torch.Tensor,
                 temperature: float = 1.0, tail: Optional[torch.Tensor] = None,
                 count: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None):
    """(loss, grad) of each row: DistillPlan.step."""
    plan = DistillPlan(max(1, logits.shape[0]), logits.shape[1], idx.shape[1], logits.dtype,
                       temperature, val.dtype, check=status is None)
    return plan.step(logits, idx, val, tail=tail, count=count, weight=weight, status=status)


def verify_draft(target: torch.Tensor, drafts: torch.Tensor, tokens: torch.Tensor,
                 uniform: torch.Tensor, noise: torch.Tensor, temperature: float = 1.0,
                 length: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """(accepted, tokens, logp) of each sequence: VerifyPlan.execute."""
    plan = VerifyPlan(max(1, target.shape[0]), drafts.shape[1], target.shape[2], target.dtype,
                      temperature, check=status is None)
    return plan.execute(target, drafts, tokens, uniform, noise, length=length, status=status)


def score_tokens(logits: torch.Tensor, tokens: torch.Tensor, k: int = 0, temperature: float = 1.0,
                 status: Optional[torch.Tensor] = None):
    """(logp, entropy, idx, val) of each row: ScorePlan.execute."""
    plan = ScorePlan(max(1, logits.shape[0]), logits.shape[1], k, logits.dtype, temperature,
                     check=status is None)
    return plan.execute(logits, tokens, status=status)
