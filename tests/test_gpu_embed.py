"""EmbedPlan (forward, backward, lists) against the oracle: types, sizes, strides,
distributions of tokens, padding, and lists that the update plan takes."""
import math

import numpy as np
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu
from oracle import score as oracle
from rows_common import EPS, STORE, TYPES, device_rows, vec

pytestmark = pytest.mark.gpu

KINDS = ("few", "uniform", "law", "one", "two", "none", "each", "ends")


def some_tokens(rng, kind, n, vocab):
    if kind == "uniform":
        return rng.integers(0, vocab, n)
    if kind == "few":
        return rng.choice([-1, 0, vocab // 3, vocab - 1], n)
    if kind == "law":
        w = 1.0 / (np.arange(vocab) + 2.7)
        t = rng.choice(vocab, n, p=w / w.sum())
        t[rng.random(n) < 0.1] = -1
        return t
    if kind == "one":
        return np.full(n, vocab // 2)
    if kind == "two":       # one word, but for its neighbours at the ends
        t = np.full(n, vocab // 2)
        t[: n // 3] = vocab - 1
        return t
    if kind == "none":
        return np.full(n, -1)
    if kind == "each":
        return np.arange(n) % vocab
    return np.where(np.arange(n) % 2 == 0, 0, vocab - 1)


def bits_of(t):
    return t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


def check_lookup(rng, n, vocab, width, table_type, out_type, scale, tokens, pad=0, shift=0, opad=0):
    announce(f"lookup {n} of {vocab}x{width} {table_type}->{out_type}")
    dev = need_gpu()
    table, _ = device_rows(rng.normal(size=(vocab, width)), table_type, pad, shift)
    plan = tk.EmbedPlan(n + 3, vocab, width, dtype=TYPES[table_type], out_dtype=TYPES[out_type],
                        scale=scale, check=True)
    wide = torch.full((n, width + opad), 7.0, dtype=TYPES[out_type], device=dev)
    out = plan.forward(table, vec(tokens, torch.int32), out=wide[:, :width])
    assert bool((wide[:, width:] == 7.0).all())
    # one product in binary32, rounded once to the type: the same everywhere
    t = torch.as_tensor(tokens)
    want = table.cpu().float()[t.clamp(min=0)] * torch.tensor(scale, dtype=torch.float32)
    want[t < 0] = 0.0
    assert torch.equal(bits_of(out.cpu()), bits_of(want.to(TYPES[out_type])))


def gradient_case(rng, n, width, out_type, tokens, pad=0, shift=0):
    dout, exact = device_rows(rng.normal(size=(n, width)), out_type, pad, shift)
    dead = np.asarray(tokens) < 0
    if dead.any():
        dout[torch.as_tensor(np.nonzero(dead)[0])] = math.nan   # padding is not read
        exact[dead] = math.nan
    return dout, exact, vec(tokens, torch.int32)


def close(got, want, size, counts, store, add=None):
    """c terms are added in some order, each sum rounds to binary32 (c - 1 units of the sum
    of magnitudes at most), the scale and what is added round once more each, the
    result once to its type."""
    half, least = store
    total = want if add is None else want + add
    tol = EPS * (counts[:, None] + 1) * size + np.abs(total) * half * 1.01 + least
    if add is not None:
        tol = tol + EPS * (np.abs(total) + size)
    err = np.abs(got - total)
    bad = np.argwhere(~(err <= tol))
    assert bad.size == 0, (bad[:4], got[tuple(bad[0])], total[tuple(bad[0])], tol[tuple(bad[0])])


def check_gradient(rng, n, vocab, width, out_type, grad_type, scale, tokens, pad=0, shift=0, gpad=0):
    announce(f"gradient {n} of {vocab}x{width} {out_type}->{grad_type} pad={pad}")
    dev = need_gpu()
    dout, exact, tok = gradient_case(rng, n, width, out_type, tokens, pad, shift)
    plan = tk.EmbedPlan(n + 5, vocab, width, dtype=torch.float32, out_dtype=TYPES[out_type],
                        grad_dtype=TYPES[grad_type], scale=scale, check=True)
    want, size, counts = oracle.embed_sums(tokens, exact, vocab, float(np.float32(scale)))
    wide = torch.full((vocab, width + gpad), 7.0, dtype=TYPES[grad_type], device=dev)
    got = plan.backward(tok, dout, grad_out=wide[:, :width])
    assert bool((wide[:, width:] == 7.0).all())
    close(got.double().cpu().numpy(), want, size, counts, STORE[grad_type])
    assert bool((bits_of(got)[torch.as_tensor(counts == 0).to(dev)] == 0).all())
    again = plan.backward(tok, dout)
    assert torch.equal(bits_of(again), bits_of(got))
    # with another gradient added: into a new buffer, and in place
    other, other_exact = device_rows(rng.normal(size=(vocab, width)), grad_type, gpad)
    summed = plan.backward(tok, dout, add=other)
    close(summed.double().cpu().numpy(), want, size, counts, STORE[grad_type], add=other_exact)
    plan.backward(tok, dout, add=other, grad_out=other)
    assert torch.equal(bits_of(other), bits_of(summed))


def check_lists(rng, n, vocab, width, out_type, val_type, scale, tokens, offset=0, pad=0):
    announce(f"lists {n} of {vocab}x{width} {out_type}->{val_type}")
    dev = need_gpu()
    dout, exact, tok = gradient_case(rng, n, width, out_type, tokens, pad)
    plan = tk.EmbedPlan(n + 5, vocab, width, dtype=torch.float32, out_dtype=TYPES[out_type],
                        val_dtype=TYPES[val_type], scale=scale, check=True)
    want, size, counts = oracle.embed_sums(tokens, exact, vocab, float(np.float32(scale)))
    idx = torch.full((plan.most(n) + 7,), -9, dtype=torch.int32, device=dev)
    val = torch.full((plan.most(n) + 7,), 7.0, dtype=TYPES[val_type], device=dev)
    _, _, nnz = plan.lists(tok, dout, offset=offset, idx_out=idx, val_out=val)
    words = np.nonzero(counts)[0]
    m = words.size * width
    assert int(nnz.item()) == m
    at = (words[:, None] * width + np.arange(width)[None]).ravel() + offset
    assert (idx[:m].cpu().numpy() == at).all()
    assert bool((idx[m:] == -9).all()) and bool((val[m:] == 7.0).all())
    if m:
        close(val[:m].double().cpu().numpy().reshape(-1, width), want[words], size[words],
              counts[words], STORE[val_type])


@pytest.mark.parametrize("table_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("out_type", ["f32", "f16", "bf16"])
def test_lookup_types(table_type, out_type):
    rng = np.random.default_rng(1)
    for n, vocab, width, scale in ((5, 7, 1, 2.0), (33, 100, 64, 0.3), (4, 1000, 515, 22.627417),
                                   (300, 50, 1030, -1.0), (9, 20, 2051, 1.0)):
        check_lookup(rng, n, vocab, width, table_type, out_type, scale,
                     some_tokens(rng, "law", n, vocab))


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 63, 64, 65, 1000, 5001])
@pytest.mark.parametrize("width", [1, 2, 7, 8, 9, 63, 512, 1000])
def test_lookup_sizes(n, width):
    rng = np.random.default_rng(n * 3 + width)
    check_lookup(rng, n, 333, width, "f32", "bf16", 1.5, some_tokens(rng, "uniform", n, 333),
                 pad=n % 3, shift=n % 5, opad=n % 4)
    check_lookup(rng, n, 333, width, "bf16", "bf16", 1.0, some_tokens(rng, "few", n, 333),
                 pad=n % 4, shift=n % 3, opad=n % 2)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 7, 8, 9, 64, 65, 100, 255, 256, 257, 513, 2048, 2049, 3000])
def test_gradient_tokens(n, kind):
    rng = np.random.default_rng(n)
    for vocab, width in ((1, 5), (50, 33), (1000, 64), (2111, 8)):
        tokens = some_tokens(rng, kind, n, vocab)
        check_gradient(rng, n, vocab, width, "f32", "f32", 1.5, tokens)
        check_lists(rng, n, vocab, width, "f32", "f32", 1.5, tokens, offset=12345)


@pytest.mark.parametrize("out_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("grad_type", ["f32", "f16", "bf16"])
def test_gradient_types(grad_type, out_type):
    rng = np.random.default_rng(2)
    for n, vocab, width in ((300, 90, 512), (200, 70, 515), (64, 40, 1030), (50, 30, 2051),
                            (77, 1100, 64), (270, 500, 515), (290, 30, 2051), (301, 2000, 4)):
        tokens = some_tokens(rng, "law", n, vocab)
        check_gradient(rng, n, vocab, width, out_type, grad_type, 0.37, tokens, pad=n % 3,
                       shift=n % 5, gpad=n % 4)
        check_lists(rng, n, vocab, width, out_type, "f16" if grad_type == "f16" else "f32", -0.37,
                    tokens, pad=n % 4)


@pytest.mark.parametrize("kind", ["law", "one", "two", "uniform"])
@pytest.mark.parametrize("n,width", [(16383, 5), (16384, 8), (18433, 65), (32769, 9), (70001, 16),
                                     (300_000, 3)])
def test_gradient_of_many_tokens(n, width, kind):
    rng = np.random.default_rng(n)
    tokens = some_tokens(rng, kind, n, 1500)
    check_gradient(rng, n, 1500, width, "bf16", "f32", 1.0, tokens)
    check_lists(rng, n, 1500, width, "f32", "f32", 1.0, tokens)


@pytest.mark.parametrize("vocab", [(1 << 17) + 5, 1 << 20])
def test_gradient_of_large_vocabularies(vocab):
    rng = np.random.default_rng(vocab)
    for n, kind in ((700, "uniform"), (700, "law"), (700, "ends"), (130, "uniform"), (9, "ends"),
                    (20000, "law"), (16500, "ends"), (40000, "uniform")):
        tokens = some_tokens(rng, kind, n, vocab)
        check_gradient(rng, n, vocab, 3, "f32", "f32", 1.0, tokens)
        check_lists(rng, n, vocab, 3, "f32", "f32", 1.0, tokens)


@pytest.mark.parametrize("kind", ["law", "one", "two"])
@pytest.mark.parametrize("n,width,out_type,grad_type", [
    (17000, 1030, "bf16", "f32"), (17000, 2051, "f16", "f16"), (66000, 260, "bf16", "f32"),
    (66000, 515, "bf16", "bf16"), (132000, 257, "f32", "f32")])
def test_gradient_of_many_wide_rows(n, width, out_type, grad_type, kind):
    """Groups of whole waves, tiles of 16, 32 and 64 tokens, words over many tiles."""
    rng = np.random.default_rng(n + width)
    tokens = some_tokens(rng, kind, n, 700)
    check_gradient(rng, n, 700, width, out_type, grad_type, -0.5, tokens)
    check_lists(rng, n, 700, width, out_type, "f32", -0.5, tokens)


@pytest.mark.parametrize("n", [40, 900])
def test_gradient_against_differences(n):
    """The lookup is linear in the table: half the difference of its products with dout at
    table + D and table - D is the gradient's product with D, whatever D's size. Each of
    the n * width products, of numbers that round once to binary32, is off by EPS, and each
    entry of the gradient by EPS a term."""
    rng = np.random.default_rng(n)
    vocab, width = 300, 17
    tokens = some_tokens(rng, "law", n, vocab)
    tok = vec(tokens, torch.int32)
    dout, exact, _ = gradient_case(rng, n, width, "f32", tokens)
    plan = tk.EmbedPlan(n, vocab, width, dtype=torch.float32, scale=3.0, check=True)
    table, step = vec(rng.normal(size=(vocab, width))), vec(rng.normal(size=(vocab, width)))
    up, down = table + step, table - step
    step = (up.double() - down.double()) / 2     # what the rounded tables differ by
    live = torch.as_tensor(tokens >= 0)
    d = dout.double().cpu()[live]
    high, low = (plan.forward(t, tok).double().cpu()[live] for t in (up, down))
    slope = float(((high - low) / 2 * d).sum())
    grad = plan.backward(tok, dout).double().cpu()
    want = float((grad * step.cpu()).sum())
    _, size, counts = oracle.embed_sums(tokens, exact, vocab, 3.0)
    tol = EPS * (float(((high.abs() + low.abs()) * d.abs()).sum())
                 + float((size * (counts[:, None] + 2) * step.abs().cpu().numpy()).sum()))
    assert abs(slope - want) <= tol


def test_no_tokens():
    """The dense gradient is 0, or what is added; the list is empty."""
    dev = need_gpu()
    plan = tk.EmbedPlan(4, 300, 17, dtype=torch.float32, check=True)
    tok, dout = torch.zeros(0, dtype=torch.int32, device=dev), torch.zeros(0, 17, device=dev)
    grad = torch.full((300, 17), 7.0, device=dev)
    assert bool((plan.backward(tok, dout, grad_out=grad) == 0).all())
    add = torch.randn(300, 17, device=dev)
    assert torch.equal(plan.backward(tok, dout, add=add, grad_out=grad), add)
    before = add.clone()
    assert torch.equal(plan.backward(tok, dout, add=add, grad_out=add), before)
    idx, val, nnz = plan.lists(tok, dout)
    assert int(nnz.item()) == 0
    assert plan.forward(add, tok).shape == (0, 17)


def test_words_outside_the_vocabulary():
    """They are padding, with the status bit; -1 raises none."""
    dev = need_gpu()
    tok = torch.tensor([3, 50, -1, -2, 2 ** 31 - 1, 3, -2 ** 31], dtype=torch.int32, device=dev)
    table, dout = torch.randn(50, 9, device=dev), torch.randn(7, 9, device=dev)
    plan = tk.EmbedPlan(7, 50, 9, dtype=torch.float32)
    for call in ("forward", "backward", "lists"):
        status = torch.zeros(1, dtype=torch.int32, device=dev)
        if call == "forward":
            out = plan.forward(table, tok, status=status)
            assert torch.equal(out[0], table[3]) and torch.equal(out[5], table[3])
            assert int((out != 0).any(1).sum()) == 2
        elif call == "backward":
            g = plan.backward(tok, dout, status=status)
            assert torch.equal(g[3], dout[0] + dout[5])
            g[3] = 0
            assert not bool(g.any())
        else:
            idx, val, nnz = plan.lists(tok, dout, status=status)
            assert int(nnz.item()) == 9 and idx[:9].tolist() == list(range(27, 36))
        assert int(status.item()) == tk.STATUS_INDEX_RANGE
    with pytest.raises(tk.TkefStatusError):
        tk.embed_tokens(table, tok)
    with pytest.raises(tk.TkefStatusError):
        tk.embed_gradient(tok, dout, 50)
    with pytest.raises(tk.TkefStatusError):
        tk.embed_lists(tok, dout, 50)
    tok[[1, 3, 4, 6]] = -1
    assert torch.equal(tk.embed_tokens(table, tok)[5], table[3])
    idx, val = tk.embed_lists(tok, dout, 50)
    assert idx.tolist() == list(range(27, 36)) and torch.equal(val, dout[0] + dout[5])
    assert torch.equal(tk.embed_gradient(tok, dout, 50)[3], val)


@pytest.mark.parametrize("form", ["weights", "sum", "columns"])
def test_autograd(form):
    """Under autograd, tokens of two dimensions; a gradient whose rows share memory, and one that
    is columns of wider rows."""
    rng = np.random.default_rng(21)
    dev = need_gpu()
    tokens = some_tokens(rng, "law", 60, 40).reshape(5, 12)
    table = vec(rng.normal(size=(40, 24))).requires_grad_()
    plan = tk.EmbedPlan(60, 40, 24, dtype=torch.float32, out_dtype=torch.bfloat16, scale=4.0)
    x = plan.lookup(table, vec(tokens, torch.int32))
    assert x.shape == (60, 24) and x.dtype == torch.bfloat16
    w = torch.ones(60, 24, dtype=torch.bfloat16, device=dev)
    if form == "sum":
        x.sum().backward()
    elif form == "weights":
        w = vec(rng.normal(size=(60, 24)), torch.bfloat16)
        (x * w).sum().backward()
    else:
        w = vec(rng.normal(size=(60, 24)), torch.bfloat16)
        both = vec(rng.normal(size=(60, 30)), torch.bfloat16)
        both[:, :24] = w
        torch.autograd.backward(x, both[:, :24])
    want, size, counts = oracle.embed_sums(tokens, w.double().cpu().numpy(), 40, 4.0)
    close(table.grad.double().cpu().numpy(), want, size, counts, STORE["f32"])


def test_lists_of_workers_update_the_table():
    """Two workers' lists, gathered, through UpdatePlan: the embedding is updated with the sum of
    their gradients, beside another tensor that stays as it is."""
    rng = np.random.default_rng(22)
    dev = need_gpu()
    vocab, width, n, before = 120, 16, 90, 37
    plan = tk.EmbedPlan(n, vocab, width, dtype=torch.float32, scale=2.0, check=True)
    stride = plan.most(n)
    idx = torch.zeros(2, stride, dtype=torch.int32, device=dev)
    val = torch.zeros(2, stride, device=dev)
    nnz = torch.zeros(2, dtype=torch.int32, device=dev)
    total = np.zeros((vocab, width))
    mass = np.zeros_like(total)
    counts = np.zeros(vocab)
    for p in range(2):
        tokens = some_tokens(rng, "law", n, vocab)
        dout, exact, tok = gradient_case(rng, n, width, "f32", tokens)
        plan.lists(tok, dout, offset=before, idx_out=idx[p], val_out=val[p], nnz_out=nnz[p: p + 1])
        g, a, c = oracle.embed_sums(tokens, exact, vocab, 2.0)
        total, mass, counts = total + g, mass + a, counts + c
    params = [torch.ones(before, device=dev), torch.zeros(vocab, width, device=dev)]
    up = tk.UpdatePlan([before, vocab * width], P=2, stride=stride).bind(params)
    up.execute(idx, val, nnz=nnz, lr=0.5)
    assert bool((params[0] == 1).all())
    # (half of a sum is exact; the two lists' sum rounds once more)
    close(params[1].double().cpu().numpy() / -0.5, total, mass, counts + 1, STORE["f32"])
