"""The embedding's gradient where nothing rounds: rows of small whole numbers, none of them 0,
and a scale that is a power of two, so that every sum is exact whatever its order and a
single token that is lost, doubled or given to another word shows. Long words over many tiles,
the most tokens, the widest rows, tables and batches beyond 2^32 bytes."""
import numpy as np
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu
from rows_common import TYPES
from test_gpu_embed import some_tokens

MOST = 8            # of a number's magnitude: 2^20 tokens sum to at most 2^23
SCALE = -0.5

# tokens, words, columns, type of the rows: whole waves a group and parts of one, tiles of 16 to
# 256 tokens, joins of both sizes
CASES = [
    (3000, 50, 33, "f32"), (9000, 700, 512, "bf16"), (16383, 1500, 5, "bf16"),
    (17000, 700, 1030, "bf16"), (17000, 700, 2051, "f16"), (66000, 700, 260, "bf16"),
    (66000, 700, 515, "bf16"), (70001, 1500, 16, "bf16"), (132000, 700, 257, "f32"),
    (300_000, 1500, 3, "f16"), (1 << 20, 1000, 257, "bf16"), (1 << 20, 131071, 64, "f32"),
    (1 << 20, 1 << 20, 3, "f32")]
KINDS = ["law", "one", "two", "uniform"]


def whole_numbers(n, width, dtype, dev, seed):
    gen = torch.Generator(device=dev).manual_seed(seed)
    x = torch.randint(1, MOST + 1, (n, width), generator=gen, device=dev, dtype=torch.int8)
    sign = torch.randint(0, 2, (n, width), generator=gen, device=dev, dtype=torch.int8)
    return (x * (2 * sign - 1)).to(dtype)


def sums(tokens, dout, vocab, step=256):
    """The gradient in 64 bits, where these sums are exact too, some columns at a time: differences
    of running sums over the sorted tokens. (index_add_ of 131,072 rows into one word of 2^20
    takes 45 s on the GPU.)"""
    out = torch.zeros(vocab, dout.shape[1], dtype=torch.float64, device=dout.device)
    live = (tokens >= 0).nonzero()[:, 0]
    word, order = tokens[live].long().sort(stable=True)
    words, counts = word.unique_consecutive(return_counts=True)
    last = counts.cumsum(0) - 1
    for c in range(0, dout.shape[1], step):
        run = dout[live[order], c:c + step].double().t().contiguous().cumsum(1)
        out[words, c:c + step] = torch.diff(run[:, last], prepend=run.new_zeros(len(run), 1)).t()
    return out * SCALE


def case(n, vocab, width, dtype, kind, dev):
    rng = np.random.default_rng(n + width)
    tokens = torch.as_tensor(some_tokens(rng, kind, n, vocab).astype(np.int32)).to(dev)
    return tokens, whole_numbers(n, width, TYPES[dtype], dev, n + 1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,vocab,width,dtype", [c for c in CASES if c[0] < 1 << 20])
def test_the_comparison_sees_one_token(n, vocab, width, dtype, kind):
    """(On the CPU, the mistake in the reference.) A token left out, taken twice or given to another
    word changes each column of a sum by at least half a unit, and all values are exact in
    binary32."""
    width = min(width, 4)
    tokens, dout = case(n, vocab, width, dtype, kind, "cpu")
    want = sums(tokens, dout, vocab)
    assert torch.equal(want, want.float().double())
    at = int((tokens >= 0).nonzero()[n // 3, 0])
    for mistake in ("lost", "doubled", "moved"):
        t, d = tokens.clone(), dout
        if mistake == "lost":
            t[at] = -1
        elif mistake == "moved":
            t[at] = (t[at] + 1) % vocab
        else:
            t, d = torch.cat([t, t[at:at + 1]]), torch.cat([d, d[at:at + 1]])
        off = (sums(t, d, vocab) - want).abs()
        assert bool((off[int(tokens[at])] >= 0.5).all()), mistake


def check(n, vocab, width, dtype, kind, grad, lists=True):
    announce(f"exact gradient {n} of {vocab}x{width} {dtype}->{grad} {kind}")
    dev = need_gpu()
    tokens, dout = case(n, vocab, width, dtype, kind, dev)
    want = sums(tokens, dout, vocab)
    plan = tk.EmbedPlan(n, vocab, width, dtype=torch.float32, out_dtype=TYPES[dtype],
                        grad_dtype=TYPES[grad], val_dtype=TYPES["f16" if grad == "f16" else "f32"],
                        scale=SCALE, check=True)
    got = plan.backward(tokens, dout)
    assert torch.equal(got, want.to(TYPES[grad]))   # (one rounding, of an exact sum)
    add = whole_numbers(vocab, width, TYPES[grad], dev, 5)
    summed = (want + add).to(TYPES[grad])
    assert torch.equal(plan.backward(tokens, dout, add=add), summed)
    assert torch.equal(plan.backward(tokens, dout, add=add, grad_out=add), summed)
    if not lists:
        return
    idx, val, nnz = plan.lists(tokens, dout, offset=11)
    words = tokens[tokens >= 0].unique().long()
    m = words.numel() * width
    assert int(nnz.item()) == m
    at = words[:, None] * width + torch.arange(width, device=dev) + 11
    assert torch.equal(idx[:m].long(), at.view(-1))
    assert torch.equal(val[:m], want[words].to(val.dtype).view(-1))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,vocab,width,dtype", CASES)
def test_exact_sums(n, vocab, width, dtype, kind):
    check(n, vocab, width, dtype, kind, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("grad", ["f16", "bf16"])
@pytest.mark.parametrize("n,vocab,width,dtype", [(200, 90, 515, "bf16"), (9000, 700, 512, "f32"),
                                                 (66000, 700, 260, "f16")])
def test_exact_sums_rounded_to_16_bits(n, vocab, width, dtype, grad):
    check(n, vocab, width, dtype, "law", grad)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [192, 223, 224, 225, 256, 257])
def test_few_tokens_in_one_launch_and_in_three(n, kind):
    for vocab, width in ((150, 33), (32000, 515), (131073, 64)):
        check(n, vocab, width, "bf16", kind, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("n", [7, 256, 257, 3000, 17000])
def test_the_widest_rows(n):
    check(n, 40, 1 << 16, "bf16", "law", "f32")


@pytest.mark.gpu
def test_a_batch_beyond_2_32_bytes():
    check(1 << 20, 700, 2051, "bf16", "law", "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("n", [200, 5000, 20000])
def test_a_table_beyond_2_32_bytes(n):
    """2^20 words of 4,099 columns, 8.6 GB: lookup, gradient, and words at the table's ends."""
    announce(f"table of 2^20 x 4099, {n} tokens")
    dev = need_gpu()
    vocab, width = 1 << 20, 4099
    tokens, dout = case(n, vocab, width, "bf16", "uniform", dev)
    tokens[: n // 2 : 2] = vocab - 1
    tokens[1 : n // 2 : 2] = 0
    table = torch.empty(vocab, width, dtype=torch.bfloat16, device=dev)
    for i in range(0, vocab, 1 << 16):
        table[i:i + (1 << 16)] = whole_numbers(1 << 16, width, torch.bfloat16, dev, i)
    plan = tk.EmbedPlan(n, vocab, width, dtype=torch.bfloat16, scale=SCALE, check=True)
    out = plan.forward(table, tokens)
    assert torch.equal(out, table[tokens.long()] * SCALE)
    words, place = tokens.long().unique(return_inverse=True)
    want = sums(place.int(), dout, words.numel()).to(torch.bfloat16)
    got = plan.backward(tokens, dout, grad_out=torch.full_like(table, 3.0))
    assert torch.equal(got[words], want)
    there = torch.zeros(vocab, dtype=torch.bool, device=dev)
    there[words] = True
    for i in range(0, vocab, 1 << 16):
        block = slice(i, i + (1 << 16))
        assert not bool(got[block][~there[block]].any())
    del got, out
    rest = plan.backward(tokens, dout, add=table)
    for i in range(0, vocab, 1 << 16):
        block = slice(i, i + (1 << 16))
        assert torch.equal(rest[block][~there[block]], table[block][~there[block]])
    assert torch.equal(rest[words], (sums(place.int(), dout, words.numel())
                                     + table[words]).to(torch.bfloat16))
