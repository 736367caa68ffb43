"""VerifyPlan against the oracle: accepted counts and tokens exactly (where the
oracle's decisions are not within rounding of the other outcome), and
log-probabilities within the rounding of a 32-bit sum."""
import math

import numpy as np
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu
from oracle import rows
from rows_common import INF, TYPES, finite_max, logits, rounding, vec

pytestmark = pytest.mark.gpu


def block(x, dtype, pad):
    """x (b, places, v) as a view of longer rows (the gaps hold NaN)."""
    b, places, v = x.shape
    wide = torch.full((b, places, v + pad), math.nan, dtype=TYPES[dtype], device=need_gpu())
    view = wide[..., :v]
    view.copy_(torch.from_numpy(x).to(TYPES[dtype]))
    return view, view.double().cpu().numpy()


def drafted(rng, drafts, temperature):
    noise = rng.gumbel(size=drafts.shape)
    return (drafts / temperature + noise).argmax(-1)


def check(rng, b, draft, v, dtype, temperature=1.0, ragged=False, pad=0, target=None, drafts=None,
          tokens=None, uniform=None, noise=None):
    announce(f"verify {b}x{draft}x{v} {dtype} T={temperature} ragged={ragged} pad={pad}")
    if target is None:
        target = rng.normal(size=(b, draft + 1, v)) * 3 * temperature
    if drafts is None:
        drafts = target[:, :draft] + rng.normal(size=(b, draft, v)) * 0.7 * temperature
    t_dev, t_h = block(target, dtype, pad)
    d_dev, d_h = block(drafts, dtype, pad)
    tokens = drafted(rng, d_h, temperature) if tokens is None else np.asarray(tokens)
    uniform = rng.random((b, draft)) if uniform is None else np.asarray(uniform)
    noise = rng.exponential(size=(b, v)) if noise is None else noise
    length = rng.integers(0, draft + 1, b) if ragged else np.full(b, draft)
    u_dev, e_dev = vec(uniform), vec(noise)
    plan = tk.VerifyPlan(b + 1, draft, v, dtype=TYPES[dtype], temperature=temperature, check=True)
    got = plan.execute(t_dev, d_dev, vec(tokens, torch.int32), u_dev, e_dev,
                       length=vec(length, torch.int32) if ragged else None)
    acc, out, logp = [g.cpu().numpy() for g in got]
    u_h, e_h = u_dev.double().cpu().numpy(), e_dev.double().cpu().numpy()
    close = 0
    for s in range(b):
        want = rows.verify(t_h[s], d_h[s], tokens[s], u_h[s], e_h[s], int(length[s]), temperature)
        rel = rounding(v, finite_max(t_h[s], d_h[s]) / temperature)
        if want.margin < 8 * rel:   # rounding may decide otherwise
            close += 1
            assert 0 <= acc[s] <= length[s]
            continue
        assert acc[s] == want.accepted, (s, acc[s], want.accepted, want.margin)
        assert out[s].tolist() == want.tokens, (s, out[s], want.tokens, want.margin)
        tol = rel + 2.0 ** -22 * finite_max(want.logp)
        assert np.abs(logp[s] - want.logp).max() <= tol, (s, logp[s], want.logp)
    assert close <= max(1, b // 8), close


SIZES = [(1, 1, 1), (2, 1, 2), (3, 2, 7), (5, 3, 64), (4, 8, 65), (9, 4, 1000), (1, 4, 32000),
         (3, 5, 32000), (2, 63, 515), (2, 2, 65537), (1, 7, 131071), (3, 3, 131073),
         (2, 1, 300007), (33, 5, 4099), (300, 2, 1030)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("b,draft,v", SIZES)
def test_sizes(b, draft, v, dtype):
    rng = np.random.default_rng(b * 1000 + draft * 10 + v)
    check(rng, b, draft, v, dtype, temperature=[1.0, 0.7, 1.6][v % 3])
    check(rng, b, draft, v, dtype, ragged=True, pad=[0, 1, 5, 64][draft % 4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [50, 5000, 40000])
def test_masks_and_edges(v, dtype):
    rng = np.random.default_rng(v)
    b, draft = 8, 3
    target = logits(rng, b * (draft + 1), v).reshape(b, draft + 1, v)
    drafts = target[:, :draft] + rng.normal(size=(b, draft, v)) * 0.5
    tokens = rng.integers(0, v, (b, draft))
    uniform = np.full((b, draft), 0.5)
    target[0, 1, tokens[0, 1]] = -INF       # an impossible token
    uniform[0] = 0.0
    target[1, 0] = -INF                     # the target leaves nothing
    drafts[2, 0] = -INF                     # the draft model left nothing: accepted
    target[3, :, v // 2:] = -INF            # banned words
    drafts[3, :, : v // 2] = -INF
    drafts[4] = target[4, :draft]           # equal models: every token accepted
    target[5, 0] = -INF
    target[5, 0, 3] = 1.0                   # one word left
    target[6] = 0.0                         # flat
    uniform[7] = [0.0, 1.0 - 2.0 ** -24, 0.0]
    check(rng, b, draft, v, dtype, target=target, drafts=drafts, tokens=tokens, uniform=uniform)


def test_rejection_where_the_residual_is_empty_samples_from_the_target():
    """A rejected token beside a residual without a positive entry (draft
    probabilities that are not a number) samples from the target's own."""
    dev = need_gpu()
    v = 1000
    target = torch.randn(1, 2, v, device=dev)
    drafts = torch.full((1, 1, v), math.nan, device=dev)
    noise = torch.empty(1, v, device=dev).exponential_()
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    plan = tk.VerifyPlan(1, 1, v, dtype=torch.float32)
    acc, out, _ = plan.execute(target, drafts, torch.zeros(1, 1, dtype=torch.int32, device=dev),
                               torch.zeros(1, 1, device=dev), noise, status=status)
    p = rows.softmax(target[0, 0].double().cpu().numpy())
    assert acc.tolist() == [0]
    assert out.tolist() == [[int(np.argmax(p / noise[0].double().cpu().numpy())), -1]]
    assert int(status.item()) == tk.STATUS_NAN


def test_ties_of_the_race_go_to_the_lower_word():
    dev = need_gpu()
    for v in (3, 70, 5000, 70001):
        target = torch.zeros(2, 2, v, device=dev)
        drafts = torch.zeros(2, 1, v, device=dev)
        noise = torch.full((2, v), 2.0, device=dev)
        noise[1, : v // 2] = 3.0
        tokens = torch.zeros(2, 1, dtype=torch.int32, device=dev)
        got = tk.verify_draft(target, drafts, tokens, torch.zeros(2, 1, device=dev), noise)
        assert got[0].tolist() == [1, 1]
        assert got[1].tolist() == [[0, 0], [0, v // 2]]


def test_token_out_of_range_is_rejected():
    dev = need_gpu()
    v = 9000
    target, drafts = torch.randn(3, 3, v, device=dev), torch.randn(3, 2, v, device=dev)
    tokens = torch.tensor([[v, 1], [-1, 1], [2 ** 31 - 1, 5]], dtype=torch.int32, device=dev)
    noise = torch.empty(3, v, device=dev).exponential_()
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    plan = tk.VerifyPlan(3, 2, v, dtype=torch.float32)
    announce("verify with tokens out of range")
    acc, out, _ = plan.execute(target, drafts, tokens, torch.zeros(3, 2, device=dev), noise,
                               status=status)
    assert acc.tolist() == [0, 0, 0] and int(status.item()) == tk.STATUS_INDEX_RANGE
    assert bool((out[:, 0] >= 0).all()) and bool((out[:, 1:] == -1).all())


def test_repeatable_fewer_sequences_and_other_stream():
    dev = need_gpu()
    v, draft = 32000, 4
    plan = tk.VerifyPlan(20, draft, v, dtype=torch.bfloat16)
    gen = torch.Generator(device=dev).manual_seed(3)
    target = (torch.randn(20, draft + 1, v, generator=gen, device=dev) * 3).bfloat16()
    drafts = target[:, :draft].contiguous()
    tokens = torch.randint(0, v, (20, draft), generator=gen, device=dev, dtype=torch.int32)
    uniform = torch.rand(20, draft, generator=gen, device=dev)
    noise = torch.empty(20, v, device=dev).exponential_(generator=gen)
    a = plan.execute(target, drafts, tokens, uniform, noise)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = plan.execute(target, drafts, tokens, uniform, noise, stream=s)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    for n in (1, 7):
        c = plan.execute(target[:n], drafts[:n], tokens[:n], uniform[:n], noise[:n])
        assert torch.equal(c[1], a[1][:n]) and torch.equal(c[0], a[0][:n])
    assert plan.execute(target[:0], drafts[:0], tokens[:0], uniform[:0], noise[:0])[0].shape == (0,)


def test_refusals():
    dev = need_gpu()
    plan = tk.VerifyPlan(2, 3, 50, dtype=torch.float32)
    ok = dict(target=torch.zeros(2, 4, 50, device=dev), drafts=torch.zeros(2, 3, 50, device=dev),
              tokens=torch.zeros(2, 3, dtype=torch.int32, device=dev),
              uniform=torch.zeros(2, 3, device=dev), noise=torch.ones(2, 50, device=dev))
    for kw in (dict(target=ok["target"].half()), dict(target=ok["drafts"]),
               dict(drafts=ok["drafts"][:1]), dict(tokens=ok["tokens"].long()),
               dict(uniform=ok["uniform"].double()), dict(noise=ok["noise"][:, :49]),
               dict(noise=ok["noise"].cpu()), dict(length=torch.zeros(2, device=dev)),
               dict(target=torch.zeros(3, 4, 50, device=dev))):
        with pytest.raises(ValueError):
            plan.execute(**{**ok, **kw})
    for args in ((0, 3, 50), (2, 0, 50), (2, 64, 50), (2, 3, 0), (65537, 3, 50)):
        with pytest.raises(tk.TkefError):
            tk.VerifyPlan(*args)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [300, 32000])
def test_masks_at_the_lowest_value_of_the_type(v, dtype):
    rng = np.random.default_rng(v + 3)
    low = -65504.0 if dtype == "f16" else float(torch.finfo(TYPES[dtype]).min)
    b, draft = 5, 2
    target = logits(rng, b * (draft + 1), v).reshape(b, draft + 1, v)
    drafts = target[:, :draft] + rng.normal(size=(b, draft, v)) * 0.5
    tokens = rng.integers(0, v, (b, draft))
    uniform = np.full((b, draft), 0.25)
    target[0] = low                          # uniform
    target[1, :, v // 2:] = low              # half the words masked in the target
    tokens[1, 0] = v - 1                     # such a word drafted
    drafts[2, :, : v // 2] = low
    target[3] = low
    target[3, :, 7] = 0.0                    # one word left
    drafts[4] = low                          # a uniform draft
    check(rng, b, draft, v, dtype, target=target, drafts=drafts, tokens=tokens, uniform=uniform)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("b,draft,v", [(600, 2, 1030), (40, 7, 70001), (530, 1, 9001)])
def test_many_places(b, draft, v, dtype):
    """Enough rows to leave those after a rejection unread."""
    rng = np.random.default_rng(b + v)
    check(rng, b, draft, v, dtype, temperature=0.9)
    check(rng, b, draft, v, dtype, ragged=True, pad=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [-1e9, -1e10, -1e30, -2e38])
@pytest.mark.parametrize("b,v", [(5, 300), (5, 32000), (350, 8191), (20, 140001)])
def test_masks_of_great_size(b, v, mask, dtype):
    rng = np.random.default_rng(v + 7)
    draft = 2
    target = logits(rng, b * (draft + 1), v).reshape(b, draft + 1, v)
    drafts = target[:, :draft] + rng.normal(size=(b, draft, v)) * 0.5
    tokens = rng.integers(0, v, (b, draft))
    uniform = np.full((b, draft), 0.25)
    target[0] = mask                         # uniform
    target[1, :, v // 8:] = mask             # most words masked in the target
    tokens[1, 0] = v - 1                     # such a word drafted
    drafts[2, :, : v // 2] = mask
    target[3] = mask
    target[3, :, 7] = 0.0                    # one word left
    drafts[4] = -mask                        # a uniform draft, as far above zero
    for temperature in (1.0, 0.8):
        check(rng, b, draft, v, dtype, temperature=temperature, target=target, drafts=drafts,
              tokens=tokens, uniform=uniform)
