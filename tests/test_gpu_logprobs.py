"""Log probabilities of tokens, entropy and top alternatives against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2511_04477_b200 import binding as spqt

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def logits(rows, vocab, dtype, seed, spread=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((rows, vocab), generator=g, device="cuda") * spread
    return (x + 2.0 * (x / spread - 2.0).clamp(min=0) ** 2).to(TYPES[dtype])


def off(got, want):
    """How far, where both are -infinity not at all."""
    got = got.cpu().double()
    return torch.where(got == want, torch.zeros_like(want), (got - want).abs())


def check(x, tokens, top, got=None):
    """The sums are of positive terms, pairwise but for up to vocab / 512 / ctas of a thread: 2^-24 * 400 at most of the sum; an
    exponential is off by 2^-22 and by 2^-24 of its argument, which is 0 where it counts and below 2^7 elsewhere: 2^-17 with the
    term's share, which is below 2^-(argument).  Log probabilities: 2^-15 absolute and 2^-22 of the value.  Entropy, a difference of two
    such sums, the second of terms up to its value: 2^-15 and 2^-17 of it."""
    if got is None:
        got = spqt.spqt_token_logprobs(x, tokens, top=top)
    torch.cuda.synchronize()
    logprob, entropy, best, index = got
    d = x.double().cpu()
    lse = torch.logsumexp(d, 1, keepdim=True)
    logp = d - lse
    if tokens is not None:
        want = torch.gather(logp, 1, tokens.cpu().long()[:, None])[:, 0]
        err = off(logprob, want)
        assert bool((err <= 2.0 ** -15 + 2.0 ** -22 * want.abs()).all()), float(err.max())
    p = torch.exp(logp)
    want = -(p * torch.where(p > 0, logp, torch.zeros_like(p))).sum(1)
    if entropy is not None:
        err = (entropy.cpu().double() - want).abs()
        assert bool((err <= 2.0 ** -15 + 2.0 ** -17 * want).all()), float(err.max())
    order = torch.sort(d, dim=1, descending=True, stable=True)[1][:, :top]
    assert torch.equal(index.cpu().long(), order)
    want = torch.gather(logp, 1, order)
    if top:
        err = off(best, want)
        assert bool((err <= 2.0 ** -15 + 2.0 ** -22 * want.abs()).all()), float(err.max())


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (2, 31), (5, 257), (4, 512), (2, 1000), (3, 4097), (7, 32000), (1, 50257), (2, 128256), (300, 777), (900, 9001)])
def test_against_the_definition(dtype, rows, vocab):
    x = logits(rows, vocab, dtype, seed=rows + vocab)
    tokens = torch.randint(0, vocab, (rows,), device="cuda", dtype=torch.int32)
    check(x, tokens, min(vocab, 5))
    check(x, tokens, min(vocab, 32))
    check(x, tokens, 0)


@pytest.mark.parametrize("dtype,vocab", [("fp16", 1 << 20), ("fp32", 1 << 20), ("bf16", 700001)])
def test_rows_that_shared_memory_does_not_hold(dtype, vocab):
    x = logits(2, vocab, dtype, seed=3)
    check(x, torch.tensor([0, vocab - 1], dtype=torch.int32, device="cuda"), 32)


@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
@pytest.mark.parametrize("offset", [0, 1, 3, 7])
def test_rows_at_any_address(dtype, offset):
    wide = torch.full((6, 5003), float("nan"), dtype=TYPES[dtype], device="cuda")
    wide[:, offset:offset + 4096 + offset] = logits(6, 4096 + offset, dtype, seed=offset)
    x = wide[:, offset:offset + 4096 + offset]
    check(x, torch.zeros(6, dtype=torch.int32, device="cuda") + 4095, 20)


@pytest.mark.parametrize("vocab", [40, 3001, 32000, 128256])
@pytest.mark.parametrize("top", [1, 32])
def test_equal_logits(vocab, top):
    """All equal, and a few levels only: the lower places first, also where more of them are equal than a list would hold."""
    flat = torch.full((3, vocab), 1.5, dtype=torch.float16, device="cuda")
    flat[1] = (torch.arange(vocab, device="cuda") % 7).half()
    flat[2, ::2] = -float("inf")
    check(flat, torch.tensor([0, 1, 1], dtype=torch.int32, device="cuda"), top)


def test_sorted_rows():
    """The largest values side by side, in the hands of a few threads."""
    up = torch.linspace(-20, 20, 32768, device="cuda").repeat(2, 1)
    up[1] = up[1].flip(0)
    for t in (torch.float32, torch.float16):
        check(up.to(t), torch.tensor([5, 9], dtype=torch.int32, device="cuda"), 32)


def test_zeros_of_both_signs_are_equal():
    x = torch.full((1, 2000), -0.0, device="cuda")
    x[0, 100:] = 0.0
    check(x, None, 32)


def test_rows_and_tokens_without_a_probability():
    inf, nan = float("inf"), float("nan")
    x = logits(7, 5000, "fp32", seed=9)
    x[1, :] = -inf
    x[2, 17] = nan
    x[3, 4999] = inf
    x[4, 1:] = -inf
    tokens = torch.tensor([0, 0, 0, 0, 0, -1, 5000], dtype=torch.int32, device="cuda")
    logprob, entropy, best, index = (t.cpu() for t in spqt.spqt_token_logprobs(x, tokens, top=3))
    d = x.double().cpu()
    assert bool(torch.isnan(logprob[[1, 2, 3, 5, 6]]).all()) and bool(torch.isnan(entropy[[1, 2, 3]]).all()) and bool(torch.isnan(best[[1, 2, 3]]).all())
    assert abs(float(logprob[0] - (d[0, 0] - torch.logsumexp(d[0], 0)))) < 2 ** -15
    assert logprob[4] == 0 and entropy[4] == 0 and best[4, 0] == 0 and bool(torch.isneginf(best[4, 1:]).all())
    assert index[1].tolist() == [0, 1, 2] and index[4].tolist() == [0, 1, 2] and index[2, 0] == 17 and index[3, 0] == 4999
    assert bool(torch.isfinite(entropy[5:]).all()) and bool(torch.isfinite(best[5:]).all())
    lone = spqt.spqt_token_logprobs(x[:, :1], top=1, entropy=False)
    assert lone[0] is None and lone[1] is None and lone[3].flatten().tolist() == [0] * 7


def test_streams_graphs_and_repetition():
    x = logits(9, 60001, "bf16", seed=10)
    tokens = torch.arange(9, dtype=torch.int32, device="cuda")
    first = spqt.spqt_token_logprobs(x, tokens, top=8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        spqt.spqt_token_logprobs(x, tokens, top=8)
    s.synchronize()
    with torch.cuda.graph(g, stream=s):
        again = spqt.spqt_token_logprobs(x, tokens, top=8)
    g.replay()
    torch.cuda.synchronize()
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    x.copy_(logits(9, 60001, "bf16", seed=11))
    g.replay()
    check(x, tokens, 8, got=again)


def test_refusals():
    x = logits(2, 100, "fp16", seed=1)
    t = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (lambda: spqt.spqt_token_logprobs(x.cpu(), t), lambda: spqt.spqt_token_logprobs(x.double(), t), lambda: spqt.spqt_token_logprobs(x, t.long())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: spqt.spqt_token_logprobs(x[0], t), lambda: spqt.spqt_token_logprobs(x.T, None), lambda: spqt.spqt_token_logprobs(x, t[:1]),
                lambda: spqt.spqt_token_logprobs(x, t, top=-1)):
        with pytest.raises(ValueError):
            bad()
    before = spqt.spqt_launch_count()
    for kw, status in ((dict(top=101), 1), (dict(top=33), 2)):
        with pytest.raises(spqt.SpqtError) as e:
            spqt.spqt_token_logprobs(x, t, **kw)
        assert e.value.status == status
    empty = spqt.spqt_token_logprobs(x[:0], t[:0], top=4)
    assert [tuple(v.shape) for v in empty] == [(0,), (0,), (0, 4), (0, 4)]
    assert spqt.spqt_launch_count() == before


# Rows of a warp, of 128 threads, of 256, of a cluster: (rows, vocab) with 16-bit logits, with fp32.
SHAPES = {"warp": ((9, 1500), (9, 1500)), "team": ((9, 8000), (9, 4000)), "cta": ((301, 40000), (301, 20000)), "cluster": ((9, 128256), (9, 128256))}


def check_shifted(x, tokens, top):
    """As check, from logits less their row's maximum, which fp64 holds where x - log sum exp(x) has no digits left (x = -3.4e38).
    The kernel takes the same difference: log probabilities and entropy keep check's tolerances."""
    logprob, entropy, best, index = (t.cpu() for t in spqt.spqt_token_logprobs(x, tokens, top=top))
    d = x.double().cpu()
    order = torch.sort(d, dim=1, descending=True, stable=True)[1][:, :top]
    d = d - d.max(1, keepdim=True)[0]
    logp = d - torch.logsumexp(d, 1, keepdim=True)
    want = torch.gather(logp, 1, tokens.cpu().long()[:, None])[:, 0]
    assert bool((off(logprob, want) <= 2.0 ** -15 + 2.0 ** -22 * want.abs()).all()), (logprob, want)
    p = torch.exp(logp)
    want = -(p * torch.where(p > 0, logp, torch.zeros_like(p))).sum(1)
    assert bool(((entropy.double() - want).abs() <= 2.0 ** -15 + 2.0 ** -17 * want).all()), (entropy, want)
    assert torch.equal(index.long(), order)
    want = torch.gather(logp, 1, order)
    assert bool((off(best, want) <= 2.0 ** -15 + 2.0 ** -22 * want.abs()).all()), (best, want)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_logits_masked_with_the_lowest_values_of_the_type(dtype, shape):
    """Finite masks: what is masked has no share in the entropy, wherever the few ordinary values of a row are.  (A sum that has
    met only masked values moves to an ordinary maximum over a distance that times the sum's count has no finite value.)"""
    rows, vocab = SHAPES[shape][dtype == "fp32"]
    x = logits(rows, vocab, dtype, seed=41)
    lowest = torch.finfo(TYPES[dtype]).min
    second = lowest if dtype == "fp16" else -1e38
    masked = torch.full_like(x, lowest)
    masked[1::2] = second
    masked[2::5, ::3] = second
    masked[4::5, ::7] = -float("inf")
    g = torch.Generator(device="cuda")
    g.manual_seed(42)
    stays = torch.rand((rows, vocab), generator=g, device="cuda") < 0.01
    for row, where in ((0, slice(0, 6)), (1, slice(vocab // 2, vocab // 2 + 6)), (2, slice(vocab - 6, vocab)), (3, slice(vocab - 1, vocab)), (4, slice(0, 0)), (5, slice(0, 1))):
        stays[row] = False
        stays[row, where] = True
    x = torch.where(stays, x, masked)
    tokens = torch.full((rows,), vocab // 2, dtype=torch.int32, device="cuda")
    check_shifted(x, tokens, 5)
    check_shifted(x, tokens, 0)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_logits_further_apart_than_the_largest_value(dtype, shape):
    """The difference of two logits overflows: the lower ones have probability zero."""
    rows, vocab = SHAPES[shape][dtype == "fp32"]
    x = torch.full((rows, vocab), -3e38, dtype=TYPES[dtype], device="cuda")
    high = [0, vocab // 2, vocab - 1]
    for r in range(rows):
        x[r, high[:r % 3 + 1]] = 3e38
    logprob, entropy, best, index = spqt.spqt_token_logprobs(x, torch.zeros(rows, dtype=torch.int32, device="cuda"), top=3)
    want = torch.log(torch.arange(rows, device="cuda") % 3 + 1.0)
    # (equal terms: a logarithm, off by 2^-22 of it, and nothing else)
    assert not bool(torch.isnan(entropy).any()), entropy
    assert bool(((entropy - want).abs() <= 2.0 ** -20).all()) and bool(((logprob + want).abs() <= 2.0 ** -20).all())
    for r in range(rows):
        n = r % 3 + 1
        assert index[r, :n].tolist() == high[:n] and bool(((best[r, :n] + want[r]).abs() <= 2.0 ** -20).all()) and bool(torch.isneginf(best[r, n:]).all())


def test_as_many_rows_as_a_whole_number_counts():
    """2^31 - 1 rows of one value: every row is answered once, and nothing in front of the first or behind the last."""
    rows, far = 2 ** 31 - 1, 4096
    buf = torch.zeros(far + rows + far, dtype=torch.float16, device="cuda")
    odd = [0, 1, 4735, 4736, rows - 4737, rows - 4736, rows - 2, rows - 1]
    for r in odd:
        buf[far + r] = float("nan")
    out = torch.full((rows,), 7.0, device="cuda")       # (what the answers' memory holds, if they get this)
    del out
    entropy = spqt.spqt_token_logprobs(buf[far:far + rows].view(rows, 1))[1]
    assert entropy.shape == (rows,)
    found = []
    for at in range(0, rows, 1 << 28):
        part = entropy[at:at + (1 << 28)]
        nan = torch.isnan(part)
        found += (nan.nonzero().flatten() + at).tolist()
        assert bool((nan | (part == 0)).all())
    assert found == odd
    del buf, entropy, part, nan
    torch.cuda.empty_cache()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("top", [1, 20, 32])
def test_more_values_equal_to_the_bound_than_a_list_holds(dtype, shape, top):
    """Filtered logits: few values, or none, above those that are all alike; these in front, behind, everywhere or in a stretch, with a
    lower value elsewhere."""
    rows, vocab = SHAPES[shape][dtype == "fp32"]
    rows = max(rows, 12)
    g = torch.Generator(device="cuda")
    g.manual_seed(51)
    x = torch.empty((rows, vocab), dtype=TYPES[dtype], device="cuda")
    inf = float("inf")
    for r in range(rows):
        alike, lower = [(-inf, -inf), (-65504.0, -inf), (0.5, -3.0), (-0.0, -inf)][r % 4]
        x[r] = alike
        if r % 3 == 1:
            x[r, :vocab // 2] = lower                    # the equal ones at the end
        elif r % 3 == 2:
            x[r] = lower
            x[r, vocab // 3:2 * vocab // 3] = alike
        keep = [0, 1, 3, 19, 50, 200][r % 6]
        at = torch.randperm(vocab, generator=g, device="cuda")[:keep]
        x[r, at] = (torch.randn(keep, generator=g, device="cuda").abs() * 3 + 1).to(TYPES[dtype])
        if alike == -inf and keep == 0:
            x[r, vocab - 1] = 2.0
    x[3, 5] = 0.0                                        # a zero of the other sign is equal too
    check_shifted(x, torch.full((rows,), vocab - 1, dtype=torch.int32, device="cuda"), top)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
def test_more_values_above_the_bound_than_a_list_holds(dtype, shape):
    """The largest values all in the hands of a few threads, whose other maxima are low, so that the bound is low as well."""
    rows, vocab = SHAPES[shape][dtype == "fp32"]
    per = {"warp": 32, "team": 128, "cta": 256, "cluster": 512}[shape] * (16 if dtype == "fp16" else 8) // 2
    x = torch.full((rows, vocab), -1.0, dtype=TYPES[dtype], device="cuda")
    place = torch.arange(vocab, device="cuda")
    hands = (place % per) < (64 if shape != "warp" else 96)
    g = torch.Generator(device="cuda")
    g.manual_seed(52)
    x = torch.where(hands, torch.randn((rows, vocab), generator=g, device="cuda").to(TYPES[dtype]) * 2 + 9, x)
    x[:, 1::2] = torch.where(hands[1::2], x[:, 1::2], torch.full_like(x[:, 1::2], -2.0))
    for top in (5, 32):
        check_shifted(x, torch.zeros(rows, dtype=torch.int32, device="cuda"), top)
