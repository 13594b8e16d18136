"""Calls on another stream than the current one: what they make is that stream's.

Memory that a call makes may have been given back a moment before by a tensor of the current stream that work there still writes, and
goes to the current stream's next tensor when the result is dropped early.  Both are looked at with a current stream that is kept busy
for long enough that the call on the other one is through before."""
import pytest
import torch

from paper_2511_04477_b200 import binding as spqt

pytestmark = pytest.mark.gpu

BUSY = 200_000_000      # clock cycles: a tenth of a second


def a_linear(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    W = (torch.randn((1024, 2048), generator=g, device="cuda") * 0.05).half()
    return W, torch.randn(2048, generator=g, device="cuda").half()


def calls():
    """name -> (call with a stream or None, its outputs as a list)"""
    W, x = a_linear(1)
    p = spqt.spqt_pack(W)
    ws = spqt.new_workspace(p.m, p.n, 4, 128)
    X = torch.stack([x, x.flip(0)])
    bws = spqt.new_gemm_small_workspace(p)
    idx, count = spqt.spqt_sparsify(x, 0.5)
    kq = spqt.spqt_kq_pack(W)
    kws = spqt.new_kq_workspace(kq)
    rw = spqt.spqt_rowwise_pack(W)
    cache = spqt.KVCache.new(2, 2, 64, 16, 64, 16)
    cache.table.copy_(torch.arange(64, dtype=torch.int32).view(2, 2, 16))
    aws = spqt.new_kv_workspace(cache, 8)
    kv = [torch.randn((2, 100, 2, 64), device="cuda").half() for _ in range(2)]
    spqt.spqt_kv_append(cache, *kv, aws)
    q = torch.randn((2, 1, 8, 64), device="cuda").half()
    logits, tokens = torch.randn((4, 5000), device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda")

    def collected(s):
        y, i, c = spqt.spqt_sparsify_gemv(p, x, 0.5, ws, stream=s)
        return [y, c]

    def packed(s):
        n = spqt.spqt_pack(W, stream=s)
        return [n.codes, n.scale_zero]

    def batch(s):
        y, i, c = spqt.spqt_sparse_gemm_small(p, X, 0.5, bws, stream=s)
        return [y, c]
    return {
        "kv_attention": lambda s: [spqt.spqt_kv_attention(cache, q, aws, stream=s)],
        "token_logprobs": lambda s: list(spqt.spqt_token_logprobs(logits, tokens, top=4, stream=s)),
        "sparsify": lambda s: list(spqt.spqt_sparsify(x, 0.5, stream=s))[1:],
        "sparse_gemv": lambda s: [spqt.spqt_sparse_gemv(p, x, idx, count, ws, stream=s)],
        "sparsify_gemv": collected,
        "dense_gemv": lambda s: [spqt.spqt_dense_gemv(p, x, ws, stream=s)],
        "sparse_gemm_small": batch,
        "dense_gemm_small": lambda s: [spqt.spqt_dense_gemm_small(p, X, bws, stream=s)],
        "kq_dense_gemv": lambda s: [spqt.spqt_kq_dense_gemv(kq, x, kws, stream=s)],
        "pack": packed,
        "kq_pack": lambda s: [spqt.spqt_kq_pack(W, stream=s).records],
        "unpack": lambda s: [spqt.spqt_unpack(p, stream=s)],
        "rowwise_pack": lambda s: [spqt.spqt_rowwise_pack(W, stream=s).codes],
        "rowwise_dense_gemv": lambda s: [spqt.spqt_rowwise_dense_gemv(rw, x, stream=s)],
        "rowwise_thresholded_gemv": lambda s: [spqt.spqt_rowwise_thresholded_gemv(rw, x, 0.5, stream=s)],
        "calibrate_threshold": lambda s: [spqt.spqt_calibrate_threshold(x, 0.5, stream=s)],
    }


NAMES = ["kv_attention", "token_logprobs", "sparsify", "sparse_gemv", "sparsify_gemv", "dense_gemv", "sparse_gemm_small", "dense_gemm_small", "kq_dense_gemv", "pack",
         "kq_pack", "unpack", "rowwise_pack", "rowwise_dense_gemv", "rowwise_thresholded_gemv", "calibrate_threshold"]


@pytest.fixture(scope="module")
def made():
    c = calls()
    assert sorted(c) == sorted(NAMES)
    return c


def given_back(outs):
    """Tensors of the outputs' sizes whose memory the current stream's pool has again while work of the current stream writes it."""
    held = [torch.empty_like(o) for o in outs]
    torch.cuda._sleep(BUSY)
    for h in held:
        h.fill_(9)


@pytest.mark.parametrize("name", NAMES)
def test_outputs_do_not_lie_where_the_current_stream_still_writes(made, name):
    call = made[name]
    want = [o.clone() for o in call(None)]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    given_back(want)
    got = call(other)
    assert not torch.cuda.current_stream().query()      # (it is still busy)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b), name


@pytest.mark.parametrize("name", NAMES)
def test_outputs_that_are_dropped_early_are_not_given_to_the_current_stream(made, name):
    call = made[name]
    like = [o.clone() for o in call(None)]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        torch.cuda._sleep(BUSY)
    call(other)                                          # (the result goes at once)
    fresh = [torch.zeros_like(o) for o in like for _ in range(2)]
    torch.cuda.current_stream().synchronize()
    assert not other.query()
    torch.cuda.synchronize()
    for f in fresh:
        assert not bool(f.view(torch.uint8).any()), name


@pytest.mark.parametrize("name", NAMES)
def test_outputs_may_be_read_on_the_current_stream_and_dropped(made, name):
    """Where the current stream waits for the other one, reads the result and drops it, the other stream's next call leaves the memory
    alone until that is read."""
    call = made[name]
    want = [o.clone() for o in call(None)]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(other)
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda._sleep(BUSY)
    copies = [g.clone() for g in got]
    del got
    with torch.cuda.stream(other):
        junk = [torch.full_like(w, 9) for w in want for _ in range(2)]
    other.synchronize()
    assert not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    for a, b in zip(copies, want):
        assert torch.equal(a, b), name
    del junk


def test_on_the_default_stream_from_another():
    """The default stream has no handle of its own."""
    made_ = calls()
    side = torch.cuda.Stream()
    default = torch.cuda.default_stream()
    side.wait_stream(default)
    for name in ("kv_attention", "token_logprobs", "rowwise_dense_gemv", "calibrate_threshold"):
        want = [o.clone() for o in made_[name](None)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            got = made_[name](default)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name
