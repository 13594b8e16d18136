"""Attention over the 8-bit cache against the formula in 64 bits: formats, head layouts, lengths, masks, refusals."""
import numpy as np
import pytest
import torch

from kv_util import Streams, check
from paper_2511_04477_b200 import binding as spqt

pytestmark = pytest.mark.gpu


def attend(st, q, accumulate=False, ws=None, **kw):
    qd = torch.from_numpy(q).cuda()
    ws = st.workspace(q.shape[2], q.shape[1]) if ws is None else ws
    out = spqt.spqt_kv_attention(st.cache, qd, ws, accumulate=accumulate, **kw)
    torch.cuda.synchronize()
    assert spqt.spqt_kv_status(ws) == 0
    return out


def compare(st, q, accumulate, scale=None, **kw):
    out = attend(st, q, accumulate, scale=scale, **kw)
    want, tol, got, got_tol = st.attention(q, scale)
    check(out, want, tol, "out")
    w = st.cache.weight.cpu().numpy().astype(np.float64)
    if accumulate:
        check(w, st.weight + got, got_tol, "weight")
    else:
        assert np.array_equal(w, st.weight)
    return out


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dim,bt", [(128, 32), (64, 16), (96, 64), (256, 128)])
def test_lengths_around_blocks_and_tiles(fmt, dim, bt):
    lengths = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, bt - 1, bt, bt + 1, 127, 128, 129, 200, 257]
    st = Streams(lengths, 2, dim, bt, fmt, seed=dim + bt)
    compare(st, st.queries(8, 1, seed=1, amplitude=2.0), accumulate=True)


@pytest.mark.parametrize("kv_heads,group,queries", [(1, 1, 1), (3, 2, 1), (2, 3, 1), (2, 4, 2), (1, 7, 1), (2, 8, 1), (1, 5, 3), (1, 16, 1), (2, 4, 5),
                                                    (1, 64, 1), (1, 64, 2), (1, 3, 16), (2, 1, 16)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_head_layouts_and_queries(kv_heads, group, queries, accumulate):
    st = Streams([0, 1, 3, 16, 40, 333], kv_heads, 128, 32, "int8", seed=10 * group + queries)
    compare(st, st.queries(kv_heads * group, queries, seed=2, amplitude=1.5), accumulate)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("group", [4, 8, 16])
def test_every_head_size_with_few_and_many_rows(fmt, dim, group):
    st = Streams([0, 33, 700], 2, dim, 32, fmt, seed=dim + group)
    compare(st, st.queries(2 * group, 1, seed=6), accumulate=True)


@pytest.mark.parametrize("fmt,dim,bt,group,queries", [("int8", 128, 32, 4, 1), ("e4m3", 128, 64, 8, 1), ("int8", 64, 16, 5, 2), ("int8", 256, 32, 16, 1), ("e4m3", 96, 128, 1, 1)])
def test_streams_that_many_ctas_share(fmt, dim, bt, group, queries):
    st = Streams([20011, 7, 4097], 2, dim, bt, fmt, seed=5)
    compare(st, st.queries(2 * group, queries, seed=3, amplitude=3.0), accumulate=True)


@pytest.mark.parametrize("fmt,dim,bt", [("int8", 128, 32), ("e4m3", 64, 16), ("int8", 96, 64), ("e4m3", 256, 128), ("e4m3", 128, 64), ("int8", 256, 16)])
@pytest.mark.parametrize("group,queries", [(16, 1), (3, 4), (8, 3), (5, 7)])
def test_many_rows_of_many_streams(fmt, dim, bt, group, queries):
    """More than sixteen streams: sixteen rows at a time, in one group or in several."""
    lengths = [0, 1, 2, 16, 17, 40, 130, 333, 500, 1025]
    st = Streams(lengths, 2, dim, bt, fmt, seed=group + queries)
    compare(st, st.queries(2 * group, queries, seed=7, amplitude=1.5), accumulate=True)


def test_offsets_beyond_32_bits():
    """The last blocks of a pool whose codes take more than 2^32 bytes, against the same contents in a small pool."""
    st = Streams([300], 1, 256, 128, "int8", seed=31)
    q = torch.from_numpy(st.queries(4, 1, seed=32)).cuda()
    small = spqt.spqt_kv_attention(st.cache, q, st.workspace(4), accumulate=True)
    c, far = st.cache, (1 << 32) // (128 * 256) + 64
    big = far + c.k_codes.shape[0]
    codes = [torch.empty((big, 128, 256), dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.full((big,), float("nan"), device="cuda") for _ in range(2)]
    weight = torch.zeros((big, 128), device="cuda")
    for to, of in zip(codes + scales, (c.k_codes, c.v_codes, c.k_scale, c.v_scale)):
        to[far:] = of
    weight[far:] = torch.from_numpy(st.weight).cuda()
    table = torch.where(c.table >= 0, c.table + far, c.table)
    other = spqt.KVCache(*codes, *scales, c.k_tail, c.v_tail, table, c.length, weight)
    ws = spqt.new_kv_workspace(other, 4)
    out = spqt.spqt_kv_attention(other, q, ws, accumulate=True)
    assert torch.equal(out, small) and torch.equal(weight[far:], c.weight) and torch.count_nonzero(weight[:far]) == 0
    k = [torch.zeros((1, 300, 1, 256), dtype=torch.float16, device="cuda") for _ in range(4)]
    spqt.spqt_kv_read(c, k[0], k[1], ws)
    spqt.spqt_kv_read(other, k[2], k[3], ws)
    assert torch.equal(k[0], k[2]) and torch.equal(k[1], k[3])
    new = torch.randn((1, 84, 1, 256), device="cuda").half()
    spqt.spqt_kv_append(other, new, new, ws)                # fills the block at the end of the pool
    assert spqt.spqt_kv_status(ws) == 0 and other.length.tolist() == [[384]]
    spqt.spqt_kv_read(other, k[0], k[1], ws)                # (the first 300 tokens)
    assert bool(((k[0][0, 256:300] - k[2][0, 256:300]).abs() <= k[2][0, 256:300].abs().max() * 2 ** -7 + new.abs().max() * 2 ** -7).all())


def test_two_calls_at_once():
    """On two streams with a workspace each, over one cache."""
    st = Streams([3000, 70], 2, 128, 32, "int8", seed=33)
    qs = [torch.from_numpy(st.queries(8, 1, seed=34 + i)).cuda() for i in range(2)]
    want = [spqt.spqt_kv_attention(st.cache, q, st.workspace(8)) for q in qs]
    ws = [st.workspace(8) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[], []]
    torch.cuda.synchronize()
    for _ in range(50):
        for i in range(2):
            outs[i].append(spqt.spqt_kv_attention(st.cache, qs[i], ws[i], stream=streams[i]))
            outs[i][-1].record_stream(streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in outs[i])


def test_a_workspace_for_several_shapes():
    """One workspace, the largest need, for caches of other shapes in turn; nothing of one call is left for the next."""
    sts = [Streams([2000, 5], 2, 128, 32, "int8", seed=35), Streams([900], 1, 64, 16, "e4m3", seed=36), Streams([4000] * 3, 3, 96, 64, "int8", seed=37)]
    ws = torch.zeros(max(st.workspace(16 * st.H, 2).numel() for st in sts), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        for st, q_heads, queries in zip(sts, (8, 16, 3), (2, 1, 2)):
            q = st.queries(q_heads, queries, seed=38)
            st.cache.weight.copy_(torch.from_numpy(st.weight))
            out = attend(st, q, True, ws=ws)
            want, tol, got, got_tol = st.attention(q)
            check(out, want, tol)
            check(st.cache.weight, st.weight + got, got_tol)


def test_more_streams_than_their_lengths_are_kept_of():
    rng = np.random.Generator(np.random.PCG64(9))
    lengths = rng.integers(0, 70, (420, 3)) * (rng.random((420, 3)) < 0.7)      # streams of their own lengths, many empty
    st = Streams(lengths, 3, 64, 16, "int8", seed=9)
    compare(st, st.queries(6, 1, seed=4), accumulate=True)


def test_nothing_to_see_at_all():
    st = Streams([0, 0, 0], 2, 128, 32, "int8", seed=1)
    out = compare(st, st.queries(8, 3, seed=4), accumulate=True)
    assert torch.count_nonzero(out) == 0


@pytest.mark.parametrize("amplitude,q_amplitude,scale", [(1e-4, 1.0, 1.0), (3000.0, 0.01, None), (1.0, 20.0, None), (1.0, 1.0, -0.3), (1.0, 1.0, 0.0)])
def test_magnitudes_and_scales(amplitude, q_amplitude, scale):
    """Blocks whose scales are far below and above one, peaked and flat probabilities."""
    st = Streams([100, 700], 2, 128, 32, "int8", seed=7, amplitude=amplitude)
    compare(st, st.queries(8, 1, seed=8, amplitude=q_amplitude), accumulate=True, scale=scale)


def test_one_token_that_outweighs_thousands_of_others():
    """The others hold a third of the weight, 2e-5 of the largest each: what 16 bits cannot hold of small probabilities must not be lost."""
    st = Streams([16384], 1, 128, 32, "int8", seed=11)
    q = st.queries(1, 1, seed=12, amplitude=0.2)
    k0 = st.kv[0, 0][0][0]
    q[0, 0, 0] += (k0 * (10.0 * 128 ** 0.5 / (k0 @ k0))).astype(np.float16)
    compare(st, q, accumulate=True)


def test_views_of_wider_rows():
    """q as the stacked linear leaves it, an output with strides of its own."""
    st = Streams([50, 3, 129], 2, 128, 32, "int8", seed=13)
    q = st.queries(8, 2, seed=14)
    wide = torch.full((3, 2, 8 + 4, 128), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, :, :8] = torch.from_numpy(q).cuda()
    out = torch.full((3, 5, 8 + 3, 128), 7.0, dtype=torch.float16, device="cuda")
    ws = st.workspace(8, 2)
    got = spqt.spqt_kv_attention(st.cache, wide[:, :, :8], ws, out=out[:, 1:3, :8])
    torch.cuda.synchronize()
    want, tol, _, _ = st.attention(q)
    check(got, want, tol)
    assert bool((out[:, 0] == 7).all() and (out[:, 3:] == 7).all() and (out[:, :, 8:] == 7).all())


def test_calls_repeat_bit_for_bit_and_in_a_graph():
    st = Streams([5000, 33, 900], 2, 128, 32, "int8", seed=15)
    q = torch.from_numpy(st.queries(8, 1, seed=16)).cuda()
    ws = st.workspace(8)
    first = spqt.spqt_kv_attention(st.cache, q, ws, accumulate=True)
    w1 = st.cache.weight.clone()
    out = torch.empty_like(first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        spqt.spqt_kv_attention(st.cache, q, ws, out=out)
    s.synchronize()
    assert torch.equal(out, first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        spqt.spqt_kv_attention(st.cache, q, ws, accumulate=True, out=out)
    out.zero_()
    st.cache.weight.copy_(torch.from_numpy(st.weight))
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first) and torch.equal(st.cache.weight, w1)
    # the recorded call reads lengths when it runs
    st.cache.length.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.count_nonzero(out) == 0


def test_a_block_that_is_not_a_number_reaches_those_who_see_it_only():
    """Queries of a speculative step: the last block holds a future token for the first of them."""
    st = Streams([64 + 1], 2, 128, 16, "int8", seed=17)
    q = st.queries(4, 1, seed=18)
    st.cache.v_scale[int(st.table[0, 1, 0])] = float("nan")
    out = attend(st, q).cpu().numpy()
    want, tol, _, _ = st.attention(q)
    check(out[:, :, :2].astype(np.float64), want[:, :, :2], tol[:, :, :2])
    assert np.isnan(out[:, :, 2:]).all()
    # sixteen queries and blocks of as many tokens: the first query sees one token of the last block, which holds not-a-number altogether
    st = Streams([64], 1, 128, 16, "int8", seed=19)
    st.cache.v_scale[int(st.table[0, 0, 3])] = float("nan")
    assert bool(torch.isnan(attend(st, st.queries(2, 16, seed=20))).all())
    st.cache.length.fill_(48)                # nobody sees it
    assert bool(torch.isfinite(attend(st, st.queries(2, 16, seed=20))).all())


def test_values_that_are_not_finite_in_the_open_block():
    """A future token's infinity or not-a-number stays with the queries that see it."""
    st = Streams([32 + 9], 1, 128, 32, "int8", seed=22)
    for value, seen in ((float("inf"), np.isposinf), (float("-inf"), np.isneginf), (float("nan"), np.isnan)):
        q = st.queries(3, 4, seed=23)
        st.cache.v_tail[0, 0, 7, 5] = value     # token 39 of 41: seen by the queries 2 (sees 40) and 3
        out = attend(st, q).cpu().numpy()
        want, tol, _, _ = st.attention(q)
        other = np.arange(128) != 5
        check(out[:, :, :, other].astype(np.float64), want[:, :, :, other], tol[:, :, :, other])
        check(out[:, :2, :, 5].astype(np.float64), want[:, :2, :, 5], tol[:, :2, :, 5])
        assert seen(out[:, 2:, :, 5]).all()
    st.cache.v_tail[0, 0, 7, 5] = 0.0
    st.cache.k_tail[0, 0, 8] = float("nan")      # a key of the last token
    out = attend(st, q).cpu().numpy()
    assert np.isfinite(out[:, :3]).all() and np.isnan(out[:, 3]).all()


def test_contents_that_are_refused():
    st = Streams([100, 40, 70], 2, 128, 32, "int8", seed=24)
    q = st.queries(8, 1, seed=25)
    want, tol, _, _ = st.attention(q)
    qd, ws = torch.from_numpy(q).cuda(), st.workspace(8)
    for bad in (-1, st.blocks, 1 << 30):
        st.cache.table.copy_(torch.from_numpy(st.table))
        st.cache.table[0, 1, 1] = bad
        out = spqt.spqt_kv_attention(st.cache, qd, ws, accumulate=True)
        assert spqt.spqt_kv_status(ws) == 3
        ws.zero_()
        got = out.cpu().numpy().astype(np.float64)
        assert np.isnan(got[0, 0, 4:]).all()
        check(got[0, 0, :4], want[0, 0, :4], tol[0, 0, :4])
        check(got[1:], want[1:], tol[1:])
    st.cache.table.copy_(torch.from_numpy(st.table))
    for bad in (-1, st.W * 32 + 1, 2 ** 31 - 1):
        st.cache.length[1, 0] = bad
        out = spqt.spqt_kv_attention(st.cache, qd, ws)
        assert spqt.spqt_kv_status(ws) == 3
        ws.zero_()
        got = out.cpu().numpy().astype(np.float64)
        assert (got[1, 0, :4] == 0).all()
        check(got[0], want[0], tol[0])
        check(got[1, 0, 4:], want[1, 0, 4:], tol[1, 0, 4:])


def test_arguments_that_are_refused():
    st = Streams([40], 2, 128, 32, "int8", seed=26, weight=False)
    q = torch.from_numpy(st.queries(8, 1, seed=27)).cuda()
    ws = st.workspace(8)
    for bad in (lambda: spqt.spqt_kv_attention(st.cache, q.float(), ws), lambda: spqt.spqt_kv_attention(st.cache, q.cpu(), ws),
                lambda: spqt.spqt_kv_attention(object(), q, ws)):
        with pytest.raises((TypeError, AttributeError)):
            bad()
    for bad in (q[:, :, :, :64], q[0], q.expand(2, 1, 8, 128), q[:, :, :, ::2]):
        with pytest.raises(ValueError):
            spqt.spqt_kv_attention(st.cache, bad, ws)
    for call, status in ((lambda: spqt.spqt_kv_attention(st.cache, q, ws, accumulate=True), 1),      # no weights are kept
                         (lambda: spqt.spqt_kv_attention(st.cache, q[:, :, :7], ws), 2),             # 7 heads on 2
                         (lambda: spqt.spqt_kv_attention(st.cache, q.transpose(1, 2), ws), 2),       # 8 tokens of one head
                         (lambda: spqt.spqt_kv_attention(st.cache, q.expand(1, 17, 8, 128), ws), 2),
                         (lambda: spqt.spqt_kv_attention(st.cache, q, ws[:1024]), 4),
                         (lambda: spqt.spqt_kv_attention(st.cache, torch.zeros(1032, dtype=torch.float16, device="cuda")[4:1028].view(1, 1, 8, 128), ws), 3)):
        before = spqt.spqt_launch_count()
        with pytest.raises(spqt.SpqtError) as e:
            call()
        assert e.value.status == status
        assert spqt.spqt_launch_count() == before


# A table for 65536 tokens a stream: the work is then divided among all CTAs, whatever the lengths are (the tests above have few and
# small streams, each of which a cluster of CTAs takes).
WIDE = 2048


@pytest.mark.parametrize("fmt,dim,group,queries", [("int8", 128, 4, 1), ("e4m3", 64, 8, 1), ("int8", 96, 3, 3), ("e4m3", 256, 5, 2)])
@pytest.mark.parametrize("lengths", [[0], [1], [0, 1, 31, 32, 33, 0], [70, 2500, 0, 16]])
def test_wide_tables(fmt, dim, group, queries, lengths):
    st = Streams(lengths, 2, dim, 32, fmt, seed=41 + dim, width=WIDE)
    compare(st, st.queries(2 * group, queries, seed=42, amplitude=2.0), accumulate=True)


def test_wide_and_narrow_tables_agree():
    """The same contents either way: within the tolerances of both, and rows of a table beyond a stream's blocks are not read."""
    for lengths in ([513], [40, 300], [65] * 16):
        st = [Streams(lengths, 1, 128, 32, "int8", seed=43, width=width) for width in (None, WIDE)]
        q = st[0].queries(4, 1, seed=44)
        outs = [compare(s, q, True).double() for s in st]
        _, tol, _, _ = st[0].attention(q)
        assert bool(((outs[0] - outs[1]).abs() <= 2 * torch.from_numpy(tol).cuda()).all())


def test_wide_tables_in_a_graph_and_on_two_streams():
    st = Streams([3000, 70], 2, 128, 32, "int8", seed=45, width=WIDE)
    qs = [torch.from_numpy(st.queries(8, 1, seed=46 + i)).cuda() for i in range(2)]
    ws = [st.workspace(8) for _ in range(2)]
    want = [spqt.spqt_kv_attention(st.cache, q, ws[0]) for q in qs]
    outs = [torch.zeros_like(w) for w in want]
    streams = [torch.cuda.Stream() for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.graph(graphs[i], stream=streams[i]):
            for _ in range(3):
                spqt.spqt_kv_attention(st.cache, qs[i], ws[i], out=outs[i])
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(outs[i], want[i]) for i in range(2))
    assert all(spqt.spqt_kv_status(w) == 0 for w in ws)
    with torch.cuda.stream(streams[0]):      # with weights: the lengths of the replay
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[0]):
            spqt.spqt_kv_attention(st.cache, qs[0], ws[0], accumulate=True, out=outs[0])
        g.replay()
    torch.cuda.synchronize()
    _, _, got, got_tol = st.attention(qs[0].cpu().numpy())
    check(st.cache.weight, st.weight + got, got_tol)
    st.cache.length.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.count_nonzero(outs[0]) == 0


def test_wide_tables_whose_contents_are_refused():
    st = Streams([100, 40, 70], 2, 128, 32, "int8", seed=47, width=WIDE)
    q = st.queries(8, 1, seed=48)
    want, tol, _, _ = st.attention(q)
    qd, ws = torch.from_numpy(q).cuda(), st.workspace(8)
    for bad in (-1, st.blocks, 1 << 30):
        st.cache.table.copy_(torch.from_numpy(st.table))
        st.cache.table[0, 1, 1] = bad
        got = spqt.spqt_kv_attention(st.cache, qd, ws, accumulate=True).cpu().numpy().astype(np.float64)
        assert spqt.spqt_kv_status(ws) == 3
        ws.zero_()
        assert np.isnan(got[0, 0, 4:]).all()
        check(got[0, 0, :4], want[0, 0, :4], tol[0, 0, :4])
        check(got[1:], want[1:], tol[1:])
    st.cache.table.copy_(torch.from_numpy(st.table))
    for bad in (-1, WIDE * 32 + 1, 2 ** 31 - 1):
        st.cache.length[1, 0] = bad
        got = spqt.spqt_kv_attention(st.cache, qd, ws).cpu().numpy().astype(np.float64)
        assert spqt.spqt_kv_status(ws) == 3
        ws.zero_()
        assert (got[1, 0, :4] == 0).all()
        check(got[0], want[0], tol[0])
        check(got[1, 0, 4:], want[1, 0, 4:], tol[1, 0, 4:])


def test_wide_tables_and_values_that_are_not_finite():
    st = Streams([64 + 1], 2, 128, 16, "int8", seed=49, width=2 * WIDE)
    q = st.queries(4, 1, seed=50)
    st.cache.v_scale[int(st.table[0, 1, 0])] = float("nan")
    out = attend(st, q).cpu().numpy()
    want, tol, _, _ = st.attention(q)
    check(out[:, :, :2].astype(np.float64), want[:, :, :2], tol[:, :, :2])
    assert np.isnan(out[:, :, 2:]).all()
    st = Streams([32 + 9], 1, 128, 32, "int8", seed=51, width=WIDE)
    q = st.queries(3, 4, seed=52)
    st.cache.v_tail[0, 0, 7, 5] = float("inf")     # token 39 of 41: seen by the queries 2 and 3
    st.cache.k_tail[0, 0, 8] = float("nan")        # a key of the last token: seen by the last query
    out = attend(st, q).cpu().numpy()
    want, tol, _, _ = st.attention(q)
    check(out[:, :2].astype(np.float64), want[:, :2], tol[:, :2])
    assert np.isposinf(out[:, 2, :, 5]).all() and np.isfinite(np.delete(out[:, 2], 5, -1)).all() and np.isnan(out[:, 3]).all()


def test_wide_tables_and_views():
    st = Streams([50, 3, 129], 2, 128, 32, "int8", seed=53, width=WIDE)
    q = st.queries(8, 2, seed=54)
    wide = torch.full((3, 2, 8 + 4, 128), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, :, :8] = torch.from_numpy(q).cuda()
    out = torch.full((3, 5, 8 + 3, 128), 7.0, dtype=torch.float16, device="cuda")
    got = spqt.spqt_kv_attention(st.cache, wide[:, :, :8], st.workspace(8, 2), out=out[:, 1:3, :8])
    torch.cuda.synchronize()
    want, tol, _, _ = st.attention(q)
    check(got, want, tol)
    assert bool((out[:, 0] == 7).all() and (out[:, 3:] == 7).all() and (out[:, :, 8:] == 7).all())


@pytest.mark.parametrize("fmt,dim,group,queries", [("int8", 128, 4, 1), ("e4m3", 128, 8, 1), ("int8", 64, 5, 2), ("e4m3", 96, 1, 1), ("int8", 256, 2, 4)])
@pytest.mark.parametrize("lengths", [[4001], [16000, 1, 0], [5000, 0, 31, 33, 127, 6001, 17]])
def test_few_streams_of_middling_tables(fmt, dim, group, queries, lengths):
    """One to seven streams whose tables hold 4000 to 18000 tokens: the largest clusters, where the device takes that many."""
    st = Streams(lengths, 1, dim, 32, fmt, seed=61 + dim)
    compare(st, st.queries(group, queries, seed=62, amplitude=2.0), accumulate=True)


@pytest.mark.parametrize("fmt,dim,bt", [("int8", 128, 32), ("e4m3", 64, 16), ("int8", 96, 64), ("e4m3", 256, 128)])
@pytest.mark.parametrize("group,queries", [(4, 1), (16, 1), (3, 4), (8, 3)])
def test_wide_tables_of_many_streams(fmt, dim, bt, group, queries):
    lengths = [0, 1, 2, 16, 17, 40, 130, 333, 500, 1025]
    st = Streams(lengths, 2, dim, bt, fmt, seed=65 + group, width=65536 // bt)
    compare(st, st.queries(2 * group, queries, seed=66, amplitude=1.5), accumulate=True)


@pytest.mark.parametrize("streams", [9, 16, 23, 34, 50, 75, 148, 149])
@pytest.mark.parametrize("fmt,dim,group,queries", [("int8", 128, 4, 1), ("e4m3", 64, 8, 2), ("int8", 256, 5, 3)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_numbers_of_streams(streams, fmt, dim, group, queries, accumulate):
    """Clusters of every size, down to one CTA, and one stream more than the device has SMs."""
    rng = np.random.Generator(np.random.PCG64(streams))
    lengths = rng.integers(0, 400, streams) * (rng.random(streams) < 0.9)
    lengths[0] = 500
    st = Streams(lengths, 1, dim, 32, fmt, seed=67 + streams)
    compare(st, st.queries(group, queries, seed=68, amplitude=2.0), accumulate)
