"""Appending to the 8-bit cache, reading it back and evicting from it, against a restatement in 64 bits."""
import numpy as np
import pytest
import torch

from kv_util import DTYPE, E4M3, Streams, from_codes, to_codes
from paper_2511_04477_b200 import binding as spqt

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def raw(t):
    return t.view(torch.uint8).cpu().numpy()


def fresh_rows(st, tokens, seed, amplitude=1.0):
    rng = np.random.Generator(np.random.PCG64(seed))
    return (amplitude * rng.standard_normal((2, st.B, tokens, st.H, st.D))).astype(np.float16)


def with_blocks(lengths, new, kv_heads, dim, bt, fmt, seed, **kw):
    """A cache whose streams own the blocks for `new` more tokens."""
    st = Streams(lengths, kv_heads, dim, bt, fmt, seed, **kw)
    need = -(-(st.n + new) // bt)
    extra = need - -(-st.n // bt)
    old = st.blocks
    blocks = old + int(extra.sum())
    W = int(need.max())
    table = np.full((st.B, st.H, W), -7, dtype=np.int32)
    at = old
    for b in range(st.B):
        for h in range(st.H):
            have = -(-int(st.n[b, h]) // bt)
            table[b, h, :have] = st.table[b, h, :have]
            table[b, h, have:need[b, h]] = np.arange(at, at + extra[b, h])
            at += int(extra[b, h])
    grow = lambda t: torch.cat([t, torch.zeros((blocks - old,) + t.shape[1:], dtype=t.dtype, device="cuda")])
    codes = lambda t: grow(t.view(torch.uint8)).view(t.dtype)
    c = st.cache
    weight = torch.full((blocks, bt), 5.0, device="cuda") if c.weight is not None else None
    st.cache = spqt.KVCache(codes(c.k_codes), codes(c.v_codes), grow(c.k_scale), grow(c.v_scale), c.k_tail, c.v_tail, dev(table), c.length, weight)
    st.table, st.W, st.blocks = table, W, blocks
    return st


def appended(st, kv, counts):
    """What the cache has to hold: per stream the code bytes, scales and tails; codes and tails of each kind and stream."""
    want = {}
    for b in range(st.B):
        for h in range(st.H):
            n, c, bt = int(st.n[b, h]), int(counts[b]), st.bt
            first = n // bt
            for k, tail in enumerate((st.tails[0], st.tails[1])):
                rows = np.concatenate([tail[b, h, :n - first * bt], kv[k, b, :c, h]])
                full = len(rows) // bt
                codes, scale = to_codes(rows[:full * bt].reshape(full, bt, st.D), st.fmt) if full else (None, None)
                want[k, b, h] = (first, full, codes, scale, rows[full * bt:])
    return want


def check_append(st, kv, counts, length_out=None, device_counts=None):
    st.tails = [st.cache.k_tail.cpu().numpy(), st.cache.v_tail.cpu().numpy()]
    ws = st.workspace(st.H)
    before = [raw(st.cache.k_codes), raw(st.cache.v_codes)]
    scales = [st.cache.k_scale.cpu().numpy(), st.cache.v_scale.cpu().numpy()]
    want = appended(st, kv, counts)
    k, v = (dev(x) for x in kv)
    length = spqt.spqt_kv_append(st.cache, k, v, ws, counts=device_counts, length_out=length_out)
    torch.cuda.synchronize()
    assert spqt.spqt_kv_status(ws) == 0
    c = st.cache
    codes, scale, tail = (raw(c.k_codes), raw(c.v_codes)), (c.k_scale.cpu().numpy(), c.v_scale.cpu().numpy()), (c.k_tail.cpu().numpy(), c.v_tail.cpu().numpy())
    touched = np.zeros(st.blocks, dtype=bool)
    for (kind, b, h), (first, full, want_codes, want_scale, rows) in want.items():
        ids = st.table[b, h, first:first + full]
        touched[ids] = True
        if full:
            assert np.array_equal(scale[kind][ids], want_scale, equal_nan=True)
            assert np.array_equal(codes[kind][ids], want_codes)
        assert np.array_equal(tail[kind][b, h, :len(rows)].view(np.uint16), rows.view(np.uint16))
    for kind in range(2):                      # nothing else has changed
        assert np.array_equal(codes[kind][~touched], before[kind][~touched])
        assert np.array_equal(scale[kind][~touched], scales[kind][~touched], equal_nan=True)
    new = st.n + np.asarray(counts)[:, None]
    assert np.array_equal(length.cpu().numpy(), new)
    if c.weight is not None:
        w = np.full((st.blocks, st.bt), 5.0)
        for b in range(st.B):
            for h in range(st.H):
                t = np.arange(st.n[b, h], new[b, h])
                w[st.table[b, h, t // st.bt], t % st.bt] = 0.0
        assert np.array_equal(c.weight.cpu().numpy(), w)
    return ws


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dim,bt", [(128, 32), (64, 16), (96, 16), (96, 64), (128, 128), (256, 128), (256, 16)])
@pytest.mark.parametrize("tokens", [1, 5, 133])
def test_append(fmt, dim, bt, tokens):
    st = with_blocks([0, 1, bt - 1, bt, bt + 1, 2 * bt + bt // 2], tokens, 3, dim, bt, fmt, seed=dim + bt + tokens)
    check_append(st, fresh_rows(st, tokens, seed=tokens), [tokens] * st.B)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_of_a_padded_batch(fmt):
    st = with_blocks([0, 3, 40, 64, 31], 100, 2, 128, 32, fmt, seed=3)
    counts = [100, 0, 1, 64, 33]
    kv = fresh_rows(st, 100, seed=4)
    for b, c in enumerate(counts):
        kv[:, b, c:] = np.nan                  # padding
    old = st.cache.length.clone()
    out = torch.full((5, 2), -1, dtype=torch.int32, device="cuda")
    check_append(st, kv, counts, length_out=out, device_counts=torch.tensor(counts, dtype=torch.int32, device="cuda"))
    assert torch.equal(st.cache.length, old)


def test_append_where_the_rounding_is_hardest():
    """Quotients at ties and next to them: a scale that is a power of two makes exact ties, others near ones; tiny and huge rows."""
    for fmt, top in (("int8", 127.0), ("e4m3", 448.0)):
        st = with_blocks([0] * 6, 32, 1, 128, 32, fmt, seed=5)
        kv = fresh_rows(st, 32, seed=6)
        grid = np.arange(32 * 128).reshape(32, 128)
        kv[:, 0, :, 0] = (grid % 255 - 127) / 2.0                       # halves
        kv[:, 0, 0, 0, 0] = top
        kv[:, 1, :, 0] = (grid % 4096).astype(np.uint16).view(np.float16) * np.float16(1.0)   # subnormal and small numbers
        kv[:, 2] = np.float16(65504.0)
        kv[:, 3] = 0.0
        kv[:, 3, 1] = -0.0
        kv[:, 4, :, 0] = np.linspace(-448, 448, 32 * 128).reshape(32, 128)
        kv[:, 5, :, 0] = (np.random.Generator(np.random.PCG64(1)).integers(0, 0x7c00, (32, 128)).astype(np.uint16)).view(np.float16)   # every magnitude
        check_append(st, kv.astype(np.float16), [32] * 6)


def test_append_of_values_that_are_not_finite():
    st = with_blocks([0, 20], 40, 2, 128, 32, "int8", seed=7)
    kv = fresh_rows(st, 40, seed=8)
    kv[0, 0, 3, 0, 17] = np.inf
    kv[1, 1, 5, 1, 0] = np.nan
    kv[0, 1, 39, 0, 2] = -np.inf              # stays in the tail
    ws = check_append(st, kv, [40, 40])
    scale = st.cache.k_scale.cpu().numpy()
    assert np.isnan(scale[st.table[0, 0, 0]]) and np.isfinite(scale[st.table[0, 1, 0]])
    k = torch.zeros((2, 60, 2, 128), dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    spqt.spqt_kv_read(st.cache, k, v, ws)
    assert bool(torch.isnan(k[0, :32, 0]).all()) and bool(torch.isfinite(k[0, 32:40, 0]).all()) and bool(torch.isfinite(k[0, :40, 1]).all())
    assert bool(torch.isneginf(k[1, 59, 0, 2]))


def test_tokens_one_by_one_give_what_a_prompt_gives():
    kv = None
    held = []
    for steps in ([70], [1] * 70, [5, 27, 1, 36, 1]):
        st = with_blocks([0, 9], 70, 2, 64, 32, "e4m3", seed=9)
        kv = fresh_rows(st, 70, seed=10)
        ws, at = st.workspace(2), 0
        k, v = (dev(x) for x in kv)
        for n in steps:
            spqt.spqt_kv_append(st.cache, k[:, at:at + n], v[:, at:at + n], ws)
            at += n
        out = [torch.full((2, 79, 2, 64), 3.0, dtype=torch.float16, device="cuda") for _ in range(2)]
        spqt.spqt_kv_read(st.cache, out[0], out[1], ws)
        assert spqt.spqt_kv_status(ws) == 0
        assert st.cache.length.tolist() == [[70, 70], [79, 79]]
        held.append(torch.stack(out))
    assert torch.equal(held[0], held[1]) and torch.equal(held[0], held[2])


def test_append_in_a_graph_advances_with_every_replay():
    st = with_blocks([30, 0], 8, 2, 128, 32, "int8", seed=11)
    k, v = (dev(x) for x in fresh_rows(st, 1, seed=12))
    ws = st.workspace(2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        spqt.spqt_kv_append(st.cache, k, v, ws)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        spqt.spqt_kv_append(st.cache, k, v, ws)
    for i in range(6):
        k.fill_(float(i))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
    assert st.cache.length.tolist() == [[37, 37], [7, 7]]
    out = torch.zeros((2, 37, 2, 128), dtype=torch.float16, device="cuda")
    spqt.spqt_kv_read(st.cache, out, torch.zeros_like(out), ws)
    assert out[1, 1:7, 0, 0].tolist() == [0, 1, 2, 3, 4, 5] and out[0, 32:37, 1, 9].tolist() == [1, 2, 3, 4, 5]


def test_streams_that_cannot_take_the_tokens_stay_as_they_were():
    def untouched(st, before, stream):
        b, h = stream
        c = st.cache
        assert np.array_equal(raw(c.k_codes), before[0]) and np.array_equal(c.k_scale.cpu().numpy(), before[1], equal_nan=True)
        assert np.array_equal(c.k_tail[b, h].cpu().numpy().view(np.uint16), before[2][b, h].view(np.uint16))
        assert np.array_equal(c.weight.cpu().numpy(), before[3])

    for what in ("full", "block", "later block", "negative length", "count"):
        st = with_blocks([40], 60, 1, 128, 32, "int8", seed=13)
        tokens = 60
        counts = torch.tensor([tokens], dtype=torch.int32, device="cuda")
        if what == "full":
            tokens = st.W * 32 - 40 + 1
            counts[0] = tokens
        elif what == "block":
            st.cache.table[0, 0, 1] = st.blocks
        elif what == "later block":
            st.cache.table[0, 0, 3] = -1
        elif what == "negative length":
            st.cache.length[0, 0] = -5
        else:
            counts[0] = 61
        c = st.cache
        before = [raw(c.k_codes), c.k_scale.cpu().numpy(), c.k_tail.cpu().numpy(), c.weight.cpu().numpy()]
        old = c.length.clone()
        k, v = (dev(x) for x in fresh_rows(st, tokens, seed=14))
        ws = st.workspace(1)
        spqt.spqt_kv_append(c, k, v, ws, counts=counts)
        assert spqt.spqt_kv_status(ws) == 3, what
        untouched(st, before, (0, 0))
        assert torch.equal(c.length, old), what


@pytest.mark.parametrize("fmt,dim,bt", [("int8", 128, 32), ("e4m3", 64, 16), ("int8", 96, 64), ("e4m3", 256, 128)])
def test_read(fmt, dim, bt):
    st = Streams([0, 1, bt, 2 * bt + 5, 100], 3, dim, bt, fmt, seed=15)
    T = int(st.n.max()) + 4
    ws = st.workspace(3)
    wide = torch.full((2, st.B, 3 + 1, T, dim), 9.0, dtype=torch.float16, device="cuda")     # heads in front of tokens
    k, v = wide[0, :, :3].transpose(1, 2), wide[1, :, :3].transpose(1, 2)
    spqt.spqt_kv_read(st.cache, k, v, ws)
    assert spqt.spqt_kv_status(ws) == 0
    got = wide.cpu().numpy()
    for (b, h), rows in st.kv.items():
        n = int(st.n[b, h])
        for kind in range(2):
            # the product of a code and a scale, 24 + 8 bits, is rounded to fp32 and then to fp16
            want = rows[kind].astype(np.float32).astype(np.float16)
            assert np.array_equal(got[kind, b, h, :n], want)
            assert (got[kind, b, h, n:] == 9).all()
    assert (got[:, :, 3] == 9).all()
    few = torch.full((st.B, 7, 3, dim), 9.0, dtype=torch.float16, device="cuda")
    spqt.spqt_kv_read(st.cache, few, torch.empty_like(few), ws, length=st.cache.length)
    full = wide[0, :, :3].transpose(1, 2)[:, :7]
    assert torch.equal(few, full)


# ---------------------------------------------------------------- eviction


def evicted(row, w, n, bt, keep, first, recent):
    closed = n // bt
    if closed <= keep:
        return list(row), n
    score = [np.float32(w[i].astype(np.float64).sum()) for i in row[:closed]]
    inner = sorted(range(first, closed - recent), key=lambda j: (-np.inf if np.isnan(score[j]) else -score[j], j))
    nan = [j for j in range(first, closed - recent) if np.isnan(score[j])]
    inner = nan + [j for j in inner if j not in nan]
    stay = set(inner[:keep - first - recent]) | set(range(first)) | set(range(closed - recent, closed))
    some = [closed] if n % bt else []
    order = sorted(stay) + some + [j for j in range(closed) if j not in stay] + list(range(closed + len(some), len(row)))
    return [row[j] for j in order], keep * bt + n % bt


def plain_cache(lengths, heads, bt, width, seed, weight):
    """A cache of which only the table, the lengths and the weights matter."""
    rng = np.random.Generator(np.random.PCG64(seed))
    B, blocks = len(lengths), len(lengths) * heads * width
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    c = spqt.KVCache.new(B, heads, 64, bt, blocks, width, weight=True)
    c.table.copy_(dev(rng.permutation(blocks).astype(np.int32).reshape(B, heads, width)))
    c.length.copy_(n[:, None] if n.dim() == 1 else n)
    w = weight(rng, (blocks, bt)).astype(np.float32)
    c.weight.copy_(dev(w))
    return c, w


def check_evict(c, w, keep, first, recent, in_place=False):
    bt = c.k_codes.shape[1]
    table, length = c.table.cpu().numpy(), c.length.cpu().numpy()
    ws = spqt.new_kv_workspace(c, c.table.shape[1])
    outs = {} if in_place else {"table_out": torch.full_like(c.table, -9), "length_out": torch.full_like(c.length, -9)}
    got_table, got_length = spqt.spqt_kv_evict(c, keep, ws, first=first, recent=recent, **outs)
    assert spqt.spqt_kv_status(ws) == 0
    if not in_place:
        assert np.array_equal(c.table.cpu().numpy(), table) and np.array_equal(c.length.cpu().numpy(), length)
    got_table, got_length = got_table.cpu().numpy(), got_length.cpu().numpy()
    for b in range(table.shape[0]):
        for h in range(table.shape[1]):
            row, n = evicted(table[b, h], w, int(length[b, h]), bt, keep, first, recent)
            assert got_length[b, h] == n
            assert got_table[b, h].tolist() == [int(i) for i in row], (b, h, int(length[b, h]))


HEAVY = lambda rng, shape: np.exp(3 * rng.standard_normal(shape))


@pytest.mark.parametrize("bt", [16, 32, 64, 128])
@pytest.mark.parametrize("keep,first,recent", [(0, 0, 0), (1, 0, 0), (1, 1, 0), (4, 1, 2), (5, 0, 5), (7, 3, 4), (100, 1, 1)])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(bt, keep, first, recent, in_place):
    lengths = [0, 1, bt - 1, bt, bt + 1, 4 * bt, 5 * bt + 3, 8 * bt - 1, 19 * bt, 20 * bt]
    c, w = plain_cache(lengths, 2, bt, 20, seed=keep + bt, weight=HEAVY)
    check_evict(c, w, keep, first, recent, in_place)


@pytest.mark.parametrize("kind", ["heavy", "equal", "few values", "zeros and signs", "not finite"])
@pytest.mark.parametrize("width", [1, 600, 1500, 4096])
def test_evict_of_long_rows_and_equal_weights(kind, width):
    def weight(rng, shape):
        if kind == "heavy":
            return HEAVY(rng, shape)
        if kind == "equal":
            return np.ones(shape)
        if kind == "few values":
            return np.repeat(rng.integers(0, 3, (shape[0], 1)), shape[1], 1)
        if kind == "zeros and signs":
            return np.where(rng.random((shape[0], 1)) < 0.5, -0.0, rng.integers(-1, 2, shape))
        w = HEAVY(rng, shape)
        w[rng.random(shape[0]) < 0.1, 3] = np.nan
        w[rng.random(shape[0]) < 0.1, 5] = np.inf
        return w
    bt = 16
    lengths = [width * bt, max(0, width * bt - 5), width * bt // 2 + 1]
    c, w = plain_cache(lengths, 1, bt, width, seed=width, weight=weight)
    for keep, first, recent in ((width // 3, min(1, width // 3), min(width // 3, 2) // 2), (max(1, width - 1), 0, 0)):
        check_evict(c, w, keep, first, recent)


@pytest.mark.parametrize("width", [5119, 6143, 6144, 16384])
def test_evict_of_the_longest_rows(width):
    """Rows for which a CTA needs more shared memory than it has without asking."""
    c, w = plain_cache([width * 16, width * 16 - 1], 1, 16, width, seed=width, weight=HEAVY)
    check_evict(c, w, width // 2 + 1, 2, 3)


@pytest.mark.parametrize("inner", [511, 512, 513, 2047, 2048, 2049])
def test_evict_around_the_sizes_of_the_search(inner):
    """As many blocks to choose among as one warp's registers, or four warps', hold, one fewer and one more."""
    few = lambda rng, shape: np.repeat(rng.integers(0, 5, (shape[0], 1)), shape[1], 1)
    for weight in (HEAVY, few):
        c, w = plain_cache([(inner + 5) * 32, (inner + 5) * 32 + 7, (inner + 4) * 32 + 31], 1, 32, inner + 6, seed=inner, weight=weight)
        for keep in (6, 5 + inner // 2, 5 + inner - 2):
            check_evict(c, w, keep, 2, 3)


def test_evict_refuses():
    c, w = plain_cache([40], 1, 16, 4, seed=1, weight=HEAVY)
    ws = spqt.new_kv_workspace(c, 1)
    for args in ((-1, 0, 0), (2, 2, 1), (2, -1, 0), (2, 0, -1), (2, 2 ** 31 - 1, 2 ** 31 - 1)):
        with pytest.raises(spqt.SpqtError) as e:
            spqt.spqt_kv_evict(c, args[0], ws, first=args[1], recent=args[2])
        assert e.value.status == 1
    with pytest.raises(ValueError):
        spqt.spqt_kv_evict(c, 1, ws, table_out=torch.zeros((1, 1, 3), dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        spqt.spqt_kv_evict(c, 1, ws, length_out=torch.zeros((1, 1), device="cuda"))
    # contents: a length that the row cannot hold, a block outside the pool
    c.length[0, 0] = 4 * 16 + 1
    table = c.table.clone()
    spqt.spqt_kv_evict(c, 1, ws)
    assert spqt.spqt_kv_status(ws) == 3 and torch.equal(c.table, table) and c.length.tolist() == [[65]]
    ws.zero_()
    c.length[0, 0] = 64
    c.table[0, 0, 2] = 4
    spqt.spqt_kv_evict(c, 3, ws)
    assert spqt.spqt_kv_status(ws) == 3 and c.table[0, 0].tolist() == [table[0, 0, 0].item(), table[0, 0, 1].item(), table[0, 0, 3].item(), 4]


def test_cache_objects_refuse_what_does_not_fit():
    c = spqt.KVCache.new(2, 3, 64, 16, 10, 4, weight=True)
    parts = {n: getattr(c, n) for n in spqt.KVCache.TENSORS}
    for name, bad, error in (("v_codes", c.k_codes.view(torch.uint8).view(torch.float8_e4m3fn), TypeError), ("k_scale", c.k_scale[:9], ValueError),
                             ("k_tail", c.k_tail.float(), TypeError), ("length", c.length.long(), TypeError), ("table", c.table[0], TypeError),
                             ("weight", c.weight[:, :8], ValueError), ("v_tail", c.v_tail.transpose(0, 1), ValueError), ("k_scale", c.k_scale.cpu(), TypeError)):
        with pytest.raises(error):
            spqt.KVCache(**{**parts, name: bad})
    with pytest.raises(AttributeError):
        c.table = c.table
    with pytest.raises(spqt.SpqtError) as e:
        spqt.new_kv_workspace(spqt.KVCache.new(1, 1, 80, 16, 1, 1), 1)
    assert e.value.status == 2
    with pytest.raises(spqt.SpqtError) as e:
        spqt.new_kv_workspace(spqt.KVCache.new(1, 1, 64, 24, 1, 1), 1)
    assert e.value.status == 2


def test_more_tokens_or_rows_than_a_whole_number_counts_are_refused():
    """Views of one row; an error, with the interpreter's lock held when it is raised."""
    c, w = plain_cache([70], 1, 16, 6, seed=2, weight=HEAVY)
    ws = spqt.new_kv_workspace(c, 1)
    row = torch.zeros((1, 1, 1, 64), dtype=torch.float16, device="cuda")
    many = row.expand(1, 2 ** 31, 1, 64)
    before = spqt.spqt_launch_count()
    for call in (lambda: spqt.spqt_kv_append(c, many, many, ws), lambda: spqt.spqt_kv_read(c, many, many, ws), lambda: spqt.spqt_kv_attention(c, many, ws, out=row),
                 lambda: spqt.spqt_token_logprobs(row.view(1, 64).expand(2 ** 31, 64))):
        with pytest.raises(ValueError, match="too large"):
            call()
    assert spqt.spqt_launch_count() == before


@pytest.mark.parametrize("number", [2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 31 - 1, -2 ** 32, 2 ** 63, -2 ** 70])
def test_numbers_beyond_32_bits_are_refused(number):
    c, w = plain_cache([70], 1, 16, 6, seed=2, weight=HEAVY)
    ws = spqt.new_kv_workspace(c, 1)
    table = c.table.clone()
    before = spqt.spqt_launch_count()
    x = torch.zeros((2, 40), device="cuda")
    W = torch.zeros((256, 256), dtype=torch.float16, device="cuda")
    for call in (lambda: spqt.spqt_kv_evict(c, number, ws), lambda: spqt.spqt_kv_evict(c, 3, ws, first=number), lambda: spqt.spqt_kv_evict(c, 3, ws, recent=number),
                 lambda: spqt.spqt_token_logprobs(x, top=number), lambda: spqt.spqt_pack(W, number, 128), lambda: spqt.spqt_pack(W, 4, number),
                 lambda: spqt.new_kv_workspace(c, number), lambda: spqt.new_kv_workspace(c, 1, number)):
        with pytest.raises(ValueError):
            call()
    torch.cuda.synchronize()
    assert spqt.spqt_launch_count() == before and c.length.tolist() == [[70]] and torch.equal(c.table, table)


def test_the_status_of_what_is_no_workspace_is_refused():
    for size in (0, 4, 255):
        with pytest.raises(ValueError):
            spqt.spqt_kv_status(torch.zeros(size, dtype=torch.uint8, device="cuda"))
    with pytest.raises(TypeError):
        spqt.spqt_kv_status(torch.zeros(256, dtype=torch.uint8))
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    assert spqt.spqt_kv_status(ws) == 0
    ws.view(torch.int32)[63] = 3
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    assert spqt.spqt_kv_status(ws) == 3 and spqt.spqt_kv_status(ws, stream=s) == 3


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_read_is_the_product_in_fp32_rounded_to_fp16(fmt):
    """Every code with scales that append gives, of blocks of the smallest to the largest maxima, bit for bit."""
    top = 127.0 if fmt == "int8" else 448.0
    maxima = np.array([m * 2.0 ** e for e in range(-24, 16, 3) for m in (1.0, 1.25, 1.875, 1.9990234375)] + [2.0 ** -10, 65504.0, 0.0])
    maxima = maxima[maxima <= 65504].astype(np.float16)
    scale = (maxima.astype(np.float64) / top).astype(np.float32)
    blocks, bt, dim = len(scale), 16, 64
    codes = np.resize(np.arange(256, dtype=np.uint8), (blocks, bt, dim))
    codes[(codes & 127) == 127 if fmt == "e4m3" else codes == 128] = 0       # (not-a-number; -128, which no append writes)
    c = spqt.KVCache.new(1, 1, dim, bt, blocks, blocks, dtype=DTYPE[fmt])
    c.table.copy_(torch.arange(blocks, dtype=torch.int32).view(1, 1, -1))
    c.length.fill_(blocks * bt)
    for t in (c.k_codes, c.v_codes):
        t.view(torch.uint8).copy_(dev(codes))
    for t in (c.k_scale, c.v_scale):
        t.copy_(dev(scale))
    k, v = (torch.empty((1, blocks * bt, 1, dim), dtype=torch.float16, device="cuda") for _ in range(2))
    ws = spqt.new_kv_workspace(c, 1)
    spqt.spqt_kv_read(c, k, v, ws)
    exact = from_codes(codes, scale, fmt)
    want = exact.astype(np.float32).astype(np.float16)
    for got in (k, v):
        assert np.array_equal(got.cpu().numpy().view(np.uint16).reshape(want.shape), want.view(np.uint16))
    once = exact.astype(np.float16)
    step = np.maximum(np.abs(exact) * 2.0 ** -10, 2.0 ** -24)
    assert (np.abs(want.astype(np.float64) - once.astype(np.float64)) <= step).all()
    assert fmt == "int8" or (want != once).any()         # 7 * 2^-9 with the scale of 2^-10: 0, of which the nearest is 2^-24


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("bt", [16, 32, 64, 128])
def test_append_of_every_head_and_block_size(fmt, dim, bt):
    """Every launch shape that there is, and no other: the largest block has eight pieces a thread."""
    test_append(fmt, dim, bt, bt + 3)
