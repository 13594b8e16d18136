"""Host-side checks of the calls over the 8-bit cache and over logits that need no GPU: sizes, and refusals before anything is launched."""
import ctypes

import pytest

from paper_2511_04477_b200 import binding, build


@pytest.fixture(scope="module")
def L():
    build.build()
    return binding.lib()


@pytest.fixture(scope="module")
def a16():
    buf = ctypes.create_string_buffer(4096)
    yield (ctypes.addressof(buf) + 15) // 16 * 16        # a fake device address; never dereferenced


def desc(a16, **kw):
    d = binding.KVCacheDesc(2, 4, 128, 32, 0, 100, 10, *[a16] * 9)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def size(L, d, q_heads=8, queries=1):
    out = ctypes.c_size_t(0)
    rc = L.spqt_kv_workspace(ctypes.byref(d), q_heads, queries, ctypes.byref(out))
    return rc, out.value


BAD = [(dict(batch=0), 1), (dict(kv_heads=-1), 1), (dict(blocks=0), 1), (dict(table_width=0), 1), (dict(k_codes=None), 1), (dict(v_scale=None), 1),
       (dict(length=None), 1), (dict(head_dim=80), 2), (dict(head_dim=0), 2), (dict(block_tokens=8), 2), (dict(block_tokens=48), 2), (dict(format=2), 2),
       (dict(table_width=16385), 2), (dict(batch=4097), 2), (dict(batch=2 ** 31 - 1, kv_heads=2 ** 31 - 1), 2)]


@pytest.mark.parametrize("kw,status", BAD)
def test_caches_that_are_refused(L, a16, kw, status):
    d = desc(a16, **kw)
    r = ctypes.byref(d)
    before = binding.spqt_launch_count()
    assert size(L, d)[0] == status
    assert L.spqt_kv_append(r, a16, a16, 1, 0, 0, None, None, a16, 1 << 20, None) == status
    assert L.spqt_kv_read(r, None, a16, a16, 1, 0, 0, 0, a16, 1 << 20, None) == status
    assert L.spqt_kv_attention(r, a16, 0, 0, 8, 1, 1.0, 0, a16, 0, 0, a16, 1 << 30, None) == status
    assert L.spqt_kv_evict(r, 1, 0, 0, None, None, a16, 1 << 20, None) == status
    assert binding.spqt_launch_count() == before


@pytest.mark.parametrize("name", ["k_codes", "v_codes", "k_tail", "v_tail", "weight", "k_scale", "v_scale", "table", "length"])
def test_addresses_that_are_refused(L, a16, name):
    wide = name in ("k_codes", "v_codes", "k_tail", "v_tail", "weight")
    d = desc(a16, **{name: a16 + (8 if wide else 2)})
    assert size(L, d)[0] == 3
    assert L.spqt_kv_evict(ctypes.byref(d), 1, 0, 0, None, None, a16, 1 << 20, None) == 3


def test_arguments_that_are_refused(L, a16):
    d = desc(a16)
    r = ctypes.byref(d)
    n = binding.spqt_launch_count()
    rc, ws = size(L, d)
    assert rc == 0 and 0 < ws < 64 << 20
    assert size(L, d, 8, 16)[0] == 0 and size(L, d, 8, 16)[1] >= size(L, d, 8, 3)[1] >= ws
    assert size(L, d, 0)[0] == 1 and size(L, d, 8, 0)[0] == 1
    assert size(L, d, 6)[0] == 2 and size(L, d, 4 * 65)[0] == 2 and size(L, d, 8, 17)[0] == 2
    assert L.spqt_kv_workspace(r, 8, 1, None) == 1 and L.spqt_kv_workspace(None, 8, 1, ctypes.byref(ctypes.c_size_t())) == 1
    # more tiles than 31 bits count
    assert size(L, desc(a16, batch=1024, kv_heads=16, table_width=16384, block_tokens=128, weight=None), 16)[0] in (0, 2)
    assert size(L, desc(a16, batch=4096, kv_heads=4, table_width=16384, block_tokens=128), 4)[0] == 0
    assert size(L, desc(a16, batch=4096, kv_heads=4), 4 * 32)[0] == 2      # streams times row groups
    # append
    ap = lambda **k: L.spqt_kv_append(r, k.get("k", a16), k.get("v", a16), k.get("tokens", 3), k.get("bs", 512 * 3), k.get("ts", 512), k.get("counts"), k.get("out"),
                                      k.get("ws", a16), k.get("bytes", 4096), None)
    assert ap(k=None) == 1 and ap(v=None) == 1 and ap(tokens=0) == 1 and ap(tokens=-1) == 1 and ap(bs=-8) == 1 and ap(ts=-8) == 1
    assert ap(k=a16 + 8) == 3 and ap(ts=516) == 3 and ap(bs=4) == 3 and ap(counts=a16 + 2) == 3 and ap(out=a16 + 1) == 3 and ap(ws=a16 + 8) == 3
    assert ap(ws=None) == 1 and ap(bytes=256) == 4 and ap(tokens=2 ** 31 - 1) == 2
    # read
    rd = lambda **k: L.spqt_kv_read(r, k.get("length"), k.get("k", a16), k.get("v", a16), k.get("tokens", 3), k.get("bs", 0), k.get("ts", 512), k.get("hs", 128),
                                    k.get("ws", a16), k.get("bytes", 4096), None)
    assert rd(k=None) == 1 and rd(tokens=0) == 1 and rd(hs=-8) == 1 and rd(hs=4) == 3 and rd(v=a16 + 2) == 3 and rd(length=a16 + 2) == 3
    assert rd(ws=None) == 1 and rd(bytes=255) == 4
    # attention
    at = lambda **k: L.spqt_kv_attention(r, k.get("q", a16), k.get("qb", 0), k.get("qt", 0), k.get("heads", 8), k.get("queries", 1), 1.0, k.get("acc", 0), k.get("out", a16),
                                         0, k.get("ot", 0), k.get("ws", a16), k.get("bytes", ws), None)
    assert at(q=None) == 1 and at(out=None) == 1 and at(qb=-8) == 1 and at(heads=7) == 2 and at(queries=17) == 2 and at(queries=0) == 1
    assert at(q=a16 + 8) == 3 and at(qt=4) == 3 and at(ot=12) == 3 and at(ws=a16 + 4) == 3 and at(ws=None) == 1 and at(bytes=ws - 1, acc=1) == 4 and at(bytes=1024) == 4
    none = desc(a16, weight=None)
    assert L.spqt_kv_attention(ctypes.byref(none), a16, 0, 0, 8, 1, 1.0, 1, a16, 0, 0, a16, 1 << 30, None) == 1
    assert size(L, none)[1] < ws
    # evict
    ev = lambda keep, first=0, recent=0, c=r, ws=a16, bytes=256, t=None: L.spqt_kv_evict(c, keep, first, recent, t, None, ws, bytes, None)
    assert ev(-1) == 1 and ev(3, 2, 2) == 1 and ev(3, -1) == 1 and ev(3, 0, -1) == 1 and ev(2, 2 ** 31 - 1, 2 ** 31 - 1) == 1
    assert ev(3, c=ctypes.byref(none)) == 1 and ev(3, ws=None) == 1 and ev(3, bytes=255) == 4 and ev(3, t=a16 + 2) == 3
    assert L.spqt_kv_status(None, ctypes.byref(ctypes.c_int()), None) == 1 and L.spqt_kv_status(a16, None, None) == 1
    assert binding.spqt_launch_count() == n


def test_logprobs_arguments_that_are_refused(L, a16):
    n = binding.spqt_launch_count()

    def lp(**k):
        g = lambda name, default: k.get(name, default)
        return L.spqt_token_logprobs(g("x", a16), g("dtype", 0), g("rows", 2), g("vocab", 100), g("stride", 100), g("tokens", a16), g("top", 3), g("logprob", a16),
                                     g("entropy", a16), g("best", a16), g("index", a16), None)
    assert lp(x=None) == 1 and lp(rows=-1) == 1 and lp(vocab=0) == 1 and lp(stride=99) == 1 and lp(top=-1) == 1 and lp(top=101) == 1
    assert lp(tokens=None) == 1 and lp(logprob=None) == 1 and lp(best=None) == 1 and lp(index=None) == 1
    assert lp(dtype=3) == 2 and lp(top=33) == 2 and lp(vocab=(1 << 20) + 1, stride=1 << 21) == 2
    assert lp(x=a16 + 1) == 3 and lp(x=a16 + 2, dtype=2) == 3 and lp(entropy=a16 + 2) == 3 and lp(index=a16 + 2) == 3
    assert lp(rows=0) == 0
    assert binding.spqt_launch_count() == n


def test_rows_to_write_that_lie_on_one_another_are_refused(L, a16):
    """Refused before a launch (which has no GPU here: a call that is not refused reports SPQT_ERR_CUDA, 5, at most)."""
    d = desc(a16)                                        # 2 sequences, 4 kv heads of 128
    ws, n = size(L, d, 8, 16)[1], binding.spqt_launch_count()

    def read(bs, ts, hs, tokens=3, k=a16, v=a16 + (1 << 20)):
        return L.spqt_kv_read(ctypes.byref(d), None, k, v, tokens, bs, ts, hs, a16, 4096, None)

    def attend(bs, ts, queries=5):
        return L.spqt_kv_attention(ctypes.byref(d), a16, 0, 0, 8, queries, 1.0, 0, a16 + (1 << 20), bs, ts, a16, ws, None)
    far = 2 ** 62
    for bad in ((0, 512, 128), (1536, 0, 128), (1536, 512, 0), (1536, 512, 120), (1536, 504, 128), (1528, 512, 128), (512, 512, 128), (128, 512, 128), (512, 1024, 1024),
                (far, 512, 64)):
        assert read(*bad) == 1, bad
    assert read(1536, 512, 128, k=a16, v=a16) == 1 and read(1536, 512, 128, v=a16 + 240) == 1 and read(1536, 512, 128, k=a16 + 240, v=a16) == 1
    assert read(1024, 0, 128, tokens=2) == 1
    for bad in ((0, 1024), (5120 - 8, 1024), (1024, 1024), (1016, 8192), (8192, 1016), (8192, 0)):
        assert attend(*bad) == 1, bad
    assert attend(1016, 0, queries=1) == 1
    assert binding.spqt_launch_count() == n
    one = desc(a16, batch=1, kv_heads=1)
    if binding.torch.cuda.is_available():
        return                                           # (the addresses are not real: the calls that are taken stay off the GPU)
    for good in ((1536, 512, 128), (4096, 1024, 256), (512, 1024, 128), (1536, 128, 384), (128, 1024, 256), (far, 512, 128)):
        assert read(*good) == 5, good
    assert read(1536, 512, 128, v=a16 + 256) == 5 and read(512, 0, 128, tokens=1) == 5
    assert L.spqt_kv_read(ctypes.byref(one), None, a16, a16 + 4096, 1, 0, 0, 0, a16, 4096, None) == 5
    for good in ((5120, 1024), (1024, 2048), (far, 1024)):
        assert attend(*good) == 5, good
    assert attend(1024, 0, queries=1) == 5


def test_the_joint_limit_of_streams_and_rows(L, a16):
    """batch * kv_heads * ceil(rows / 16) <= 16384 and nothing else refuses a cache within the single limits."""
    for batch, kv_heads, group, queries in ((4096, 4, 1, 16), (4096, 4, 16, 1), (4096, 4, 1, 1), (8192, 1, 2, 16), (8191, 1, 32, 1), (256, 1, 64, 16), (255, 1, 64, 16),
                                            (1, 16, 64, 16), (4096, 2, 3, 10), (1, 256, 64, 16)):
        assert size(L, desc(a16, batch=batch, kv_heads=kv_heads), kv_heads * group, queries)[0] == 0
    for batch, kv_heads, group, queries in ((4096, 4, 17, 1), (4096, 4, 2, 9), (8193, 1, 2, 16), (257, 1, 64, 16), (8192, 1, 4, 16), (4096, 2, 3, 16)):
        d = desc(a16, batch=batch, kv_heads=kv_heads)
        assert size(L, d, kv_heads * group, queries)[0] == 2
        assert L.spqt_kv_attention(ctypes.byref(d), a16, 0, 0, kv_heads * group, queries, 1.0, 0, a16, 0, 0, a16, 1 << 40, None) == 2
    # the largest cache there is: its tiles and scores are counted in 64 bits
    largest = desc(a16, batch=1, kv_heads=16384, table_width=16384, block_tokens=128, head_dim=256, blocks=2 ** 31 - 1)
    rc, n = size(L, largest, 16384 * 16)
    tiles = 16384 * (16384 * 128 // 32 + 8 + 16)
    assert rc == 0 and n > tiles * (16 + 32 * 16 * 4)
    assert size(L, desc(a16, batch=1024, kv_heads=16, table_width=16384, block_tokens=128, weight=None), 16)[0] == 0
