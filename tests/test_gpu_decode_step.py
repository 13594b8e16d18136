"""The calls of a decode step one after the other, as a serving loop makes them: linear, append, attention with accumulated weights,
eviction, linear, head, log probabilities; in a stream and in a replayed graph, against the same steps in 64 bits."""
import pathlib
import subprocess
import sys

import numpy as np
import pytest
import torch

import oracle
from kv_util import to_codes
from paper_2511_04477_b200 import binding as spqt
from paper_2511_04477_b200 import inputs

pytestmark = pytest.mark.gpu

HQ, HK, D, BT, HIDDEN, VOCAB = 8, 2, 64, 16, 512, 1024


class Model:
    def __init__(self):
        self.Wqkv = inputs.weights((HQ + 2 * HK) * D, HIDDEN, seed=1)
        self.Whead = inputs.weights(VOCAB, HQ * D, seed=2)
        dev = lambda W: torch.from_numpy(W).cuda()
        self.qkv, self.head = spqt.spqt_pack(dev(self.Wqkv), 4, 64), spqt.spqt_pack(dev(self.Whead), 4, 64)
        width, blocks = 12, 2 * 12
        self.cache = spqt.KVCache.new(1, HK, D, BT, blocks, width, weight=True)
        self.cache.table.copy_(torch.from_numpy(np.random.Generator(np.random.PCG64(3)).permutation(blocks).astype(np.int32).reshape(1, HK, width)).cuda())
        self.ws = [spqt.new_workspace(p.m, p.n, 4, 64) for p in (self.qkv, self.head)]
        self.kws = spqt.new_kv_workspace(self.cache, HQ)
        self.x = torch.empty(HIDDEN, dtype=torch.float16, device="cuda")
        self.y = torch.empty((HQ + 2 * HK) * D, dtype=torch.float16, device="cuda")
        self.att = torch.empty((1, 1, HQ, D), dtype=torch.float16, device="cuda")
        self.logits = torch.empty((1, VOCAB), dtype=torch.float16, device="cuda")
        self.token = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(self, evict):
        rows = self.y.view(1, 1, -1, D)
        spqt.spqt_dense_gemv(self.qkv, self.x, self.ws[0], self.y)
        spqt.spqt_kv_append(self.cache, rows[:, :, HQ:HQ + HK], rows[:, :, HQ + HK:], self.kws)
        spqt.spqt_kv_attention(self.cache, rows[:, :, :HQ], self.kws, accumulate=True, out=self.att)
        if evict:
            spqt.spqt_kv_evict(self.cache, 4, self.kws, first=1, recent=1)
        spqt.spqt_dense_gemv(self.head, self.att.view(-1), self.ws[1], self.logits.view(-1))
        return spqt.spqt_token_logprobs(self.logits, self.token, top=5)


def test_a_run_of_decode_steps_against_64_bits_and_in_graphs():
    tokens = 130
    xs = [inputs.activations(HIDDEN, seed=100 + t) for t in range(tokens)]
    results = []
    for graphs in (False, True):
        m = Model()
        if graphs:
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                m.x.copy_(torch.from_numpy(xs[0]))
                m.step(False), m.step(True)
                m.cache.length.zero_()
            s.synchronize()
            played = []
            for evict in (False, True):
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=s):
                    out = m.step(evict)
                played.append((g, out))
        got = []
        for t in range(tokens):
            evict = t % BT == BT - 1
            m.x.copy_(torch.from_numpy(xs[t]))
            torch.cuda.synchronize()
            if graphs:
                played[evict][0].replay()
                out = played[evict][1]
            else:
                out = m.step(evict)
            torch.cuda.synchronize()
            got.append([m.y.cpu().numpy(), m.att.cpu().numpy(), m.logits.cpu().numpy()] + [v.cpu().numpy() for v in out] +
                       [m.cache.table.cpu().numpy(), m.cache.length.cpu().numpy(), m.cache.weight.cpu().numpy()])
        assert spqt.spqt_kv_status(m.kws) == 0
        results.append(got)
    for a, b in zip(*results):                       # a replayed graph gives the bits of the calls
        for u, v in zip(a[:-3], b[:-3]):
            assert np.array_equal(u, v)
        assert np.array_equal(a[-2], b[-2])

    # the same steps in 64 bits, from the projections that the linear gave (its own tests hold it to the oracle)
    held = {h: [[], [], []] for h in range(HK)}        # keys, values, weight of the tokens that are there
    for t, (y, att, logits, logprob, entropy, top, index, table, length, weight) in enumerate(results[0]):
        rows = y.reshape(-1, D)
        for h in range(HK):
            k, v, w = held[h]
            k.append(rows[HQ + h]), v.append(rows[HQ + HK + h]), w.append(0.0)
            if len(k) % BT == 0:                       # a block is full: rounded once
                for rows_of in (k, v):
                    code, scale = to_codes(np.array(rows_of[-BT:])[None], "int8")
                    rows_of[-BT:] = list(code.view(np.int8)[0].astype(np.float64) * np.float64(scale[0]))
            K, V = np.array(k, dtype=np.float64), np.array(v, dtype=np.float64)
            G = HQ // HK
            q = rows[h * G:(h + 1) * G].astype(np.float64)
            s = q @ K.T * D ** -0.5
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            e = (D / 16 + 4) * 2.0 ** -23 * D ** -0.5 * (np.abs(q) @ np.abs(K).T).max()
            want = p @ V
            tol = 2.0 ** -11 * np.abs(want) + 2.0 ** -25 + (2 * e + 2.0 ** -19) * (p @ np.abs(V))
            assert (np.abs(att[0, 0, h * G:(h + 1) * G] - want) <= tol).all(), t
            for i, dp in enumerate(p.sum(0)):
                w[i] += dp
            if t % BT == BT - 1 and len(k) // BT > 4:
                n = len(k) // BT
                score = [np.float32(sum(w[j * BT:(j + 1) * BT])) for j in range(n)]
                inner = sorted(range(1, n - 1), key=lambda j: (-score[j], j))
                stay = sorted([0, n - 1] + inner[:2])
                # (a choice between sums that the accumulated rounding could exchange would prove nothing)
                assert score[inner[1]] - score[inner[2]] > 1e-4 * score[inner[1]] if len(inner) > 2 else True
                held[h] = [[r for j in stay for r in rows_of[j * BT:(j + 1) * BT]] for rows_of in (k, v, w)]
            assert length[0, h] == len(held[h][0])
        x = logits.astype(np.float64)[0]
        lse = np.log(np.exp(x - x.max()).sum()) + x.max()
        assert abs(logprob[0] - (x[0] - lse)) <= 2.0 ** -15 + 2.0 ** -22 * abs(x[0] - lse)
        assert index[0].tolist() == sorted(range(VOCAB), key=lambda i: (-x[i], i))[:5]
    assert max(len(held[h][0]) for h in held) <= 4 * BT + BT


def test_the_decode_workload_runs():
    from paper_2511_04477_b200 import sweep
    r = sweep.run_decode(layers=1, context=512, keep=128, tokens=32)
    assert r["device_status"] == 0 and r["length"] == 128 and r["tokens"] == 32 and r["ms_per_token"] > 0
    assert np.isfinite(r["logprob"]) and 0 <= r["entropy"] <= np.log(sweep.DECODE_VOCAB) and len(set(r["top_index"])) == 5


FIRST_CALLS_IN_A_GRAPH = """
import torch
from paper_2511_04477_b200 import binding as spqt
torch.manual_seed(0)
def caches():
    torch.manual_seed(1)
    c = spqt.KVCache.new(2, 2, 128, 16, 64, width, weight=True)
    c.table.copy_(torch.arange(4 * 16, dtype=torch.int32, device="cuda").view(2, 2, 16).repeat(1, 1, width // 16))
    for x in (c.k_codes, c.v_codes, c.weight, c.k_tail, c.v_tail):
        x.zero_()
    return c
def step(c, ws, out):
    spqt.spqt_kv_append(c, *kv, ws)
    spqt.spqt_kv_attention(c, q, ws, accumulate=True, out=out)
    spqt.spqt_kv_evict(c, 1, ws)
    return spqt.spqt_token_logprobs(logits, token, top=3)
kv = [torch.randn(2, 40, 2, 128, device="cuda").half() for _ in range(2)]
q = torch.randn(2, 1, 8, 128, device="cuda").half()
logits, token = torch.randn(2, 500, device="cuda").half(), torch.tensor([3, 7], dtype=torch.int32, device="cuda")
for width in (16, 2048):
    runs = []
    for graph in (True, False):
        c = caches()
        ws = spqt.new_kv_workspace(c, 8)
        out = torch.zeros(2, 1, 8, 128, dtype=torch.float16, device="cuda")
        torch.cuda.synchronize()
        if graph:
            s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                scores = step(c, ws, out)
            g.replay()
        else:
            scores = step(c, ws, out)
        torch.cuda.synchronize()
        assert spqt.spqt_kv_status(ws) == 0 and c.length.tolist() == [[24, 24], [24, 24]]
        runs.append([out, c.table, c.weight, c.k_codes, c.v_tail[:, :, :8]] + [x for x in scores if x is not None])
    assert all(torch.equal(x, y) for x, y in zip(*runs)), width
print("same")
"""


def test_the_first_calls_of_a_process_can_be_captured():
    """What a kernel is prepared with on its first launch can be done while a graph is recorded."""
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS_IN_A_GRAPH], capture_output=True, text=True, timeout=300,
                       cwd=pathlib.Path(__file__).resolve().parents[1])
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stdout + r.stderr


def test_the_decode_workload_counts_its_launches():
    """What it says of launches is what one layer's calls launch: four linears, append, attention (weights added in the same
    kernel here), the eviction with every block's last token; the head and the log probabilities once."""
    from paper_2511_04477_b200 import sweep
    layers, block = 1, 32
    r = sweep.run_decode(layers=layers, context=512, keep=128, tokens=block, block=block)
    c = spqt.KVCache.new(1, sweep.DECODE_HEADS["kv_heads"], sweep.DECODE_HEADS["head_dim"], block, 8 * 18, 512 // block + 2, weight=True)
    ws = spqt.new_kv_workspace(c, sweep.DECODE_HEADS["q_heads"])
    q = torch.zeros((1, 1, sweep.DECODE_HEADS["q_heads"], sweep.DECODE_HEADS["head_dim"]), dtype=torch.float16, device="cuda")
    k = q[:, :, :sweep.DECODE_HEADS["kv_heads"]]
    c.table.copy_(torch.arange(8 * 18, dtype=torch.int32).view(1, 8, 18))
    counts = []
    for call in (lambda: spqt.spqt_kv_append(c, k, k, ws), lambda: spqt.spqt_kv_attention(c, q, ws, accumulate=True), lambda: spqt.spqt_kv_evict(c, 4, ws)):
        before = spqt.spqt_launch_count()
        call()
        counts.append(spqt.spqt_launch_count() - before)
    torch.cuda.synchronize()
    assert abs(r["launches_per_token"] - (layers * (4 + counts[0] + counts[1] + counts[2] / block) + 2)) < 1e-9
