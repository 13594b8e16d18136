"""The 8-bit cache, attention over it, its eviction and log probabilities, restated in 64 bits with numpy (not collected as tests)."""
import numpy as np
import torch

from paper_2511_04477_b200 import binding

LARGEST = {"int8": 127.0, "e4m3": 448.0}
DTYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def e4m3_values():
    """The value of each of the 256 codes."""
    code = np.arange(256)
    sign, ex, man = np.where(code & 128, -1.0, 1.0), (code >> 3) & 15, code & 7
    v = np.where(ex == 0, man * 2.0 ** -9, (8 + man) * 2.0 ** (ex - 10.0))
    v = np.where((code & 127) == 127, np.nan, v)
    return sign * v


E4M3 = e4m3_values()


def to_codes(x, fmt):
    """x [blocks][tokens][dim] fp16 -> (code bytes, scale fp32): one rounding of the exact quotient, ties to even.  A quotient of 11 by
    24 bits is not nearer to a tie than 2^-40 of its size unless it is one, so that fp64 decides as the exact quotient does."""
    a = np.abs(x.astype(np.float64)).max((1, 2))
    finite = np.isfinite(x.astype(np.float64)).all((1, 2))
    scale = np.where(finite, a / LARGEST[fmt], np.nan).astype(np.float32)
    with np.errstate(invalid="ignore"):
        q = np.where(finite[:, None, None], x.astype(np.float64), 0.0) / np.where(finite & (scale > 0), scale, 1.0).astype(np.float64)[:, None, None]
    if fmt == "int8":
        return np.rint(q).astype(np.int8).view(np.uint8), scale
    m = np.abs(q)
    ex = np.maximum(np.frexp(m)[1] - 1, -6)
    v = np.minimum(np.rint(np.ldexp(m, 3 - ex)) * np.ldexp(1.0, ex - 3), 448.0)
    order = np.argsort(E4M3[:127], kind="stable")
    code = order[np.searchsorted(E4M3[:127][order], v)]
    assert np.array_equal(E4M3[code], v)
    return (code | np.where(np.signbit(q), 128, 0)).astype(np.uint8), scale


def from_codes(code, scale, fmt):
    v = code.view(np.int8).astype(np.float64) if fmt == "int8" else E4M3[code]
    return v * scale.astype(np.float64)[:, None, None]


class Streams:
    """What a cache holds, stream by stream, beside a KVCache with the same contents: the unused parts of its buffers are filled with
    what must not matter (not-a-number, infinities, blocks outside the pool)."""

    def __init__(self, lengths, kv_heads, dim, bt, fmt, seed, width=None, weight=True, amplitude=1.0):
        """lengths: of each sequence, or of each stream ([batch][kv_heads])"""
        rng = np.random.Generator(np.random.PCG64(seed))
        n = np.array(lengths, dtype=np.int64)
        self.n = np.broadcast_to(n[:, None], (len(n), kv_heads)).copy() if n.ndim == 1 else n
        self.B, self.H, self.D, self.bt, self.fmt = self.n.shape[0], kv_heads, dim, bt, fmt
        need = -(-self.n // bt)
        self.W = int(width if width is not None else max(1, need.max() + 1))
        self.blocks = int(need.sum()) + 3
        ids = rng.permutation(self.blocks)
        codes = rng.integers(0, 256, (2, self.blocks, bt, dim)).astype(np.uint8)
        if fmt == "e4m3":
            codes[(codes & 127) == 127] = 1
        scale = np.full((2, self.blocks), np.nan, dtype=np.float32)
        tail = np.full((2, self.B, self.H, bt, dim), np.nan, dtype=np.float16)
        tail[:, :, :, ::2] = np.inf
        self.table = np.full((self.B, self.H, self.W), -7, dtype=np.int32)
        self.weight = rng.exponential(size=(self.blocks, bt)).astype(np.float32)
        self.kv = {}
        at = 0
        for b in range(self.B):
            for h in range(self.H):
                n, full = int(self.n[b, h]), int(self.n[b, h]) // bt
                self.table[b, h, :need[b, h]] = ids[at:at + need[b, h]]
                at += int(need[b, h])
                x = (amplitude * rng.standard_normal((2, n, dim))).astype(np.float16)
                rows = []
                for k in range(2):
                    own = self.table[b, h, :full]
                    c, s = to_codes(x[k, :full * bt].reshape(full, bt, dim), fmt) if full else (np.zeros((0, bt, dim), np.uint8), np.zeros(0, np.float32))
                    codes[k, own], scale[k, own] = c, s
                    tail[k, b, h, :n - full * bt] = x[k, full * bt:]
                    rows.append(np.concatenate([from_codes(c, s, fmt).reshape(-1, dim), x[k, full * bt:].astype(np.float64)]))
                self.kv[b, h] = rows
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.cache = binding.KVCache(dev(codes[0]).view(DTYPE[fmt]), dev(codes[1]).view(DTYPE[fmt]), dev(scale[0]), dev(scale[1]), dev(tail[0]), dev(tail[1]),
                                     dev(self.table), dev(self.n.astype(np.int32)), dev(self.weight) if weight else None)

    def queries(self, q_heads, queries, seed, amplitude=1.0):
        rng = np.random.Generator(np.random.PCG64(seed))
        return (amplitude * rng.standard_normal((self.B, queries, q_heads, self.D))).astype(np.float16)

    def attention(self, q, scale=None):
        """(out, its tolerance, weight received, its tolerance), in fp64.

        Tolerances.  A score is a sum of D exact products in fp32, in D/16 steps of a matrix instruction that cut below 2^-24 of the
        largest term, and two more roundings: off by less than e = (D/16 + 4) * 2^-23 * scale * sum|q||k|.  A probability is then off
        by a factor within 2e (its own and the sum's), its exponential, product and sums by 2^-19 at most (hundreds of additions
        of positive terms in fp32 a lane, of which the errors of the tests' sizes stay below 2^-20; 2^-22 for the two halves that it
        enters as).  The result is rounded to fp16 once, half a step: 2^-11 of it, or 2^-25 below the normal numbers."""
        B, Q, HQ, D = q.shape
        G = HQ // self.H
        scale = D ** -0.5 if scale is None else scale
        out, tol = np.zeros(q.shape), np.zeros(q.shape)
        got, got_tol = np.zeros(self.weight.shape), np.zeros(self.weight.shape)
        for (b, h), (K, V) in self.kv.items():
            n = K.shape[0]
            for i in range(Q):
                seen = n - Q + 1 + i
                if seen <= 0:
                    continue
                x = q[b, i, h * G:(h + 1) * G].astype(np.float64)
                s = x @ K[:seen].T * scale
                e = (D / 16 + 4) * 2.0 ** -23 * abs(scale) * (np.abs(x) @ np.abs(K[:seen]).T).max(1, keepdims=True)
                p = np.exp(s - s.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                o = p @ V[:seen]
                out[b, i, h * G:(h + 1) * G] = o
                tol[b, i, h * G:(h + 1) * G] = 2.0 ** -11 * np.abs(o) + 2.0 ** -25 + (2 * e + 2.0 ** -19) * (p @ np.abs(V[:seen]))
                t = np.arange(seen)
                block, row = self.table[b, h, t // self.bt], t % self.bt
                got[block, row] += p.sum(0)
                got_tol[block, row] += ((2 * e + 2.0 ** -19) * p).sum(0)
        return out, tol, got, got_tol + 2.0 ** -23 * (np.abs(self.weight) + got)

    def workspace(self, q_heads, queries=1):
        return binding.new_kv_workspace(self.cache, q_heads, queries)


def check(got, want, tol, what=""):
    got = got.detach().cpu().numpy().astype(np.float64) if isinstance(got, torch.Tensor) else got
    err = np.abs(got - want)
    bad = ~(err <= tol)
    assert not bad.any(), "%s: %d of %d out of tolerance, worst %.3g (tolerance %.3g)" % (what, bad.sum(), bad.size, err[bad].max(), tol[bad][err[bad].argmax()])
