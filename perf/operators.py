"""What stands between and behind the linears of a decode step, as cases that can be timed.

A case is a dict of plain values; ``op`` says which calls a pass makes:

  append     new keys and values into the 8-bit cache, and the cache read back as fp16   spqt_kv_append, spqt_kv_read
  attention  the step's queries over the cache; ``accumulate``: the attention weights    spqt_kv_attention
             are added up per token as well
  evict      all but the blocks with the largest accumulated weight leave the cache      spqt_kv_evict
  logprobs   log probabilities of the chosen tokens, entropy, top alternatives           spqt_token_logprobs

The cache: every (sequence, kv head) owns blocks of ``block`` tokens in a pool, named by its row of ``table``.  A block that is
full is held as 8-bit codes (int8, or e4m3 where ``fmt`` says so) times one fp32 scale; the tokens of the block that is not full
yet are held as fp16 in ``tail``.  ``length`` counts the tokens of a (sequence, kv head).  ``weight`` has an fp32 value for
each token of each block.

Where ``own`` is false a pass consists of elementary torch operations on the same buffers.
"""
import math
import random

import torch

own = False

LARGEST = {"int8": 127.0, "e4m3": 448.0}
HELD = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
LOGITS = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    kv = {"q_heads": 32, "kv_heads": 8, "dim": 128, "block": 32, "fmt": "int8"}   # a Llama-3-8B-shaped layer
    return [
        # a decode step's keys and values for eight short sequences: latency and launches count
        {"name": "append_decode_b8", "op": "append", "batch": 8, "new": 1, "tokens": 300, "ragged": True, **kv},
        # prompts of several lengths in one padded batch, into an empty cache
        {"name": "append_prompts_b4", "op": "append", "batch": 4, "new": 4099, "tokens": 0, "ragged": True, **kv},
        # the first tokens of an answer to a short question: the smallest call
        {"name": "attend_b1_45", "op": "attention", "batch": 1, "queries": 1, "tokens": 45, "ragged": False, "accumulate": False, **kv},
        # the ordinary decode step of one sequence
        {"name": "attend_b1_4001", "op": "attention", "batch": 1, "queries": 1, "tokens": 4001, "ragged": False, "accumulate": False, **kv},
        # a layer without shared heads (Llama-2-13B-shaped), four sequences, e4m3 codes, larger blocks
        {"name": "attend_mha40_b4", "op": "attention", "batch": 4, "queries": 1, "tokens": 2047, "ragged": True, "accumulate": False,
         "q_heads": 40, "kv_heads": 40, "dim": 128, "block": 64, "fmt": "e4m3"},
        # serving with a bounded cache: eight sequences of a Llama-2-70B-shaped layer, weights accumulated for the eviction
        {"name": "attend_70b_b8_weights", "op": "attention", "batch": 8, "queries": 1, "tokens": 16000, "ragged": True, "accumulate": True,
         "q_heads": 64, "kv_heads": 8, "dim": 128, "block": 32, "fmt": "int8"},
        # five speculative tokens at once, small blocks, each query seeing the tokens up to its own
        {"name": "attend_spec5_b2", "op": "attention", "batch": 2, "queries": 5, "tokens": 8191, "ragged": True, "accumulate": True,
         "q_heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "fmt": "int8"},
        # one long document: the work of a single sequence has to be spread over the device
        {"name": "attend_b1_131072", "op": "attention", "batch": 1, "queries": 1, "tokens": 131072, "ragged": False, "accumulate": False,
         "q_heads": 32, "kv_heads": 8, "dim": 128, "block": 128, "fmt": "int8"},
        # the bounded cache of one sequence, as often as it is full
        {"name": "evict_b1_4100", "op": "evict", "batch": 1, "tokens": 4100, "ragged": False, "keep": 96, "first": 1, "recent": 16, **kv},
        # sixteen long contexts cut to a quarter at once
        {"name": "evict_b16_32768", "op": "evict", "batch": 16, "tokens": 32768, "ragged": True, "keep": 256, "first": 1, "recent": 32, **kv},
        # the sampled tokens of a small decode batch over a large vocabulary
        {"name": "logprobs_8x128256", "op": "logprobs", "rows": 8, "vocab": 128256, "top": 5, "dtype": "fp16"},
        # scoring a prompt: every position's own token and its likeliest alternatives
        {"name": "logprobs_2048x32000", "op": "logprobs", "rows": 2048, "vocab": 32000, "top": 20, "dtype": "fp16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("append", "attention", "attention", "attention", "evict", "logprobs", "logprobs"))
    if op == "logprobs":
        vocab = _log(rng, 500, 160000)
        dtype = rng.choice(("fp16", "fp16", "bf16", "fp32"))
        rows = _log(rng, 1, max(1, min(4096, 65536000 // vocab // (2 if dtype == "fp32" else 1))))
        return {"op": op, "rows": rows, "vocab": vocab, "top": rng.choice((0, 1, 5, 8, 20, 32)), "dtype": dtype}
    dim, block = rng.choice((64, 96, 128, 128, 128, 256)), rng.choice((16, 32, 32, 64, 128))
    kv_heads, shared = rng.choice((1, 2, 4, 8, 8, 12, 40)), rng.choice((1, 2, 3, 4, 4, 7, 8, 16))
    c = {"op": op, "batch": _log(rng, 1, 32), "q_heads": kv_heads * shared, "kv_heads": kv_heads, "dim": dim, "block": block,
         "fmt": rng.choice(("int8", "int8", "e4m3")), "ragged": rng.random() < 0.7}
    streams = c["batch"] * kv_heads
    if op == "append":
        prompt = rng.random() < 0.6
        most = max(2, 16000000 // (streams * dim))
        c["new"] = _log(rng, 2, min(8192, most)) if prompt else 1
        c["tokens"] = rng.choice((0, block * _log(rng, 1, 64))) if prompt else _log(rng, 1, 600)
        c["tokens"] = min(c["tokens"], max(0, most - c["new"]) // block * block if prompt else most)
        return c
    c["tokens"] = _log(rng, 1, max(2, min(131072, (130000000 if op == "attention" else 400000000) // (streams * dim))))
    if op == "attention":
        c["queries"] = rng.choice((1, 1, 1, 2, 4, 8)) if shared * 8 <= 64 else 1
        c["accumulate"] = rng.random() < 0.4
        return c
    closed = max(1, c["tokens"] // block)
    c["keep"] = max(2, int(closed * rng.uniform(0.1, 0.9)))
    c["first"] = rng.choice((0, 1, 1, 2)) if c["keep"] > 8 else 0
    c["recent"] = int(rng.uniform(0, 0.5) * (c["keep"] - c["first"]))
    return c


def _counts(case, most, salt):
    """Tokens of each sequence: the first has the most, the others any part of it."""
    r = random.Random(1000 * case["batch"] + most + salt)
    return [most if b == 0 or not case["ragged"] else int(round(most * r.uniform(0.05, 1.0))) for b in range(case["batch"])]


def _lengths(case):
    most = case["tokens"]
    n = _counts(case, most, 1)
    if case["op"] == "append" and case["new"] > 1:   # prompts and their continuations begin with a block
        n = [t // case["block"] * case["block"] for t in n]
    return n


# ---------------------------------------------------------------- inputs


def _quantized(x, fmt):
    """Codes (as values) and the scale of each block; x: [..., tokens, dim] in 64 bits.  The scale is held in 32 bits."""
    scale = (x.abs().amax((-2, -1)) / LARGEST[fmt]).float()
    q = x / torch.where(scale > 0, scale, 1.0).double()[..., None, None]
    if fmt == "int8":
        return q.round(), scale
    step = torch.ldexp(torch.ones_like(q), (torch.frexp(q.abs())[1] - 1).clamp(min=-6) - 3)
    return (q / step).round() * step, scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    state = {"op": case["op"], "case": dict(case)}
    if case["op"] == "logprobs":
        rows, vocab = case["rows"], case["vocab"]
        x = torch.empty((rows, vocab), device="cuda", dtype=LOGITS[case["dtype"]])
        for r in range(0, rows, 256):   # a bulk and a few likely tokens
            z = randn(min(256, rows - r), vocab)
            x[r:r + 256] = 2.0 * z + 1.5 * (z - 2.0).clamp(min=0.0).square()
        state.update(logits=x, tokens=torch.multinomial(torch.softmax(x[:, :min(vocab, 30000)].float(), 1), 1, generator=g)[:, 0].int())
        return state

    B, H, D, bt, fmt = case["batch"], case["kv_heads"], case["dim"], case["block"], case["fmt"]
    new = _counts(case, case["new"], 2) if case["op"] == "append" else [0] * B
    lengths = _lengths(case)
    width = (max(n + t for n, t in zip(new, lengths)) + bt - 1) // bt + 2
    blocks = B * H * width
    channel = torch.exp(0.4 * randn(D))   # keys have a few large channels
    k, v = (torch.empty((blocks, bt, D), dtype=HELD[fmt], device="cuda") for _ in range(2))
    k_scale, v_scale = (torch.empty(blocks, device="cuda") for _ in range(2))
    if case["op"] == "evict":             # (an eviction moves no codes: nothing reads them)
        k_scale.fill_(1.0), v_scale.fill_(1.0)
    else:
        part = max(1, 8000000 // (bt * D))
        for i in range(0, blocks, part):
            n = min(part, blocks - i)
            for codes, scale, x in ((k, k_scale, randn(n, bt, D) * channel), (v, v_scale, randn(n, bt, D))):
                q, s = _quantized(x.half().double(), fmt)
                codes[i:i + n], scale[i:i + n] = q.float().to(HELD[fmt]), s
    state.update(
        k_codes=k, v_codes=v, k_scale=k_scale, v_scale=v_scale, k_tail=(randn(B, H, bt, D) * channel).half(), v_tail=randn(B, H, bt, D).half(),
        table=torch.randperm(blocks, generator=g, device="cuda").int().view(B, H, width),
        length=torch.tensor(lengths, dtype=torch.int32, device="cuda")[:, None].expand(B, H).contiguous(),
        weight=torch.exp(2.0 * randn(blocks, bt) - 4.0), length_out=torch.zeros((B, H), dtype=torch.int32, device="cuda"))
    if case["op"] == "evict":
        state.update(table_out=torch.zeros_like(state["table"]))
    else:
        rows, group = (max(new) if case["op"] == "append" else case["queries"]), case["q_heads"] // H
        # q, k and v of a token lie in one row, as the stacked linear leaves them
        qkv = torch.empty((B, rows, H * (group + 2), D), dtype=torch.float16, device="cuda")
        qkv[:, :, :H * group] = 1.5 * randn(B, rows, H * group, D) / channel.sqrt()
        qkv[:, :, H * group:H * (group + 1)] = randn(B, rows, H, D) * channel
        qkv[:, :, H * (group + 1):] = randn(B, rows, H, D)
        state.update(q=qkv[:, :, :H * group], k=qkv[:, :, H * group:H * (group + 1)], v=qkv[:, :, H * (group + 1):])
        if case["op"] == "append":
            state.update(counts=torch.tensor(new, dtype=torch.int32, device="cuda"))
            out = (B, max(n + t for n, t in zip(new, lengths)), H, D)
            state.update(k_out=torch.zeros(out, dtype=torch.float16, device="cuda"), v_out=torch.zeros(out, dtype=torch.float16, device="cuda"))
    if own:   # the handle of the same buffers, and the workspace, that a program keeps
        from paper_2511_04477_b200 import binding as spqt

        names = ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "table", "length", "weight")
        state["cache"] = spqt.KVCache(**{n: state[n] for n in names})
        state["ws"] = spqt.new_kv_workspace(state["cache"], case["q_heads"], case.get("queries", 1))
    return state


# ---------------------------------------------------------------- one pass


def run(s):
    if own:
        return _own(s)
    return {"append": _append, "attention": _attention, "evict": _evict, "logprobs": _logprobs}[s["op"]](s)


def _own(s):
    from paper_2511_04477_b200 import binding as spqt

    case = s["case"]
    if s["op"] == "append":
        spqt.spqt_kv_append(s["cache"], s["k"], s["v"], s["ws"], counts=s["counts"], length_out=s["length_out"])
        spqt.spqt_kv_read(s["cache"], s["k_out"], s["v_out"], s["ws"], length=s["length_out"])
        return s["k_out"], s["v_out"], s["k_scale"], s["v_scale"], s["length_out"], s["weight"]
    if s["op"] == "attention":
        out = spqt.spqt_kv_attention(s["cache"], s["q"], s["ws"], accumulate=case["accumulate"])
        return (out, s["weight"]) if case["accumulate"] else out
    if s["op"] == "evict":
        return spqt.spqt_kv_evict(s["cache"], case["keep"], s["ws"], first=case["first"], recent=case["recent"],
                                  table_out=s["table_out"], length_out=s["length_out"])
    return spqt.spqt_token_logprobs(s["logits"], s["tokens"], top=case["top"])


def _read(s, codes, scale, tail, length):
    """[B][H][width * block][dim] in 32 bits; what lies behind the last token is zero."""
    t, (B, H, W), bt = s["table"].long(), s["table"].shape, s["case"]["block"]
    held = codes.view(torch.uint8)[t].view(codes.dtype).float()
    x = held * scale[t][..., None, None]
    at = torch.arange(W, device="cuda")[:, None] * bt + torch.arange(bt, device="cuda")
    n = length[:, :, None, None]
    x = torch.where((at < n // bt * bt)[..., None], x, tail[:, :, None].float())   # the block that is not full, and those behind it
    return torch.where((at < n)[..., None], x, 0.0).flatten(2, 3)


def _append(s):
    case, (B, H, W), bt, D = s["case"], s["table"].shape, s["case"]["block"], s["case"]["dim"]
    new, length = s["k"].shape[1], s["length"]
    count = s["counts"][:, None]
    open_rows, first = length % bt, length // bt           # of the block that is not full
    nb = (bt - 1 + new) // bt + 1                          # blocks that a call can touch
    at = torch.arange(nb * bt, device="cuda").expand(B, H, -1)
    before = open_rows[..., None]
    total = (open_rows + count)[..., None]                 # rows from the beginning of that block on
    block = first[..., None] + torch.arange(nb, device="cuda")
    ids = torch.gather(s["table"], 2, block.clamp(max=W - 1).long()).long()
    closed = (torch.arange(nb, device="cuda") + 1) * bt <= total
    # (behind the end of the table no block is closed: those write what the last entry has, which nothing else writes)
    outs = []
    for x, codes, scale, tail in ((s["k"], s["k_codes"], s["k_scale"], s["k_tail"]), (s["v"], s["v_codes"], s["v_scale"], s["v_tail"])):
        rows = x.transpose(1, 2)                           # [B][H][new][D]
        old = torch.gather(tail, 2, at.clamp(max=bt - 1)[..., None].expand(-1, -1, -1, D).long())
        fresh = torch.gather(rows, 2, (at - before).clamp(0, new - 1)[..., None].expand(-1, -1, -1, D).long())
        stream = torch.where((at < before)[..., None], old, fresh)
        q, sc = _quantized(stream.view(B, H, nb, bt, D).double(), case["fmt"])
        held = q.float().to(codes.dtype).view(torch.uint8)
        raw = codes.view(torch.uint8)
        raw[ids] = torch.where(closed[..., None, None], held, raw[ids])
        scale[ids] = torch.where(closed, sc, scale[ids])
        base = total // bt * bt
        last = torch.gather(stream, 2, (base + at[..., :bt]).clamp(max=nb * bt - 1)[..., None].expand(-1, -1, -1, D).long())
        tail.copy_(torch.where((at[..., :bt] < total - base)[..., None], last, tail))
    written = ((at >= before) & (at < total)).view(B, H, nb, bt)
    s["weight"][ids] = torch.where(written, 0.0, s["weight"][ids])
    s["length_out"].copy_(length + count)
    n = s["length_out"]
    for out, codes, scale, tail in ((s["k_out"], s["k_codes"], s["k_scale"], s["k_tail"]), (s["v_out"], s["v_codes"], s["v_scale"], s["v_tail"])):
        T = out.shape[1]
        x = _read(s, codes, scale, tail, n)[:, :, :T].transpose(1, 2)
        valid = (torch.arange(T, device="cuda")[None, :, None] < n[:, None, :])[..., None]
        out.copy_(torch.where(valid, x.half(), out))
    return s["k_out"], s["v_out"], s["k_scale"], s["v_scale"], s["length_out"], s["weight"]


def _attention(s):
    case, (B, H, W), bt, D = s["case"], s["table"].shape, s["case"]["block"], s["case"]["dim"]
    K, V = (_read(s, s[c], s[sc], s[t], s["length"]) for c, sc, t in (("k_codes", "k_scale", "k_tail"), ("v_codes", "v_scale", "v_tail")))
    Q, group = case["queries"], case["q_heads"] // H
    q = s["q"].float().view(B, Q, H, group, D).permute(0, 2, 1, 3, 4).reshape(B, H, Q * group, D)
    x = (q @ K.transpose(2, 3)).view(B, H, Q, group, W * bt) * D ** -0.5
    seen = s["length"][:, :, None, None, None] - Q + 1 + torch.arange(Q, device="cuda")[:, None, None]
    x = torch.where(torch.arange(W * bt, device="cuda") < seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / torch.where(total > 0, total, 1.0), 0.0)   # a query that sees nothing gets zeros
    out = (p.view(B, H, Q * group, W * bt) @ V).view(B, H, Q, group, D).permute(0, 2, 1, 3, 4).reshape(B, Q, H * group, D).half()
    if not case["accumulate"]:
        return out
    t = s["table"].long()
    s["weight"][t] = s["weight"][t] + p.sum((2, 3)).view(B, H, W, bt)
    return out, s["weight"]


def _evict(s):
    case, (B, H, W), bt = s["case"], s["table"].shape, s["case"]["block"]
    closed = (s["length"] // bt)[..., None]
    j = torch.arange(W, device="cuda")
    score = s["weight"][s["table"].long()].double().sum(-1).float()
    score = torch.where((j < case["first"]) | (j >= closed - case["recent"]), math.inf, score)
    score = torch.where(j < closed, score, -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True)[1]
    rank = torch.empty_like(order).scatter_(-1, order, j.expand(B, H, W))
    kept = (j < closed) & (rank < case["keep"])
    opened = (j == closed) & (s["length"] % bt > 0)[..., None]
    kind = torch.where(kept, 0, torch.where(opened, 1, torch.where(j < closed, 2, 3)))   # kept, not full, free again, not used yet
    s["table_out"].copy_(torch.gather(s["table"], -1, torch.sort(kind, dim=-1, stable=True)[1]))
    s["length_out"].copy_(torch.minimum(closed[..., 0], torch.full_like(s["length"], case["keep"])) * bt + s["length"] % bt)
    return s["table_out"], s["length_out"]


def _ordered(x):
    """Whole numbers in the order of the values: the larger value, then the lower index."""
    bits = (x + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    return (key << 20) - torch.arange(x.shape[-1], device="cuda")


def _logprobs(s):
    x, top = s["logits"].float(), s["case"]["top"]
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    logsum = torch.log(total)
    logprob = (torch.gather(x, 1, s["tokens"].long()[:, None]) - m - logsum)[:, 0]
    entropy = (logsum - torch.where(e > 0, e * (x - m), 0.0).sum(1, keepdim=True) / total)[:, 0]
    key = torch.topk(_ordered(x), top, dim=1)[0]
    index = (-key) & 0xFFFFF
    return logprob, entropy, torch.gather(x, 1, index) - m - logsum, index.int()


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    if case["op"] == "logprobs":
        n, size = case["rows"] * case["vocab"], 4 if case["dtype"] == "fp32" else 2
        return {"bytes": n * size + case["rows"] * (12 + 8 * case["top"]), "flops": 6.0 * n}
    H, D, bt, lengths = case["kv_heads"], case["dim"], case["block"], _lengths(case)
    if case["op"] == "evict":   # the weights of the full blocks, the table twice, the lengths
        return {"bytes": H * sum(t // bt * bt * 4 + 8 * (t // bt) + 8 for t in lengths), "flops": float(H * sum(lengths))}
    if case["op"] == "append":
        total = nbytes = 0
        for n, t in zip(_counts(case, case["new"], 2), lengths):
            end = t + n
            full = end // bt * bt - t // bt * bt          # tokens that become codes, once all are there
            nbytes += 4 * D * (n + (t % bt if full else 0)) + 2 * full * D + 8 * full // bt + 4 * n + 12   # rows in, codes, scales, weights
            nbytes += 4 * D * min(n, end % bt)                                                            # rows of the open block
            nbytes += 2 * D * (end // bt * bt) + 8 * (end // bt) + 4 * D * (end % bt) + 4 * D * end       # read back
            total += end
        return {"bytes": H * nbytes, "flops": 4.0 * H * D * total}
    rows = case["q_heads"] * case["queries"] * case["batch"]
    nbytes = 4 * rows * D
    for t in lengths:
        full = t // bt * bt
        nbytes += H * (2 * D * full + 12 * (full // bt) + 4 * D * (t - full) + 4 + (8 * t if case["accumulate"] else 0))
    return {"bytes": nbytes, "flops": 4.0 * case["q_heads"] * case["queries"] * D * sum(lengths)}


# ---------------------------------------------------------------- the definition in 64 bits


def _nearest(q, fmt):
    """q rounded to what 8 bits can hold, ties to even."""
    if fmt == "int8":
        return torch.round(q).clamp(-127, 127)
    a = q.abs()
    exponent = torch.floor(torch.log2(torch.where(a > 0, a, 1.0)))
    exponent = torch.where(torch.pow(2.0, exponent) > a, exponent - 1, exponent).clamp(min=-6.0)
    ulp = torch.pow(2.0, exponent - 3)
    return torch.sign(q) * torch.clamp(torch.round(a / ulp) * ulp, max=448.0)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "logprobs":
        rows = []
        for i in range(case["rows"]):
            x = s["logits"][i].double()
            logp = x - torch.logsumexp(x, 0)
            p = torch.exp(logp)
            index = torch.sort(x, descending=True, stable=True)[1][:case["top"]]
            rows.append((logp[s["tokens"][i].long()], -(p * torch.where(p > 0, logp, 0.0)).sum(), logp[index], index.int()))
        return tuple(torch.stack(c) for c in zip(*rows))
    B, H, bt, D = case["batch"], case["kv_heads"], case["block"], case["dim"]
    table, length = s["table"].tolist(), s["length"].tolist()
    if case["op"] == "evict":
        new_table, new_length = s["table"].clone(), s["length"].clone()
        for b in range(B):
            for h in range(H):
                n, row = length[b][h], table[b][h]
                closed = n // bt
                if closed <= case["keep"]:
                    continue
                w = s["weight"][s["table"][b, h, :closed].long()].double().sum(1).float().tolist()
                inner = list(range(case["first"], closed - case["recent"]))
                inner.sort(key=lambda j: (-w[j], j))
                keep = set(inner[:case["keep"] - case["first"] - case["recent"]])
                keep |= set(range(case["first"])) | set(range(closed - case["recent"], closed))
                some = [closed] if n % bt else []
                order = sorted(keep) + some + [j for j in range(closed) if j not in keep] + list(range(closed + len(some), len(row)))
                new_table[b, h] = torch.tensor([row[j] for j in order], dtype=torch.int32)
                new_length[b, h] = case["keep"] * bt + n % bt
        return new_table, new_length

    def stream(b, h, kind, n):
        """The n tokens of a (sequence, kv head) as the cache holds them."""
        full = n // bt
        ids = s["table"][b, h, :full].long()
        held = s[kind + "_codes"].view(torch.uint8)[ids].view(HELD[case["fmt"]]).double() * s[kind + "_scale"][ids].double()[:, None, None]
        return torch.cat([held.reshape(-1, D), s[kind + "_tail"][b, h, :n - full * bt].double()])

    if case["op"] == "append":
        outs = {"k": s["k_out"].double(), "v": s["v_out"].double()}
        scales = {"k": s["k_scale"].double(), "v": s["v_scale"].double()}
        weight, new_length = s["weight"].double(), s["length"].clone()
        counts = s["counts"].tolist()
        for b in range(B):
            for h in range(H):
                n, c = length[b][h], counts[b]
                new_length[b, h] = n + c
                for kind in ("k", "v"):
                    old = n // bt * bt
                    x = stream(b, h, kind, n)
                    rows = torch.cat([x[old:], s[kind][b, :c, h].double()])
                    full = rows.shape[0] // bt
                    if full:
                        blocks = rows[:full * bt].view(full, bt, D)
                        scale = (blocks.abs().amax((1, 2)) / LARGEST[case["fmt"]]).float().double()
                        q = _nearest(blocks / torch.where(scale > 0, scale, 1.0)[:, None, None], case["fmt"])
                        rows = torch.cat([(q * scale[:, None, None]).reshape(-1, D), rows[full * bt:]])
                        scales[kind][s["table"][b, h, n // bt:n // bt + full].long()] = scale
                    outs[kind][b, :n + c, h] = torch.cat([x[:old], rows])
                at = torch.arange(n, n + c, device="cuda")
                weight[s["table"][b, h].long()[at // bt], at % bt] = 0.0
        return outs["k"], outs["v"], scales["k"], scales["v"], new_length, weight

    Q, group = case["queries"], case["q_heads"] // H
    out = torch.zeros((B, Q, H * group, D), dtype=torch.float64, device="cuda")
    weight = s["weight"].double()
    for b in range(B):
        for h in range(H):
            n = length[b][h]
            if n == 0:
                continue
            K, V = stream(b, h, "k", n), stream(b, h, "v", n)
            at = torch.arange(n, device="cuda")
            for i in range(Q):
                seen = n - Q + i + 1
                if seen <= 0:
                    continue
                p = torch.softmax(s["q"][b, i, h * group:(h + 1) * group].double() @ K[:seen].T / math.sqrt(D), 1)
                out[b, i, h * group:(h + 1) * group] = p @ V[:seen]
                if case["accumulate"]:
                    weight[s["table"][b, h].long()[at[:seen] // bt], at[:seen] % bt] += p.sum(0)
    return (out, weight) if case["accumulate"] else out
