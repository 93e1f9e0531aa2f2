"""The operators on a cache held in 4 bits, as cases that can be timed and compared.

Three operators: ``write`` quantises keys and values as they join a packed cache (from a block of tokens, or from the
caches of an evicting handle), ``read`` gives rows of it back, ``attend`` is the attention of a few queries, or of a
block of them, over it.

A row (one key or one value of one head, d elements) is cut into groups of 32 elements.  Of a group, let x* be the
element of the largest magnitude (the first of them):

    s = fp16(x* / -8), held to +-65504      code = clamp(rint(x / s), -8, 7)  (0 where s = 0)      value = code * s

so that x* has the code -8.  A group that holds a NaN or an infinity reads back as NaN throughout.  Attention runs
over the values: query i of a sample's I queries sees the rows first <= j < length - (I - 1 - i), and a query that sees
none has a row of zeros.
"""
from __future__ import annotations

import math

import torch

own = False
GROUP = 32

# Keys of a case (defaults in parentheses):
#   op       "write" | "read" | "attend"
#   b samples, Hq / Hkv query / KV heads, d head dimension, dtype of the inputs and outputs ("bf16")
#   n        write: the row that the first token goes to, read: the first row read, attend: the longest sample's length
#   I        tokens written, rows read, queries of a sample (1)
#   ragged   samples of unequal length (False): none, one and all of the tokens or rows among them
#   padded   attend: left-padded samples (False), among them one that is padding throughout
#   fused    q, k and v are views of one tensor, as a fused projection leaves them (False)
#   handle   write: the rows come from the caches of an evicting handle (False)


def _case(name=None, **kw):
    case = dict(I=1, dtype="bf16", ragged=False, padded=False, fused=False, handle=False)
    case.update(kw)
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # a decode step's pairs join the caches of a serving batch: the smallest write, latency alone
        _case("write_token", op="write", b=16, Hq=32, Hkv=8, d=128, n=1024, fused=True),
        # a block of a prompt, straight from the fused projection
        _case("write_block", op="write", b=16, Hq=32, Hkv=8, d=128, n=1024, I=512, fused=True),
        # prompts of unequal length in single precision; odd sizes
        _case("write_ragged_f32", op="write", b=5, Hq=6, Hkv=3, d=64, n=77, I=901, dtype="f32", ragged=True),
        # the caches that an evicting prefill left are packed for decoding
        _case("write_from_handle", op="write", b=64, Hq=32, Hkv=8, d=128, n=0, I=1024, handle=True),
        # a whole batch's caches are read back
        _case("read_caches", op="read", b=16, Hq=32, Hkv=8, d=128, n=0, I=4096),
        # single precision, odd sizes, samples that end early
        _case("read_ragged_f32", op="read", b=7, Hq=4, Hkv=4, d=64, n=13, I=1501, dtype="f32", ragged=True),
        # the smallest attention: a handful of heads in single precision, as in unit tests and debugging
        _case("attend_tiny_f32", op="attend", b=2, Hq=4, Hkv=4, d=64, n=512, dtype="f32"),
        # a decode step of a serving batch: grouped heads, samples of unequal length, some left-padded
        _case("attend_serving", op="attend", b=16, Hq=32, Hkv=8, d=128, n=4096, ragged=True, padded=True, fused=True),
        # a decode step of the batch that packing is for; an odd length
        _case("attend_large_batch", op="attend", b=384, Hq=32, Hkv=8, d=128, n=1535),
        # multi-head attention, no grouping, the 40-head shape of the larger model
        _case("attend_multi_head", op="attend", b=32, Hq=40, Hkv=40, d=128, n=2048),
        # one user, a very long context
        _case("attend_long", op="attend", b=1, Hq=32, Hkv=8, d=128, n=131072),
        # a block of a prompt attends to what is cached and to itself
        _case("attend_block", op="attend", b=4, Hq=32, Hkv=8, d=128, n=4352, I=256, fused=True),
    ]


def _between(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _draw_one(rng, values):
    op = rng.choice(["write", "read", "attend", "attend"])
    d, dtype = rng.choice([128, 128, 64]), rng.choice(["bf16", "bf16", "f32"])
    g, Hkv = rng.choice([1, 2, 4, 4, 8]), _between(rng, 1, 40)
    case = dict(op=op, Hq=g * Hkv, Hkv=Hkv, d=d, dtype=dtype, ragged=rng.random() < 0.4)
    if op == "write":
        if rng.random() < 0.25:
            case.update(handle=True, ragged=False, n=0, I=_between(rng, 16, 1200))
        else:
            case.update(n=rng.randint(0, 2000), I=_between(rng, 1, 5000), fused=rng.random() < 0.5)
        rows, most = case["I"], 128
    elif op == "read":
        case.update(n=rng.choice([0, 0, rng.randint(1, 500)]), I=_between(rng, 1, 5000))
        rows, most = case["I"], 64
    else:
        I = rng.choice([1, 1, 1, 1, _between(rng, 2, 8), _between(rng, 2, 300)])
        case.update(n=_between(rng, max(I, 8), 140000), I=I, padded=rng.random() < 0.25, fused=rng.random() < 0.5)
        rows, most = case["n"], 384
    # as many samples as leave the caches within the listed cases' sizes
    return _case(b=_between(rng, 1, max(1, min(most, values // (rows * Hkv * d)))), **case)


def _size(case):
    w = work(case)
    return w["bytes"] / 6e12 + w["flops"] / (1e15 if case["dtype"] == "bf16" else 2e14)


def draw(rng):
    most, values = max(_size(c) for c in listed()), 400_000_000    # keys of the largest listed caches
    while True:
        case = _draw_one(rng, values)
        rows = case["n"] if case["op"] == "attend" else case["n"] + case["I"]
        weights = case["b"] * case["Hq"] * case["I"] * case["n"] if case["op"] == "attend" else 0
        if _size(case) <= most and case["b"] * case["Hkv"] * case["d"] * rows <= 3 * values and weights <= values:
            return case


def _spread(count, most):
    """`count` whole numbers between 0 and `most`: all, none and one first, then evenly spread."""
    fixed = [most, 0, min(1, most)]
    return [fixed[s] if s < 3 else round(most * (0.5 + 0.618034 * s) % most) if most > 0 else 0 for s in range(count)]


def _counts(case):
    """How many of a sample's tokens, rows or cached pairs there are."""
    most = case["n"] if case["op"] == "attend" else case["I"]
    return _spread(case["b"], most) if case["ragged"] else [most] * case["b"]


def _first(case):
    """The first row that counts, per sample: the last sample is padding throughout where there are several."""
    lens = _counts(case)
    if not case["padded"]:
        return [0] * case["b"]
    first = [n * (7 * s % 5) // 10 for s, n in enumerate(lens)]
    if case["b"] > 1:
        first[-1] = lens[-1]
    return first


def _visible(case):
    """(rows that some query of a sample sees, pairs of a query and a row it sees), summed over the samples."""
    rows = pairs = 0
    I = case["I"]
    for n, first in zip(_counts(case), _first(case)):
        rows += max(0, n - first)
        longest = max(0, n - first)                 # rows of the last query; the ones before it see one less each
        shown = min(I, longest)
        pairs += shown * longest - shown * (shown - 1) // 2
    return rows, pairs


def work(case):
    """Each input read once and each output written once.  A packed row is d/2 bytes of codes and d/16 of scales."""
    e, d, Hkv, Hq, I = 2 if case["dtype"] == "bf16" else 4, case["d"], case["Hkv"], case["Hq"], case["I"]
    packed = d // 2 + d // 16
    if case["op"] == "attend":
        rows, pairs = _visible(case)
        return {"bytes": 2 * rows * Hkv * packed + 2 * case["b"] * I * Hq * d * e, "flops": 4 * d * pairs * Hq}
    kept, asked = 2 * sum(_counts(case)) * Hkv, 2 * case["b"] * I * Hkv
    if case["op"] == "read":
        return {"bytes": kept * packed + asked * d * e, "flops": kept * d}
    # the rows come in, their packed form and the values it stands for go out
    return {"bytes": kept * (d * e + packed) + asked * d * e, "flops": 4 * kept * d}


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs(case, seed):
    """q (attend), k, v of the case.  A few channels of the keys are several times larger than the others and off
    centre, as keys are behind a rotary embedding; values and queries are even."""
    gen = torch.Generator(device="cuda").manual_seed(7919 * seed + 11)
    b, Hq, Hkv, d = case["b"], case["Hq"], case["Hkv"], case["d"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32 if case["dtype"] == "f32" else torch.bfloat16)

    def keys(tokens):
        k = normal(b, tokens, Hkv, d)
        k[..., 5::41] *= 5.0
        k[..., 5::41] += 3.0
        return k

    q = k = v = None
    tokens = case["n"] if case["op"] == "attend" else case["I"]
    if case["fused"] and case["op"] == "write":
        qkv = normal(b, tokens, Hq + 2 * Hkv, d)
        k, v = qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
        k.copy_(keys(tokens))
    else:
        k, v = keys(tokens), normal(b, tokens, Hkv, d)
    if case["op"] == "attend":
        I = case["I"]
        q = normal(b, I, Hq + 2 * Hkv, d)[:, :, :Hq] if case["fused"] else normal(b, I, Hq, d)
    return q, k, v


def _quantise(x):
    """Codes (int8, (..., d / 32, 32)) and scales (fp16, (..., d / 32)) of rows x (..., d).  A quotient of 24 bits by 11
    is never nearer to a half than 32 bits tell apart, so nothing is lost by them here."""
    x = x.float().unflatten(-1, (-1, GROUP))
    size = x.abs()
    most = size.amax(-1, keepdim=True)
    place = torch.arange(GROUP, device=x.device, dtype=torch.int32)
    first = torch.where(size == most, place, GROUP - 1).amin(-1, keepdim=True)
    s = (x.gather(-1, first.long()) / -8.0).clamp(-65504.0, 65504.0)
    s = torch.where(torch.isfinite(most), s, math.nan).half()
    code = torch.round(x / s.float()).clamp(-8.0, 7.0)
    code = torch.where((s == 0) | ~torch.isfinite(most), 0.0, code)
    return code.to(torch.int8), s.squeeze(-1)


def _values(code, s):
    return (code.float() * s.float().unsqueeze(-1)).flatten(-2)


def prepare(case, seed):
    q, k, v = _inputs(case, seed)
    b, d, I, n, op = case["b"], case["d"], case["I"], case["n"], case["op"]
    counts = torch.tensor(_counts(case), dtype=torch.int32, device="cuda")
    first = torch.tensor(_first(case), dtype=torch.int32, device="cuda") if case["padded"] else None
    state = {"op": op, "I": I, "n": n, "q": q, "first": first, "lens": counts, "dtype": _dtype(case),
             "group": case["Hq"] // case["Hkv"]}
    if op == "write":
        state.update(k=k, v=v, counts=counts if case["ragged"] else None,
                     start=torch.full((b,), n, dtype=torch.int32, device="cuda"), lens=counts + n)
    elif op == "read":
        state.update(lens=counts + n if case["ragged"] else None)
    if not own:
        if op != "write":
            state["k"], state["v"] = _quantise(k), _quantise(v)
            state["counts"] = counts if case["ragged"] else None
        return state
    from paper_2412_05693_b200 import BatchMaxCache, Config, PackedCache, PackedConfig
    capacity = n if op == "attend" else n + I
    cache = PackedCache(PackedConfig(batch=b, n_q_heads=case["Hq"], n_kv_heads=case["Hkv"], head_dim=d, capacity=capacity,
                                     queries_max=I if op == "attend" else 1, dtype=case["dtype"]))
    state["cache"] = cache
    if op == "write":
        if case["handle"]:   # the caches as a prefill without a cut leaves them: the tokens' pairs in order
            cfg = Config(batch=b, n_q_heads=case["Hq"], n_kv_heads=case["Hkv"], head_dim=d, kv_max=I, block_max=I,
                         dtype=case["dtype"])
            state["handle"] = BatchMaxCache(cfg)
            queries = torch.zeros(b, I, case["Hq"], d, dtype=state["dtype"], device="cuda")
            state["handle"].prefill_block(queries, k, v, 0)
    else:
        start = torch.full((b,), n if op == "read" else 0, dtype=torch.int32, device="cuda")
        cache.write(k, v, start=start)
    return state


def run(state):
    if own:
        cache = state["cache"]
        if state["op"] == "attend":
            return cache.attend(state["q"], state["lens"], first=state["first"])
        if state["op"] == "write":
            if "handle" in state:
                cache.write_from(state["handle"])
            else:
                cache.write(state["k"], state["v"], start=state["start"], counts=state["counts"])
        return cache.read(state["n"], state["I"], lens=state["lens"])
    if state["op"] == "attend":
        return _attend(state)
    out = []
    for x in (state["k"], state["v"]):
        x = _values(*(_quantise(x) if state["op"] == "write" else x))
        if state["counts"] is not None:
            there = torch.arange(state["I"], device="cuda") < state["counts"][:, None]
            x = torch.where(there[:, :, None, None], x, 0.0)
        out.append(x.to(state["dtype"]))
    return tuple(out)


def _attend(state):
    q, lens, I, n, g = state["q"], state["lens"], state["I"], state["n"], state["group"]
    b, _, Hq, d = q.shape
    k, v = (_values(*x).transpose(1, 2) for x in (state["k"], state["v"]))      # (b, Hkv, n, d)
    q = q.float().view(b, I, Hq // g, g, d).permute(0, 2, 1, 3, 4).reshape(b, Hq // g, I * g, d)
    logits = (q @ k.transpose(-1, -2)).view(b, Hq // g, I, g, n) / math.sqrt(d)
    row, query = torch.arange(n, device="cuda"), torch.arange(I, device="cuda")
    seen = row < lens[:, None, None] - (I - 1 - query)[:, None]                  # (b, I, n)
    if state["first"] is not None:
        seen = seen & (row >= state["first"][:, None, None])
    seen = seen[:, None, :, None, :]
    logits = torch.where(seen, logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    weights = torch.exp(logits - torch.where(top == -math.inf, 0.0, top))
    total = weights.sum(-1, keepdim=True)
    out = weights.view(b, Hq // g, I * g, n) @ v
    out = out.view(b, Hq // g, I, g, d) / torch.where(total == 0, 1.0, total)
    return out.permute(0, 2, 1, 3, 4).reshape(b, I, Hq, d).to(state["dtype"])


def exact(case, seed):
    """The same from the definition in 64 bits, group by group and sample by sample."""
    q, k, v = _inputs(case, seed)
    b, Hkv, I, d, n, op = case["b"], case["Hkv"], case["I"], case["d"], case["n"], case["op"]
    counts, first = _counts(case), _first(case)

    def stands_for(x):    # (tokens, Hkv, d) -> what its packed form stands for
        x = x.double()
        parts = []
        for at in range(0, d, GROUP):
            part = x[..., at:at + GROUP]
            top, low = part.max(-1).values, -part.min(-1).values
            hit = part.abs() == torch.maximum(top, low)[..., None]
            hit &= hit.cumsum(-1) == 1
            s = ((part * hit).sum(-1, keepdim=True) * -0.125).clamp(-65504, 65504).half().double()
            parts.append(torch.where(s == 0, 0.0, torch.clamp(torch.round(part / torch.where(s == 0, 1.0, s)), -8, 7) * s))
        return torch.cat(parts, -1)

    if op != "attend":
        outs = []
        for x in (k, v):
            out = torch.zeros(b, I, Hkv, d, dtype=torch.float64, device="cuda")
            for s in range(b):
                out[s, :counts[s]] = stands_for(x[s, :counts[s]])
            outs.append(out)
        return tuple(outs)
    Hq = case["Hq"]
    out = torch.zeros(b, I, Hq, d, dtype=torch.float64, device="cuda")
    for s in range(b):
        if counts[s] <= first[s]:
            continue
        ks, vs = stands_for(k[s, first[s]:counts[s]]), stands_for(v[s, first[s]:counts[s]])
        rows = counts[s] - first[s]
        hidden = torch.arange(rows, device="cuda") > rows - I + torch.arange(I, device="cuda")[:, None]
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            score = (q[s, :, h].double() @ ks[:, kv].T) * d ** -0.5
            share = torch.softmax(score.masked_fill(hidden, -math.inf), -1)
            out[s, :, h] = torch.where(hidden.all(-1, keepdim=True), 0.0, share) @ vs[:, kv]
    return out
