"""Performance cases of the operators around a pruned decoder's blocks whose scores and norms are of other forms than the plain ones.

  attention  attention over packed sequences whose scores are capped by a tanh, fall with the distance by a slope of each head, get a
             learned bias by the bucket of their distance, or see a sequence's first keys from everywhere:
                 z_ij = cap tanh(scale q_i k_j / cap) - slope |d| + table[bucket(d)],   d = i - j counted from the sequence's end
             in training with the gradients of Q, K, V and of the table
  norm       what lies between a block's output and the next block's input: a norm behind the block, its gate and residual scale,
             the sum with the residual stream, and the next block's norm
                 n = N(y) w_y + b_y (or y),   s' = s + scale gate n,   out = N(s') w + b
             in training with the gradients of the stream, of y and of the five vectors

`run` computes them in plain form, elementary torch operations in 32 bits (sums over many tokens in 64) rounded once at the end, where
`own` is false, and by the calls of `paper_2302_05045_amd` where it is true.

Both take the same state, which `prepare` makes from the seed alone: fp16 activations and weights of a layer under way, a residual
stream in fp16 or fp32, gradients multiplied by the loss scale.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-5


# ------------------------------------------------------------------ the cases
def _attention(tokens, seqs, heads, kv_heads, dim, train=True, context=0, causal=True, window=0, cap=0.0, slopes=False, buckets=0, far=0,
               seen=0.0) -> dict:
    """context: keys in front of every sequence's queries; buckets: of one direction, from `far` on the last one; seen: the share of a
    sequence's keys that all of its queries see."""
    return dict(op="attention", train=train, tokens=tokens, seqs=seqs, context=context, heads=heads, kv_heads=kv_heads, dim=dim, causal=causal,
                window=window, cap=cap, slopes=slopes, buckets=buckets, far=far, seen=seen)


def _norm(tokens, hidden, train=True, kind="rms", after="norm", gate=True, bias=False, scale=1.0, stream32=False) -> dict:
    """after: what becomes of the block's output ("norm", "plain"; "": there is none, the norm before the first block)."""
    return dict(op="norm", train=train, tokens=tokens, hidden=hidden, kind=kind, after=after, gate=gate, bias=bias, scale=scale, stream32=stream32)


def listed() -> list:
    return [
        # a handful of one-token to few-token prompts scored together, capped: the latency of a small call
        dict(_attention(61, 9, 16, 16, 64, cap=50.0), name="attention_cap_short"),
        # the 2.7B shape (heads of 80): four sequences of 2048 tokens with capped scores, training
        dict(_attention(8192, 4, 32, 32, 80, cap=50.0), name="attention_cap_2.7b"),
        # the 6.7B width over one long context, positions by distance alone, keys and values shared by four heads each, training
        dict(_attention(8192, 1, 32, 8, 128, slopes=True), name="attention_slopes_6.7b_long"),
        # the 350M shape: packed sequences of uneven length whose first part is read in both directions, training
        dict(_attention(4093, 7, 16, 16, 64, seen=0.3), name="attention_prefix_350m_ragged"),
        # generation: one token each of five sequences behind long contexts, capped, a sliding window and the first keys
        dict(_attention(5, 5, 32, 8, 128, train=False, context=4001, window=2048, cap=30.0, seen=0.01), name="attention_cap_token"),
        # the 350M shape with a learned bias by the distance's bucket, training
        dict(_attention(4093, 7, 16, 16, 64, buckets=32, far=128), name="bias_350m_ragged"),
        # an encoder's shape: every token sees every other, buckets of both directions, training
        dict(_attention(8192, 8, 12, 12, 64, causal=False, buckets=16, far=128), name="bias_both_sides"),
        # generation: one token each of three sequences behind contexts, learned bias
        dict(_attention(3, 3, 16, 16, 64, train=False, context=2047, buckets=32, far=128), name="bias_token"),
        # generation: one token through the norms around a block
        dict(_norm(1, 2560, train=False), name="norm_token"),
        # the 350M width, a micro-batch of odd length, layer norm with its bias in front of the next block, training
        dict(_norm(1003, 1024, kind="layer", after="plain", gate=False, bias=True), name="norm_350m_layer"),
        # the 2.7B width, one sequence: norms before and after the block, gate, a residual stream in 32 bits, training
        dict(_norm(2048, 2560, scale=0.5, stream32=True), name="norm_2.7b_sandwich32"),
        # the 6.7B width, four sequences: norms before and after the block, gate, training
        dict(_norm(8192, 4096, scale=0.5), name="norm_6.7b_sandwich"),
    ]


def _log_int(rng, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng) -> dict:
    if rng.random() < 0.4:
        kind, after, train = rng.choice(["rms", "layer"]), rng.choice(["norm", "norm", "plain", ""]), rng.random() < 0.7
        return _norm(_log_int(rng, 16 if train else 1, 8192), 8 * _log_int(rng, 8, 512), train, kind, after, gate=after != "" and rng.random() < 0.6,
                     bias=kind == "layer" or rng.random() < 0.3, scale=rng.choice([1.0, 0.5, 0.22]), stream32=rng.random() < 0.4)
    kv, train, causal = rng.choice([1, 2, 4, 8, 16]), rng.random() < 0.7, rng.random() < 0.75
    tokens = _log_int(rng, 16 if train else 1, 8192 if causal else 5600)
    buckets = rng.choice([0, 8, 16, 32, 64]) if rng.random() < 0.6 else 0
    return _attention(tokens, min(_log_int(rng, 1, 16), tokens), kv * rng.choice([1, 2, 4] if kv < 16 else [1, 2]), kv, 8 * rng.randint(4, 16), train,
                      context=0 if train else rng.choice([0, _log_int(rng, 1, 2048)]), causal=causal,
                      window=_log_int(rng, 16, 4096) if causal and rng.random() < 0.25 else 0, cap=rng.choice([0.0, 0.0, 30.0, 50.0]),
                      slopes=buckets == 0 and rng.random() < 0.5, buckets=buckets, far=_log_int(rng, 80, 2000) if buckets else 0,
                      seen=round(rng.uniform(0.01, 0.6), 3) if causal and rng.random() < 0.3 else 0.0)


# ------------------------------------------------------------------ inputs
def _normal(shape, std: float, gen, mean: float = 0.0) -> torch.Tensor:
    return (torch.randn(shape, device="cuda", generator=gen, dtype=torch.float32) * std + mean).half()


def _lengths(case: dict) -> list:
    """Tokens of every sequence: uneven unless they divide evenly; the sum is the case's tokens."""
    tokens, seqs = case["tokens"], case["seqs"]
    if tokens % seqs == 0:
        return [tokens // seqs] * seqs
    weights = [1.0 + 3.0 * ((0.618034 * (i + 1)) % 1.0) for i in range(seqs)]
    lens = [max(1, int(tokens * w / sum(weights))) for w in weights]
    while sum(lens) > tokens:
        lens[lens.index(max(lens))] -= 1
    lens[-1] += tokens - sum(lens)
    return lens


def _first_keys(case: dict) -> list:
    """Keys of every sequence that all of its queries see."""
    return [int(case["seen"] * (n + case["context"])) for n in _lengths(case)]


def _prepare_attention(case: dict, gen) -> dict:
    lens = _lengths(case)
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    tq, klens = sum(lens), [n + case["context"] for n in lens]
    tk = sum(klens)
    st = dict(op="attention", train=case["train"], causal=case["causal"], window=case["window"], scale=1.0 / math.sqrt(d), cap=case["cap"],
              buckets=case["buckets"], far=case["far"], max_q=max(lens), max_k=max(klens))
    start = lambda ns: torch.tensor([sum(ns[:i]) for i in range(len(ns) + 1)], dtype=torch.int32).cuda()
    st["q_start"], st["k_start"] = start(lens), start(klens)
    st["first_keys"] = torch.tensor(_first_keys(case), dtype=torch.int32).cuda() if case["seen"] else None
    # a slope of each head, from 2^-8 to 1/2
    st["slopes"] = torch.tensor([2.0 ** (-8.0 * (1 + i) / h) for i in range(h)]).cuda() if case["slopes"] else None
    st["table"] = st["dtable"] = None
    if case["buckets"]:
        columns = case["buckets"] * (1 if case["causal"] else 2)
        st["table"] = _normal((h, columns), 0.5, gen)
        st["dtable"] = torch.zeros((h, columns), dtype=torch.float16, device="cuda")
    if tq == tk:                                       # slices of the QKV projection's output, and of its gradient
        qkv = _normal((tq, (h + 2 * hk) * d), 1.0, gen)
        dqkv = torch.zeros_like(qkv)
        cut = lambda t: (t[:, :h * d].view(tq, h, d), t[:, h * d:(h + hk) * d].view(tq, hk, d), t[:, (h + hk) * d:].view(tq, hk, d))
        st["q"], st["k"], st["v"] = cut(qkv)
        st["dq"], st["dk"], st["dv"] = cut(dqkv)
    else:
        st["q"], st["k"], st["v"] = (_normal((t, n, d), 1.0, gen) for t, n in ((tq, h), (tk, hk), (tk, hk)))
    st["out"] = torch.zeros((tq, h, d), dtype=torch.float16, device="cuda")
    st["lse"] = torch.zeros((h, tq), dtype=torch.float32, device="cuda")
    st["dout"] = _normal((tq, h, d), 1.0, gen)
    if own:                                            # the scores' form, which a program keeps beside its weights
        import paper_2302_05045_amd as samo
        st["scores"] = samo.Scores(cap=case["cap"], slopes=st["slopes"], table=st["table"], first_keys=st["first_keys"], two_sided=not case["causal"],
                                   borders=samo.samo_bucket_borders(case["buckets"], case["far"]) if case["buckets"] else None)
    return st


def _prepare_norm(case: dict, gen) -> dict:
    t, h = case["tokens"], case["hidden"]
    st = dict(op="norm", train=case["train"], kind=case["kind"], after=case["after"], scale=case["scale"])
    stream = torch.float32 if case["stream32"] else torch.float16
    st["stream"] = _normal((t, h), 2.0, gen, 0.1).to(stream)
    st["weight"], y_weight, bias, y_bias, gate = (_normal((h,), 0.1, gen, mean) for mean in (1.0, 1.0, 0.0, 0.0, 0.5))
    st["bias"] = bias if case["bias"] else None
    st["y"] = _normal((t, h), 1.5, gen) if case["after"] else None
    st["y_weight"] = y_weight if case["after"] == "norm" else None
    st["y_bias"] = y_bias if case["after"] == "norm" and case["bias"] else None
    st["gate"] = gate if case["gate"] else None
    st["out"] = torch.zeros((t, h), dtype=torch.float16, device="cuda")
    st["new_stream"] = torch.zeros_like(st["stream"]) if case["after"] else None
    if case["train"]:
        st["dout"] = _normal((t, h), 1.0, gen)
        st["dnew"] = _normal((t, h), 1.0, gen).to(stream)
        st["dstream"] = torch.zeros_like(st["stream"])
        st["dy"] = torch.zeros((t, h), dtype=torch.float16, device="cuda") if case["after"] else None
        st["stats"] = torch.zeros((t, 4), dtype=torch.float32, device="cuda")
        for name in ("weight", "bias", "y_weight", "y_bias", "gate"):
            st["d" + name] = None if st[name] is None else torch.zeros(h, dtype=torch.float16, device="cuda")
    if own:                                            # a layer's vectors, which a program keeps, and those of its gradient
        import paper_2302_05045_amd as samo
        names = ("weight", "bias", "y_weight", "y_bias", "gate")
        st["norm"] = samo.Norm(kind=case["kind"], eps=EPS, y_norm=case["after"] == "norm", scale=case["scale"], **{n: st[n] for n in names})
        st["grads"] = samo.NormGrads(**{n: st["d" + n] for n in names}) if case["train"] else None
    return st


def prepare(case: dict, seed: int) -> dict:
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return {"attention": _prepare_attention, "norm": _prepare_norm}[case["op"]](case, gen)


# ------------------------------------------------------------------ plain forms
def _padded(t: torch.Tensor, start: torch.Tensor, longest: int):
    """(sequences, heads, longest, dim) in 32 bits, which rows there are, and the lengths."""
    lens = (start[1:] - start[:-1]).long()
    row = torch.arange(longest, device=t.device)
    there = row < lens[:, None]
    at = torch.where(there, start[:-1].long()[:, None] + row, 0)
    return (t[at].float() * there[:, :, None, None]).permute(0, 2, 1, 3).contiguous(), there, lens


def _borders(buckets: int, far: int) -> list:
    """The distances at which the next bucket begins: one distance a bucket up to half of them, then by equal steps of the logarithm up to
    `far`, which begins the last but for its share.  In whole numbers: n^rest >= one^(rest - t) far^t."""
    one = buckets // 2
    rest = buckets - one
    least = lambda t: int(one * (far / one) ** (t / rest))
    first = lambda t: next(n for n in range(max(1, least(t) - 2), least(t) + 3) if n ** rest >= one ** (rest - t) * far ** t)
    return list(range(1, one + 1)) + [first(t) for t in range(1, rest)]


def _bucket(d: torch.Tensor, st: dict) -> torch.Tensor:
    """Column of the table for distances i - j."""
    borders = torch.tensor(_borders(st["buckets"], st["far"]), device=d.device)
    if st["causal"]:
        return torch.bucketize(d.clamp(min=0), borders, right=True)
    return torch.bucketize(d.abs(), borders, right=True) + torch.where(d < 0, st["buckets"], 0)


def _attention_plain(st: dict):
    q, q_there, q_lens = _padded(st["q"], st["q_start"], st["max_q"])
    k, k_there, k_lens = _padded(st["k"], st["k_start"], st["max_k"])
    v = _padded(st["v"], st["k_start"], st["max_k"])[0]
    group = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    i = torch.arange(st["max_q"], device=q.device)[:, None] + (k_lens - q_lens)[:, None, None]
    j = torch.arange(st["max_k"], device=q.device)[None, None, :]
    seen = (q_there[:, :, None] & k_there[:, None, :])
    if st["causal"]:
        near = j <= i
        if st["window"]:
            near = near & (j > i - st["window"])
        if st["first_keys"] is not None:
            near = near | (j < st["first_keys"][:, None, None])
        seen = seen & near
    seen = seen[:, None]
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * st["scale"]
    slope = None
    if st["cap"]:
        slope = torch.tanh(s / st["cap"])
        s = slope * st["cap"]
        slope = 1.0 - slope * slope
    if st["slopes"] is not None:
        s = s - st["slopes"][:, None, None] * (i - j).abs()[:, None]
    if st["table"] is not None:
        s = s + st["table"].float()[:, _bucket(i - j, st)].permute(1, 0, 2, 3)
    s = torch.where(seen, s, -math.inf)
    top = s.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(s - top)
    del s
    total = e.sum(3, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    del e
    o = torch.matmul(p, v)
    lse = (top + torch.log(total)).squeeze(3)
    heads = lambda t, there: t.permute(0, 2, 1, 3)[there]
    out, lse_packed = heads(o, q_there), lse.permute(0, 2, 1)[q_there].t().contiguous()
    if not st["train"]:
        return out.half(), lse_packed
    do = _padded(st["dout"], st["q_start"], st["max_q"])[0]
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = p * (torch.matmul(do, v.transpose(2, 3).contiguous()) - (do * o).sum(3, keepdim=True))
    del p
    dtable = None if st["table"] is None else _table_gradient(ds, k_lens - q_lens, st)
    if slope is not None:
        ds = ds * slope
        del slope
    ds = ds * st["scale"]
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    shared = lambda t: t.view(t.shape[0], -1, group, t.shape[2], t.shape[3]).sum(2)
    grads = (out.half(), lse_packed, heads(dq, q_there).half(), heads(shared(dk), k_there).half(), heads(shared(dv), k_there).half())
    return grads if dtable is None else grads + (dtable.half(),)


def _table_gradient(ds: torch.Tensor, shift: torch.Tensor, st: dict) -> torch.Tensor:
    """The sums of ds over every bucket, in 64 bits from the diagonals' on.  With rows n + m apart and the first of them last, a matrix read at rows
    one shorter has a diagonal in each column."""
    b, h, n, m = ds.shape
    apart = torch.nn.functional.pad(ds.flip(2), (0, n)).view(b, h, n * (n + m))[:, :, :n * (n + m - 1)]
    diagonals = apart.view(b, h, n, n + m - 1).sum(2, dtype=torch.float64)                 # column c: row n - 1 - r, key c - r: j - i = c - n + 1
    d = (n - 1) - torch.arange(n + m - 1, device=ds.device)[None, :] + shift[:, None]
    columns = st["table"].shape[1]
    member = (_bucket(d, st)[:, :, None] == torch.arange(columns, device=ds.device)).double()
    return (diagonals[:, :, :, None] * member[:, None]).sum((0, 2))


def _centred(x: torch.Tensor, kind: str):
    """x without its row's mean (layer), in units of its row's root mean square, and that root's reciprocal."""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    return x * r, r


def _through(g: torch.Tensor, x: torch.Tensor, r: torch.Tensor, kind: str) -> torch.Tensor:
    """The gradient in front of a norm from the one behind it."""
    if kind == "layer":
        g = g - g.mean(1, keepdim=True)
    return r * (g - x * (g * x).mean(1, keepdim=True))


def _norm_plain(st: dict):
    f = lambda name, other: other if st[name] is None else st[name].float()
    kind, s = st["kind"], st["stream"].float()
    stream = st["stream"].dtype
    factor = st["scale"] * f("gate", 1.0)
    if st["after"]:
        y = n = st["y"].float()
        if st["after"] == "norm":
            y, ry = _centred(y, kind)
            n = y * f("y_weight", 1.0) + f("y_bias", 0.0)
        s = s + factor * n
    x, r = _centred(s, kind)
    out = (x * f("weight", 1.0) + f("bias", 0.0)).half()
    first = (s.to(stream), out) if st["after"] else (out,)
    if not st["train"]:
        return first
    over = lambda t: t.sum(0, dtype=torch.float64).half()                                 # tokens
    dout = st["dout"].float()
    dweight, dbias = over(dout * x), over(dout) if st["bias"] is not None else None
    ds = st["dnew"].float() + _through(dout * f("weight", 1.0), x, r, kind)
    dy = dgate = dy_weight = dy_bias = None
    if st["after"]:
        dn = factor * ds
        dgate = over(st["scale"] * n * ds) if st["gate"] is not None else None
        dy = dn
        if st["after"] == "norm":
            dy_weight, dy_bias = over(dn * y), over(dn) if st["y_bias"] is not None else None
            dy = _through(dn * f("y_weight", 1.0), y, ry, kind)
        dy = dy.half()
    grads = (ds.to(stream), dy, dweight, dbias, dy_weight, dy_bias, dgate)
    return first + tuple(t for t in grads if t is not None)


# ------------------------------------------------------------------ the framework's calls
def _attention_own(st: dict):
    import paper_2302_05045_amd as samo
    mask = dict(causal=st["causal"], window=st["window"], scale=st["scale"], q_start=st["q_start"], k_start=st["k_start"], max_q=st["max_q"],
                scores=st["scores"])
    samo.samo_attention(st["q"], st["k"], st["v"], st["out"], st["lse"], **mask)
    if not st["train"]:
        return st["out"], st["lse"]
    samo.samo_attention_backward(st["dout"], st["q"], st["k"], st["v"], st["out"], st["lse"], st["dq"], st["dk"], st["dv"], max_k=st["max_k"],
                                 dtable=st["dtable"], **mask)
    grads = (st["out"], st["lse"], st["dq"], st["dk"], st["dv"])
    return grads if st["dtable"] is None else grads + (st["dtable"],)


def _norm_own(st: dict):
    import paper_2302_05045_amd as samo
    first = (st["new_stream"], st["out"]) if st["after"] else (st["out"],)
    if not st["train"]:
        samo.samo_norm(st["norm"], st["stream"], st["out"], y=st["y"], new_stream=st["new_stream"])
        return first
    samo.samo_norm(st["norm"], st["stream"], st["out"], y=st["y"], new_stream=st["new_stream"], stats=st["stats"])
    samo.samo_norm_backward(st["norm"], st["dout"], st["new_stream"] if st["after"] else st["stream"], st["stats"], st["dstream"], dnew=st["dnew"],
                            y=st["y"], dy=st["dy"], grads=st["grads"])
    grads = (st["dstream"], st["dy"], st["dweight"], st["dbias"], st["dy_weight"], st["dy_bias"], st["dgate"])
    return first + tuple(t for t in grads if t is not None)


def run(state: dict):
    """One pass through an operator: forward, in training with its gradients."""
    forms = {"attention": (_attention_plain, _attention_own), "norm": (_norm_plain, _norm_own)}
    return forms[state["op"]][1 if own else 0](state)


# ------------------------------------------------------------------ what a pass cannot do without
def _pairs(case: dict) -> int:
    """Visible (query, key) pairs of all sequences."""
    total = 0
    for n, first in zip(_lengths(case), _first_keys(case)):
        m = n + case["context"]
        if not case["causal"]:
            total += n * m
            continue
        end = np.arange(n, dtype=np.int64) + case["context"] + 1                # keys of every query: begin .. end - 1, and the first ones
        begin = np.maximum(end - case["window"], 0) if case["window"] else np.zeros_like(end)
        total += int((end - begin + np.where(first > end, first - end + begin, np.minimum(begin, first))).sum())
    return total


def work(case: dict) -> dict:
    if case["op"] == "attention":
        lens = _lengths(case)
        tq, tk = sum(lens), sum(n + case["context"] for n in lens)
        q, kv = 2 * tq * case["heads"] * case["dim"], 2 * tk * case["kv_heads"] * case["dim"]
        if case["window"]:                                     # keys that no query sees are not read
            kv = 2 * sum(min(n + case["context"], n + case["window"] + f) for n, f in zip(lens, _first_keys(case))) * case["kv_heads"] * case["dim"]
        products = 2 + (5 if case["train"] else 0)             # S, O; S again, dP, dV, dQ, dK
        nbytes = 2 * q + 2 * kv + 4 * tq * case["heads"] + ((2 * q + 2 * kv) if case["train"] else 0)
        return dict(bytes=nbytes, flops=2 * products * _pairs(case) * case["heads"] * case["dim"])
    n, h, stream = case["tokens"] * case["hidden"], case["hidden"], 4 if case["stream32"] else 2
    nbytes = n * (stream + 2)                                  # stream, out
    if case["after"]:
        nbytes += n * (stream + 2)                             # y, the new stream
    if case["train"]:
        nbytes += n * (2 + 3 * stream)                         # dout, the new stream again, its gradient, that of the stream
        nbytes += n * (2 if case["after"] else 0) + n * (2 if case["after"] == "norm" or case["gate"] else 0)     # dy; y again, where it is needed
    return dict(bytes=nbytes + 2 * h, flops=0)


# ------------------------------------------------------------------ from the definitions, in 64 bits
def _column(d: torch.Tensor, buckets: int, far: int, both: bool) -> torch.Tensor:
    """By the logarithm itself; distances at a border are whole powers' quotients, met within 64 bits' rounding."""
    one, away = buckets // 2, (d.abs() if both else d.clamp(min=0))
    far_part = one + torch.floor(torch.log(away.clamp(min=1).double() / one) / math.log(far / one) * (buckets - one) + 1e-9).long()
    b = torch.where(away < one, away, far_part.clamp(max=buckets - 1))
    return b + buckets * (d < 0) if both else b


def _attention_exact(case: dict, seed: int):
    st = prepare(case, seed)
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    q, k, v, do = (st[n].double() for n in ("q", "k", "v", "dout"))
    out, dq = torch.zeros_like(q), torch.zeros_like(q)
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device="cuda")
    table = None if st["table"] is None else st["table"].double()
    dtable = None if table is None else torch.zeros_like(table)
    q0 = k0 = 0
    for n, first in zip(_lengths(case), _first_keys(case)):
        m = n + case["context"]
        a = torch.arange(n, device="cuda")[:, None] + case["context"]
        b = torch.arange(m, device="cuda")[None, :]
        hidden = torch.zeros((n, m), dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden |= b > a
            if case["window"]:
                hidden |= a - b >= case["window"]
            hidden &= b >= first
        column = None if table is None else _column(a - b, case["buckets"], case["far"], not case["causal"])
        for head in range(h):
            qs, ks, vs = q[q0:q0 + n, head], k[k0:k0 + m, head * hk // h], v[k0:k0 + m, head * hk // h]
            s = qs @ ks.T / math.sqrt(d)
            if case["cap"]:
                s = case["cap"] * torch.tanh(s / case["cap"])
            z = s
            if case["slopes"]:
                z = z - 2.0 ** (-8.0 * (1 + head) / h) * (a - b).abs()
            if table is not None:
                z = z + table[head][column]
            z = z.masked_fill(hidden, -math.inf)
            lse[head, q0:q0 + n] = torch.logsumexp(z, 1)
            prob = torch.softmax(z, 1)
            del z
            out[q0:q0 + n, head] = prob @ vs
            if case["train"]:
                g = do[q0:q0 + n, head]
                dv[k0:k0 + m, head * hk // h] += prob.T @ g
                back = g @ vs.T
                back = prob * (back - (prob * back).sum(1, keepdim=True))
                if dtable is not None:
                    for c in range(table.shape[1]):
                        dtable[head, c] += torch.where(column == c, back, 0.0).sum()
                if case["cap"]:
                    back = back * (1.0 - (s / case["cap"]) ** 2)
                back = back / math.sqrt(d)
                dq[q0:q0 + n, head] = back @ ks
                dk[k0:k0 + m, head * hk // h] += back.T @ qs
        q0, k0 = q0 + n, k0 + m
    if not case["train"]:
        return out, lse
    return (out, lse, dq, dk, dv) + (() if dtable is None else (dtable,))


def _norm_exact(case: dict, seed: int):
    st = prepare(case, seed)
    names = ("stream", "y", "weight", "bias", "y_weight", "y_bias", "gate")
    d = {n: None if st[n] is None else st[n].double().requires_grad_(case["train"]) for n in names}

    def norm(x, weight, bias):
        if case["kind"] == "layer":
            x = x - x.mean(1, keepdim=True)
        x = x * (x.square().mean(1, keepdim=True) + EPS).rsqrt()
        x = x if weight is None else x * weight
        return x if bias is None else x + bias

    s = d["stream"]
    if case["after"]:
        n = norm(d["y"], d["y_weight"], d["y_bias"]) if case["after"] == "norm" else d["y"]
        s = s + case["scale"] * (n if d["gate"] is None else n * d["gate"])
    out = norm(s, d["weight"], d["bias"])
    first = (s.detach(), out.detach()) if case["after"] else (out.detach(),)
    if not case["train"]:
        return first
    wanted = [d[n] for n in names if d[n] is not None]
    grads = torch.autograd.grad([out, s], wanted, [st["dout"].double(), st["dnew"].double()])
    return first + tuple(grads)


def exact(case: dict, seed: int):
    return {"attention": _attention_exact, "norm": _norm_exact}[case["op"]](case, seed)
