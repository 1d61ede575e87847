"""Attention whose scores are capped, fall with the distance, get a learned bias by the distance's bucket, or see first keys from everywhere: forward,
backward and the table's gradient, against the definition in 64 bits.

Tolerances are those of plain scores (u = 2^-11): P and dS enter products rounded to fp16, |d out| <= 1.25 u A + u |out| and |d grad| <= 3 u B + u |grad|
+ 2^-25, with B from the magnitudes of the terms; the score's own fp32 operations (products summed, tanh within 2^-22 of the cap, a bias of up to 2^9
rounded at 2^-24) stay within the quarter of u that those grant.  lse: 2^-23 (dim + 8) S + 2^-20 (1 + |lse|) of the sums, 2^-22 cap of the tanh, 2^-22 of
the largest bias.  dS = dz (1 - tanh^2), where the tanh's slope is off by 2^-21 and less: B takes slope + 2^-11, of which 3 u is more.  The table's
gradient: dz is off by u sum |dO out| from delta's rounded out and by the quarter of u, so a column by 1.25 u times the sum of P (|dP| + |delta|), each
taken as magnitudes; and it is rounded once.
"""
import math

import numpy as np
import pytest
import torch

import paper_2302_05045_amd as samo
from gpu_util import DEV
from test_gpu_attention import seen_of

pytestmark = pytest.mark.gpu
U = 2.0 ** -11


def column_of(d, borders, two_sided):
    """The definition: the number of borders up to the distance, for keys behind the query in the table's second half."""
    borders = torch.zeros(0, device=DEV) if borders is None else borders
    n = d.abs() if two_sided else d.clamp(min=0)
    bucket = (n[..., None] >= borders.to(d.device)).sum(-1)
    return bucket + (borders.numel() + 1) * (d < 0) if two_sided else bucket


def reference(q, k, v, do, scale, seen, cap, slope, table, column, d):
    """One head of one sequence in 64 bits: results and the magnitudes of their bounds."""
    q, k, v, do = (t.double() for t in (q, k, v, do))
    x = q @ k.T * scale
    t = torch.tanh(x / cap) if cap else None
    z = cap * t if cap else x
    bias = torch.zeros_like(z)
    if slope is not None:
        bias = bias - slope.double() * d.abs()
    if table is not None:
        bias = bias + table.double()[column]
    z = torch.where(seen, z + bias, -math.inf)
    lse = torch.logsumexp(z, 1)
    p = torch.where(seen, torch.exp(z - torch.where(torch.isinf(lse), 0.0, lse)[:, None]), 0.0)
    out = p @ v
    dp = do @ v.T
    delta = (do * out).sum(1, keepdim=True)
    dz = p * (dp - delta)
    curve = 1.0 - t * t if cap else torch.ones_like(z)
    size = p * (do.abs() @ v.abs().T + (do * out).abs().sum(1, keepdim=True))
    small = 2.0 ** -25 / U * seen.double()
    ds, ssize = dz * curve, size * (curve + (2.0 ** -11 if cap else 0.0)) + small
    r = dict(out=out, lse=lse, dq=ds @ k * scale, dk=ds.T @ q * scale, dv=p.T @ do)
    b = dict(out=p @ v.abs() + small @ v.abs(), dq=ssize @ k.abs() * scale, dk=ssize.T @ q.abs() * scale, dv=(p + small).T @ do.abs())
    b["s"] = (q.abs() @ k.abs().T * scale).amax(1) if k.shape[0] else torch.zeros(q.shape[0], device=DEV)
    b["bias"] = torch.where(seen, bias.abs(), 0.0).amax(1) if k.shape[0] else b["s"]
    if table is not None:
        r["dtable"], b["dtable"] = (torch.zeros(table.numel(), dtype=torch.float64, device=DEV).index_add_(0, column.reshape(-1), w.reshape(-1)) for w in (dz, size))
    return r, b


def check(lens_q, lens_k, heads, kv_heads, dim, causal=True, window=0, cap=0.0, slopes=False, buckets=0, far=100, two_sided=None, first=None, seed=0,
          borders=None, std=1.0, slack=0, bias_std=1.0, **call):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    two_sided = not causal if two_sided is None else two_sided
    tq, tk = sum(lens_q), sum(lens_k)
    rnd = lambda *s, a=std: (torch.randn(s, generator=gen, device=DEV) * a).half()
    if lens_q == lens_k:
        qkv, dqkv = rnd(tq, heads + 2 * kv_heads, dim), torch.full((tq, heads + 2 * kv_heads, dim), float("nan"), device=DEV).half()
        (q, k, v), (dq, dk, dv) = (t.split([heads, kv_heads, kv_heads], dim=1) for t in (qkv, dqkv))
    else:
        q, k, v = rnd(tq, heads, dim), rnd(tk, kv_heads, dim), rnd(tk, kv_heads, dim)
        dq, dk, dv = (torch.full_like(t, float("nan")) for t in (q, k, v))
    out, lse, do = torch.full((tq, heads, dim), float("nan"), device=DEV).half(), torch.full((heads, tq), float("nan"), device=DEV), rnd(tq, heads, dim, a=1.0)
    table = dtable = None
    if buckets:
        table = rnd(heads, buckets * (2 if two_sided else 1), a=bias_std)
        dtable = torch.full_like(table, float("nan"))
        borders = samo.samo_bucket_borders(buckets, far) if borders is None else borders
    slope = torch.rand(heads, generator=gen, device=DEV) * 0.5 if slopes else None
    first_keys = None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV)
    scores = samo.Scores(cap=cap, slopes=slope, table=table, borders=borders, two_sided=two_sided, first_keys=first_keys)
    starts = lambda ns: torch.tensor(np.concatenate([[0], np.cumsum(ns)]), dtype=torch.int32, device=DEV)
    args = dict(causal=causal, window=window, scores=scores, **call)
    if len(lens_q) > 1:
        args.update(q_start=starts(lens_q), k_start=starts(lens_k), max_q=min(tq, max(lens_q) + slack))
    samo.samo_attention(q, k, v, out, lse, **args)
    if len(lens_q) > 1:
        args.update(max_k=min(tk, max(lens_k) + slack))
    samo.samo_attention_backward(do, q, k, v, out, lse, dq, dk, dv, dtable=dtable, **args)
    scale = dim ** -0.5
    q0 = k0 = 0
    tables = {}
    for s, (n, m) in enumerate(zip(lens_q, lens_k)):
        seen = seen_of(n, m, causal, window)
        d = torch.arange(n, device=DEV)[:, None] + (m - n) - torch.arange(m, device=DEV)[None, :]
        if first is not None:
            seen = seen | (torch.arange(m, device=DEV)[None, :] < first[s])
        column = column_of(d, borders, two_sided) if buckets else None
        grads = {}
        for h in range(heads):
            g = h * kv_heads // heads
            r, b = reference(q[q0:q0 + n, h], k[k0:k0 + m, g], v[k0:k0 + m, g], do[q0:q0 + n, h], scale, seen, cap, None if slope is None else slope[h],
                             None if table is None else table[h], column, d)
            got = dict(out=out[q0:q0 + n, h], dq=dq[q0:q0 + n, h])
            for name, most in (("out", 1.25), ("dq", 3.0)):
                off = (got[name].double() - r[name]).abs()
                bound = most * U * b[name] + U * r[name].abs() + 2.0 ** -25
                assert torch.all(off <= bound), (name, n, m, h, float((off - bound).max()), float((off / bound).max()))
            z, want = lse[h, q0:q0 + n].double(), r["lse"]
            empty = torch.isinf(want)
            assert torch.equal(torch.isneginf(z), empty)
            bound = 2.0 ** -23 * (dim + 8) * b["s"] + 2.0 ** -20 * (1 + want.abs()) + 2.0 ** -22 * (cap + b["bias"])
            assert torch.all((z - want).abs()[~empty] <= bound[~empty]), ("lse", n, m, h)
            assert torch.all(out[q0:q0 + n, h][empty] == 0) and torch.all(dq[q0:q0 + n, h][empty] == 0)
            for name in ("dk", "dv"):
                a, c = grads.get((name, g), (0, 0))
                grads[name, g] = (a + r[name], c + b[name])
            if buckets:
                a, c = tables.get(h, (0, 0))
                tables[h] = (a + r["dtable"], c + b["dtable"])
        for (name, g), (want, size) in grads.items():
            off = ((dk if name == "dk" else dv)[k0:k0 + m, g].double() - want).abs()
            bound = 3.0 * U * size + U * want.abs() + 2.0 ** -25
            assert torch.all(off <= bound), (name, n, m, g, float((off - bound).max()), float((off / bound).max()))
        q0, k0 = q0 + n, k0 + m
    for h, (want, size) in tables.items():
        off = (dtable[h].double() - want).abs()
        bound = 1.25 * U * size + U * want.abs() + 2.0 ** -25
        assert torch.all(off <= bound), ("dtable", h, float((off - bound).max()), off, bound)
        assert torch.all(dtable[h][size == 0] == 0)


FORMS = [dict(cap=5.0), dict(cap=50.0), dict(slopes=True), dict(buckets=32, far=128), dict(buckets=8, far=20, two_sided=True), dict(first=True),
         dict(cap=20.0, slopes=True, buckets=16, far=60, first=True), dict(cap=10.0, slopes=True), dict(cap=10.0, buckets=32, far=100),
         dict(slopes=True, buckets=32, far=128)]
NAMES = ["cap 5", "cap 50", "slopes", "buckets", "both sides", "first keys", "all", "cap and slopes", "cap and buckets", "slopes and buckets"]


def with_first(form, lens):
    """`first` in place of True: a share of each sequence's keys, none and all of them among the shares."""
    form = dict(form)
    if form.get("first"):
        form["first"] = [(0, n // 3, n, 65, 1, n // 2)[(i + 1) % 6] for i, n in enumerate(lens)]
    return form


@pytest.mark.parametrize("form", FORMS, ids=NAMES)
@pytest.mark.parametrize("dim", [16, 64, 80, 96, 128])
def test_every_form_and_size_of_head(form, dim):
    check([130, 67], [130, 67], 4, 2, dim, seed=dim, **with_first(form, [130, 67]))
    if not form.get("first"):
        check([97], [97], 2, 2, dim, causal=False, seed=dim + 1, **form)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 640])
def test_lengths_around_the_tiles(n):
    check([n], [n], 2, 1, 64, seed=n, cap=10.0, slopes=True, buckets=32, far=128)
    check([n], [n], 1, 1, 128, causal=False, seed=n, buckets=16, far=50)


@pytest.mark.parametrize("buckets,far", [(1, 0), (2, 2), (3, 9), (4, 3), (16, 9), (32, 17), (33, 200), (64, 5000), (64, 40)])
def test_numbers_of_buckets(buckets, far):
    """One bucket, one beside it, as many as there may be, borders that coincide, a last border behind every distance."""
    check([300, 41], [300, 41], 2, 2, 64, buckets=buckets, far=far, seed=buckets)
    check([300, 41], [300, 41], 2, 2, 32, causal=False, buckets=buckets, far=far, seed=buckets)


def test_borders_of_any_kind():
    """A border at 0 leaves the first bucket empty; borders far apart and behind every distance; distances past any of a tile's."""
    make = lambda *b: torch.tensor(b, dtype=torch.int32, device=DEV)
    check([500], [500], 1, 1, 64, buckets=4, borders=make(0, 100, 101))
    check([500], [500], 1, 1, 64, causal=False, buckets=4, borders=make(31, 64, 2 ** 31 - 1))
    check([500], [500], 1, 1, 64, causal=False, two_sided=False, buckets=3, borders=make(1, 256))


@pytest.mark.parametrize("window", [1, 33, 64, 100, 5000])
def test_windows_and_first_keys(window):
    check([300, 20, 200], [300, 20, 200], 2, 1, 96, window=window, first=[70, 20, 0], seed=window)
    check([300, 20], [450, 90], 2, 1, 64, window=window, first=[1, 64], seed=window, cap=8.0, slopes=True, buckets=12, far=90)


def test_first_keys_out_of_range():
    """Fewer than none count as none, more than a sequence has as all of them."""
    check([150, 150], [150, 150], 2, 2, 64, first=[-5, 1 << 30])


@pytest.mark.parametrize("form", FORMS, ids=NAMES)
def test_fewer_and_more_queries_than_keys(form):
    for lens_q, lens_k, dim in (([70, 200], [333, 201], 128), ([333, 130], [70, 1], 64)):
        check(lens_q, lens_k, 4, 2, dim, **with_first(form, lens_k))
        if not form.get("first"):
            check(lens_q, lens_k, 4, 2, dim, causal=False, **form)


@pytest.mark.parametrize("form", FORMS, ids=NAMES)
def test_sequences_of_no_and_one_token_among_others(form):
    lens = [0, 1, 200, 0, 3, 64, 1, 0]
    check(lens, lens, 4, 4, 64, slack=77, **with_first(form, lens))
    if not form.get("first"):
        check([0, 5, 0], [7, 0, 0], 2, 1, 64, causal=False, **form)


@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 1), (6, 3), (25, 25)])
def test_shared_heads(heads, kv):
    check([150, 40], [150, 40], heads, kv, 64, cap=10.0, slopes=True, buckets=32, far=128)


@pytest.fixture
def parts(request):
    samo.samo_debug_set(samo.KNOB_ATTENTION_SPLIT, request.param)
    yield request.param
    samo.samo_debug_set(samo.KNOB_ATTENTION_SPLIT)


@pytest.mark.parametrize("parts", [1, 2, 3, 7, 16], indirect=True)
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_keys_and_queries_in_parts(parts, dim):
    form = dict(cap=10.0, slopes=True, buckets=32, far=128)
    check([0, 1, 130, 300, 64], [7, 400, 131, 290, 0], 4, 2, dim, seed=dim, slack=60, first=[3, 100, 0, 290, 0], **form)
    check([200, 70], [90, 515], 3, 1, dim, causal=False, seed=dim + 1, **form)
    check([450, 20], [450, 20], 2, 2, dim, window=70, seed=dim + 2, first=[130, 1], **form)


@pytest.mark.parametrize("context", [1, 63, 1000, 9001])
def test_one_token_behind_a_context(context):
    lens = [context, 5, max(1, context // 2)]
    check([1, 1, 1], lens, 8, 2, 64, seed=context, cap=30.0, buckets=32, far=128)
    check([1], [context], 4, 4, 128, window=300, seed=context, slopes=True, first=[4])


@pytest.mark.parametrize("dim", [24, 64, 80])
def test_many_workgroups(dim):
    """Enough workgroups for the form in which a wave has its keys for itself."""
    lens = [130, 0, 1, 64, 257, 200, 128, 65]
    check(lens, [n + 3 * i for i, n in enumerate(lens)], 16, 16, dim, slack=700 if dim > 64 else 230, seed=dim, cap=10.0, slopes=True, buckets=32, far=128)


def test_scores_at_their_cap():
    """Products many times the cap either way: the tanh is 1, its slope next to nothing; one key takes all of a row, or many share it."""
    check([200], [200], 2, 2, 64, cap=2.0, std=4.0)
    check([200], [200], 2, 2, 128, cap=200.0, std=8.0)
    check([200], [200], 2, 2, 64, cap=2.0 ** -10)
    check([200], [200], 2, 2, 64, cap=256.0)


def test_large_biases():
    """Biases that hide whole buckets, the lowest numbers of the type among them."""
    check([300], [300], 2, 2, 64, buckets=32, far=128, bias_std=12.0)
    check([300, 2], [300, 2], 2, 2, 64, buckets=8, far=64, causal=False, bias_std=0.0, seed=3)
    q, k, v = (torch.randn(200, 2, 64, device=DEV).half() for _ in range(3))
    table = torch.full((2, 4), -65504.0, device=DEV).half()
    table[:, 0] = 0.0                                        # distances below 10 alone count: a window
    borders = torch.tensor([10, 50, 100], dtype=torch.int32, device=DEV)
    a, b, la, lb = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(2, 200, device=DEV), torch.zeros(2, 200, device=DEV)
    samo.samo_attention(q, k, v, a, la, scores=samo.Scores(table=table, borders=borders))
    samo.samo_attention(q, k, v, b, lb, window=10)
    assert float((a.float() - b.float()).abs().max()) <= 4.5 * U * float(v.float().abs().max()) and float((la - lb).abs().max()) < 1e-4


def test_without_any_form_it_is_the_plain_attention():
    q, k, v, do = (torch.randn(300, 2, 80, device=DEV).half() for _ in range(4))
    res = []
    for scores in (None, samo.Scores(), samo.Scores(cap=256.0), samo.Scores(slopes=torch.zeros(2, device=DEV))):
        o, dq, dk, dv, lse = *(torch.zeros_like(q) for _ in range(4)), torch.zeros(2, 300, device=DEV)
        samo.samo_attention(q, k, v, o, lse, scores=scores)
        samo.samo_attention_backward(do, q, k, v, o, lse, dq, dk, dv, scores=scores)
        res.append((o, dq, dk, dv, lse))
    for other in res[1:]:
        for a, b in zip(res[0], other):
            assert float((a.double() - b.double()).norm() / a.double().norm()) < 1e-3


def test_the_table_of_a_bias_that_is_not_trained():
    """dtable None: the other gradients are the same bits."""
    q, k, v, do = (torch.randn(300, 2, 64, device=DEV).half() for _ in range(4))
    table = torch.randn(2, 32, device=DEV).half()
    scores = samo.Scores(table=table, borders=samo.samo_bucket_borders(32, 128))
    o, lse = torch.zeros_like(q), torch.zeros(2, 300, device=DEV)
    samo.samo_attention(q, k, v, o, lse, scores=scores)
    res = []
    for dtable in (None, torch.zeros_like(table)):
        grads = [torch.zeros_like(q) for _ in range(3)]
        samo.samo_attention_backward(do, q, k, v, o, lse, *grads, scores=scores, dtable=dtable)
        res.append(grads)
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_table_gradient_against_differences():
    """The loss sum(out * do) along a random direction of the table, in steps that fp16 holds exactly, against its gradient; out's roundings add up as
    a random sum, 6 of whose deviations are granted, and the differences' own error is of third order in the step."""
    n, dim, eps = 150, 64, 2.0 ** -4
    gen = torch.Generator(device=DEV)
    gen.manual_seed(4)
    q, k, v, do = (torch.randn((n, 2, dim), generator=gen, device=DEV).half() for _ in range(4))
    table = (torch.randn((2, 64), generator=gen, device=DEV) * 16).round().div(16).half()
    borders = samo.samo_bucket_borders(32, 100)
    way = torch.randint(0, 2, table.shape, generator=gen, device=DEV).half() * 2 - 1
    out, lse, dtable = torch.zeros_like(q), torch.zeros(2, n, device=DEV), torch.zeros_like(table)
    form = lambda t: samo.Scores(cap=20.0, table=t, borders=borders, two_sided=True)
    samo.samo_attention(q, k, v, out, lse, causal=False, scores=form(table))
    samo.samo_attention_backward(do, q, k, v, out, lse, *(torch.zeros_like(q) for _ in range(3)), causal=False, scores=form(table), dtable=dtable)
    loss = []
    for sign in (1, -1):
        o = torch.zeros_like(q)
        samo.samo_attention(q, k, v, o, lse, causal=False, scores=form(table + sign * eps * way))
        loss.append(float((o.double() * do.double()).sum()))
    slope = (loss[0] - loss[1]) / (2 * eps)
    want = float((dtable.double() * way.double()).sum())
    noise = 6 * U * math.sqrt(float((out.double() * do.double()).square().sum()) * 2) / (2 * eps)
    assert abs(slope - want) <= noise + 0.05 * float(dtable.double().norm()), (slope, want)


def test_same_bits_again_other_stream_and_graph():
    n, dim = 500, 80
    q, k, v, do = (torch.randn(n, 4, dim, device=DEV).half() for _ in range(4))
    table = torch.randn(4, 32, device=DEV).half()
    scores = samo.Scores(cap=20.0, table=table, borders=samo.samo_bucket_borders(32, 128), first_keys=torch.tensor([99], dtype=torch.int32, device=DEV))
    bufs = lambda: [torch.zeros(n, 4, dim, device=DEV).half() for _ in range(4)] + [torch.zeros(4, n, device=DEV), torch.zeros_like(table)]

    def call(o, dq, dk, dv, lse, dtable):
        samo.samo_attention(q, k, v, o, lse, scores=scores)
        samo.samo_attention_backward(do, q, k, v, o, lse, dq, dk, dv, scores=scores, dtable=dtable)

    first, second, third = bufs(), bufs(), bufs()
    call(*first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(*second)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*third)
    for _ in range(3):
        for t in third:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(first, second, third):
            assert torch.equal(a, b) and torch.equal(a, c)
        call(*bufs())


def test_workspaces_of_the_callers_own():
    """The least workspace, and one with room for the sums of parts; one byte less is refused."""
    import ctypes
    q, k, v, do = (torch.randn(2000, 2, 64, device=DEV).half() for _ in range(4))
    table = torch.randn(2, 32, device=DEV).half()
    scores = samo.Scores(table=table, borders=samo.samo_bucket_borders(32, 128))
    o, lse = torch.zeros_like(q), torch.zeros(2, 2000, device=DEV)
    samo.samo_attention(q, k, v, o, lse, scores=scores)
    grads, dtable = [torch.zeros_like(q) for _ in range(3)], torch.zeros_like(table)
    d = samo._attention_desc(q, k, v, o, lse, None, True, 0, None, None, None, None)
    for name, t in zip(("dout", "dq", "dk", "dv"), [do] + grads):
        samo._set_heads(d, name, t)
    c, need = samo._scores_desc(scores, d, dtable), ctypes.c_size_t()
    assert samo.lib().samo_attention_scored_workspace_bytes(ctypes.byref(d), ctypes.byref(c), ctypes.byref(need)) == 0
    assert need.value > 4 * 2 * 2000
    res = []
    for room in (None, need.value, need.value + (32 << 20)):
        ws = None if room is None else torch.full((room,), 255, dtype=torch.uint8, device=DEV)
        dtable.fill_(float("nan"))
        samo.samo_attention_backward(do, q, k, v, o, lse, *grads, scores=scores, dtable=dtable, workspace=ws)
        res.append([t.clone() for t in grads + [dtable]])
    for other in res[1:]:
        for a, b in zip(res[0], other):
            assert float((a.double() - b.double()).norm() / a.double().norm()) < 2e-3
    with pytest.raises(samo.SamoError):
        samo.samo_attention_backward(do, q, k, v, o, lse, *grads, scores=scores, dtable=dtable, workspace=torch.empty(need.value - 1, dtype=torch.uint8, device=DEV))


def test_what_is_not_finite_in_places_that_are_masked():
    """Keys and values behind the diagonal, in blocks that no query of a block sees, change nothing, with the first keys seen from everywhere."""
    n, dim = 320, 64
    q, k, v, do = (torch.randn(n, 1, dim, device=DEV).half() for _ in range(4))
    table = torch.randn(1, 32, device=DEV).half()
    scores = samo.Scores(cap=20.0, table=table, borders=samo.samo_bucket_borders(32, 128), first_keys=torch.tensor([40], dtype=torch.int32, device=DEV))
    run = lambda k, v: (lambda o, lse: (samo.samo_attention(q, k, v, o, lse, scores=scores), o, lse)[1:])(torch.zeros_like(q), torch.zeros(1, n, device=DEV))
    clean = run(k, v)
    k2, v2 = k.clone(), v.clone()
    k2[256:], v2[256:] = float("nan"), float("inf")
    got = run(k2, v2)
    assert torch.equal(got[0][:256], clean[0][:256]) and torch.equal(got[1][:, :256], clean[1][:, :256])
    assert torch.isnan(got[0][256:]).all()


def test_refusals_of_the_binding():
    q = torch.zeros(6, 2, 16, device=DEV).half()
    lse, out = torch.zeros(2, 6, device=DEV), torch.full_like(q, 7.0)
    table, borders = torch.zeros(2, 4, device=DEV).half(), torch.tensor([1, 2, 3], dtype=torch.int32, device=DEV)
    first = torch.ones(1, dtype=torch.int32, device=DEV)
    for scores, what in ((samo.Scores(slopes=torch.zeros(1, device=DEV)), ValueError), (samo.Scores(slopes=torch.zeros(2, device=DEV).half()), TypeError),
                         (samo.Scores(table=table), ValueError), (samo.Scores(borders=borders), ValueError), (samo.Scores(table=table, borders=borders[:2]), ValueError),
                         (samo.Scores(table=table[:1], borders=borders), ValueError), (samo.Scores(table=table.float(), borders=borders), TypeError),
                         (samo.Scores(table=table[:, :3], borders=borders[:2], two_sided=True), TypeError),
                         (samo.Scores(table=table, borders=borders, two_sided=True), ValueError), (samo.Scores(table=table, borders=borders.cpu()), TypeError),
                         (samo.Scores(first_keys=first.long()), TypeError), (samo.Scores(cap=-1.0), samo.SamoError), (samo.Scores(cap=257.0), samo.SamoError),
                         (samo.Scores(cap=float("nan")), samo.SamoError)):
        with pytest.raises(what):
            samo.samo_attention(q, q, q, out, lse, scores=scores)
    with pytest.raises(samo.SamoError):
        samo.samo_attention(q, q, q, out, lse, causal=False, scores=samo.Scores(first_keys=first))
    starts = torch.tensor([0, 2, 6], dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        samo.samo_attention(q, q, q, out, lse, q_start=starts, k_start=starts, scores=samo.Scores(first_keys=first))
    g = [torch.full_like(q, 7.0) for _ in range(3)]
    with pytest.raises(ValueError):
        samo.samo_attention_backward(q, q, q, q, q, lse, *g, dtable=table)
    with pytest.raises(ValueError):
        samo.samo_attention_backward(q, q, q, q, q, lse, *g, scores=samo.Scores(), dtable=table)
    with pytest.raises(ValueError):
        samo.samo_attention_backward(q, q, q, q, q, lse, *g, scores=samo.Scores(table=table, borders=borders), dtable=table[:, :2].contiguous())
    assert torch.all(out == 7.0) and all(torch.all(t == 7.0) for t in g)


def test_borders_of_the_logarithm():
    for buckets, far in ((32, 128), (16, 128), (8, 80), (64, 2000), (2, 5), (3, 9)):
        borders = samo.samo_bucket_borders(buckets, far, device="cpu")
        half, n = buckets // 2, torch.arange(4000)
        log = half + torch.floor(torch.log(n.clamp(min=1).double() / half) / math.log(far / half) * (buckets - half) + 1e-9).long()
        want = torch.where(n < half, n, log.clamp(max=buckets - 1))
        assert torch.equal((n[:, None] >= borders).sum(1), want), (buckets, far)


@pytest.mark.parametrize("form", [dict(cap=20.0), dict(slopes=True), dict(first=True), dict(cap=10.0, slopes=True, first=True)],
                         ids=["cap", "slopes", "first keys", "cap, slopes and first keys"])
@pytest.mark.parametrize("heads,kv,queries", [(8, 2, 1), (32, 8, 1), (7, 1, 3), (12, 4, 20), (6, 2, 42), (6, 2, 43), (128, 1, 1), (64, 1, 2), (100, 1, 1)])
def test_heads_that_share_a_tile_with_their_queries(heads, kv, queries, form):
    """A tile's rows are all heads of a query where a sequence's are at most 128: with one query, several, as many as fit and one more."""
    lens_q, lens_k = [queries, 1, 0, max(1, queries - 1)], [queries + 300, 77, 40, queries]
    check(lens_q, lens_k, heads, kv, 64, seed=heads, **with_first(form, lens_k))
    check([queries], [queries + 1000], heads, kv, 128, window=150, seed=heads + 1, **with_first(form, [queries + 1000]))
    if not form.get("first"):
        check(lens_q, lens_k, heads, kv, 80, causal=False, seed=heads + 2, **form)


@pytest.mark.parametrize("parts", [1, 2, 5, 16], indirect=True)
def test_heads_that_share_a_tile_in_parts(parts):
    check([3, 1], [700, 90], 8, 2, 64, cap=20.0, first=[70, 0], seed=parts)
    check([3, 1], [700, 90], 12, 3, 128, slopes=True, seed=parts)
    check([2], [900], 4, 1, 96, causal=False, slopes=True, seed=parts)


@pytest.mark.parametrize("form", FORMS, ids=NAMES)
@pytest.mark.parametrize("dim", [16, 64, 80, 96, 128])
def test_few_queries_of_every_form(form, dim):
    """At most 32 rows: the four waves share the keys.  No key, one, tiles for one wave, all of them, one more; 1, 31, 32 and 33 queries of one head."""
    lens_k = [0, 1, 63, 64, 65, 256, 257, 300, 900]
    lens_q = [1, 1, 3, 1, 2, 1, 1, 0, 2]
    check(lens_q, lens_k, 4, 2, dim, seed=dim, **with_first(form, lens_k))
    for n in (31, 32, 33):
        check([n, 5], [n + 170, 700], 2, 2, dim, seed=n, **with_first(form, [n + 170, 700]))
    if not form.get("first"):
        check(lens_q, lens_k, 4, 4, dim, causal=False, seed=dim, **form)


@pytest.mark.parametrize("parts", [1, 2, 3, 9, 16], indirect=True)
def test_few_queries_in_parts(parts):
    form = dict(cap=10.0, slopes=True, buckets=32, far=128)
    check([1, 2, 0, 3], [900, 70, 30, 1], 4, 2, 64, seed=parts, first=[3, 70, 0, 1], **form)
    check([1, 4], [1500, 90], 2, 1, 128, window=200, first=[130, 0], seed=parts)
    check([2], [515], 8, 1, 80, causal=False, buckets=16, far=100, seed=parts)


def test_no_queries_and_no_keys():
    """No query at all: the table's gradient is zero; no key: out is zero, the gradients of nothing are not written."""
    table, borders = torch.randn(2, 8, device=DEV).half(), samo.samo_bucket_borders(8, 20)
    scores = samo.Scores(cap=5.0, table=table, borders=borders)
    for nq, nk in ((0, 5), (5, 0), (0, 0)):
        t = lambda n: torch.randn(n, 2, 64, device=DEV).half()
        q, k, v, do = t(nq), t(nk), t(nk), t(nq)
        out, lse, dtable = torch.full_like(q, 7.0), torch.zeros(2, nq, device=DEV), torch.full_like(table, float("nan"))
        dq, dk, dv = torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(v, 7.0)
        samo.samo_attention(q, k, v, out, lse, causal=False, scores=scores._replace(table=torch.cat([table, table], 1), two_sided=True))
        samo.samo_attention(q, k, v, out, lse, scores=scores)
        samo.samo_attention_backward(do, q, k, v, out, lse, dq, dk, dv, scores=scores, dtable=dtable)
        assert torch.all(dtable == 0) and torch.all(out == 0) and torch.all(dq == 0) and torch.all(dk == 0) and torch.all(dv == 0)


def test_two_calls_at_once_on_two_streams():
    """Calls with workspaces from the allocator, each on its own stream: the bits of each by itself."""
    make = lambda n: [torch.randn(n, 2, 64, device=DEV).half() for _ in range(4)]
    table, borders = torch.randn(2, 32, device=DEV).half(), samo.samo_bucket_borders(32, 128)
    scores = samo.Scores(table=table, borders=borders)

    def call(q, k, v, do):
        out, lse, grads, dtable = torch.zeros_like(q), torch.zeros(2, q.shape[0], device=DEV), [torch.zeros_like(q) for _ in range(3)], torch.zeros_like(table)
        samo.samo_attention(q, k, v, out, lse, scores=scores)
        samo.samo_attention_backward(do, q, k, v, out, lse, *grads, scores=scores, dtable=dtable)
        return [out, lse, *grads, dtable]

    data = [make(1500), make(1100)]
    want = [call(*d) for d in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in data]
    got = []
    for s, d in zip(streams, data):
        with torch.cuda.stream(s):
            got.append(call(*d))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for w, g in zip(want, got) for a, b in zip(w, g))


def test_rows_past_two_gibibytes():
    """Keys and values whose rows lie so far apart that the last ones begin past 2^31 bytes, read by a token and by many."""
    n, dim, apart = 700, 64, 1 << 21
    room = torch.zeros((n, apart), dtype=torch.float16, device=DEV)
    k, v = room[:, :dim].unsqueeze(1), room[:, 64:64 + dim].unsqueeze(1)
    kk, vv = (torch.randn(n, 1, dim, device=DEV).half() for _ in range(2))
    k.copy_(kk)
    v.copy_(vv)
    for form in (dict(cap=20.0), dict(slopes=torch.rand(4, device=DEV)), dict(first_keys=torch.tensor([3], dtype=torch.int32, device=DEV))):
        for queries in (1, 200):
            q = torch.randn(queries, 4, dim, device=DEV).half()
            a, b, lse = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(4, queries, device=DEV)
            samo.samo_attention(q, k, v, a, lse, scores=samo.Scores(**form))
            samo.samo_attention(q, kk, vv, b, lse, scores=samo.Scores(**form))
            assert torch.equal(a, b)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [1, 33, 130, 200])
def test_biases_above_the_range_of_the_exponent(n, dim):
    """exp(300) is no fp32 number: every score has its bias taken off with the row's largest, also beside the last row of a sequence, where lanes have no row
    whose largest to take.  A bias that all keys have is none."""
    q, k, v, do = (torch.randn(n, 2, dim, device=DEV).half() for _ in range(4))
    borders = samo.samo_bucket_borders(8, 40)
    res = []
    for value in (0.0, 300.0, -300.0):
        scores = samo.Scores(table=torch.full((2, 8), value, device=DEV).half(), borders=borders)
        out, lse, dtable, grads = torch.zeros_like(q), torch.zeros(2, n, device=DEV), torch.zeros(2, 8, device=DEV).half(), [torch.zeros_like(q) for _ in range(3)]
        samo.samo_attention(q, k, v, out, lse, scores=scores)
        samo.samo_attention_backward(do, q, k, v, out, lse, *grads, scores=scores, dtable=dtable)
        res.append([out, *grads, dtable])
        assert float((lse - value).abs().max()) < 20.0
    # fp32 holds a score beside 300 to 2^-16: P, and what is formed from it, within 2^-14 of its own
    for other in res[1:]:
        for a, b in zip(res[0], other):
            assert torch.isfinite(b).all()
            assert float((a.double() - b.double()).norm()) <= 2.0 ** -10 * float(a.double().norm()) + 1e-3


@pytest.mark.parametrize("scale, cap", [(2.0 ** 20, 1.0), (2.0 ** 60, 2.0 ** -10), (2.0 ** -20, 1.0), (2.0 ** -60, 256.0)])
def test_scales_far_from_the_cap(scale, cap):
    """Powers of scale / cap that are no fp32 numbers: a product of zero has a score of zero, one of 1 or more the cap where scale / cap is 2^20 or more, and
    almost none where it is 2^-20 or less."""
    n, dim = 70, 64
    q, k, v, do = (torch.randn(n, 2, dim, device=DEV).half() for _ in range(4))
    q[:, 0], k[:, 1] = 0, 1
    q[:, 1] = torch.randn(n, device=DEV).sign()[:, None].half()
    out, lse, grads = torch.zeros_like(q), torch.zeros(2, n, device=DEV), [torch.zeros_like(q) for _ in range(3)]
    scores = samo.Scores(cap=cap)
    samo.samo_attention(q, k, v, out, lse, causal=True, scale=scale, scores=scores)
    samo.samo_attention_backward(do, q, k, v, out, lse, *grads, causal=True, scale=scale, scores=scores)
    # every score of a row is the same: values' means, and the logarithm of their number beside the score
    counts = torch.arange(1, n + 1, device=DEV).double()
    means = v.double().cumsum(0) / counts[:, None, None]
    score = torch.zeros(2, n, device=DEV).double()
    score[1] = q[:, 1, 0].double() * (cap if scale / cap > 1 else 64 * scale)
    # P to fp16, weights below 1, and out to fp16: 2^-11 each of numbers up to the largest value
    assert float((out.double() - means).abs().max()) <= 2.0 ** -9 * float(v.abs().max())
    assert float((lse.double() - counts.log() - score).abs().max()) <= 2.0 ** -14 * 2
    # dq is scale sum dS k: of q = 0, where the tanh's slope is 1, sums of about 1 times 2^20 pass fp16's 2^16 and are its infinities
    for g in grads:
        assert not torch.isnan(g).any() and (scale > 1 or torch.isfinite(g).all())


def check_slopes(dim, lens_q, lens_k, kv, slopes):
    """The tolerances of check(); the exponents' offs are those of the keys that count: 2^-20 sum P |bias|."""
    heads = len(slopes)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(dim)
    rnd = lambda n, h: torch.randn((n, h, dim), generator=gen, device=DEV).half()
    tq, tk = sum(lens_q), sum(lens_k)
    q, k, v, do = rnd(tq, heads), rnd(tk, kv), rnd(tk, kv), rnd(tq, heads)
    out, lse, dq, dk, dv = torch.zeros_like(q), torch.zeros(heads, tq, device=DEV), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    slope = torch.tensor(slopes, device=DEV)
    starts = lambda ns: torch.tensor(np.concatenate([[0], np.cumsum(ns)]), dtype=torch.int32, device=DEV)
    args = dict(q_start=starts(lens_q), k_start=starts(lens_k), max_q=max(lens_q), max_k=max(lens_k), scores=samo.Scores(slopes=slope))
    samo.samo_attention(q, k, v, out, lse, **args)
    samo.samo_attention_backward(do, q, k, v, out, lse, dq, dk, dv, **args)
    q0 = k0 = 0
    for n, m in zip(lens_q, lens_k):
        seen = seen_of(n, m, True, 0)
        d = torch.arange(n, device=DEV)[:, None] + (m - n) - torch.arange(m, device=DEV)[None, :]
        grads = {}
        for h in range(heads):
            g = h * kv // heads
            a = [q[q0:q0 + n, h], k[k0:k0 + m, g], v[k0:k0 + m, g], do[q0:q0 + n, h]]
            r, b = reference(*a, dim ** -0.5, seen, 0.0, slope[h], None, None, d)
            z = torch.where(seen, a[0].double() @ a[1].double().T * dim ** -0.5 - slope[h].double() * d.abs(), -math.inf)
            off = (torch.softmax(z, 1) * (slope[h].double() * d).abs()).sum(1) * 2.0 ** -20
            bound = 2.0 ** -23 * (dim + 8) * b["s"] + 2.0 ** -20 * (1 + r["lse"].abs()) + off
            err = (lse[h, q0:q0 + n].double() - r["lse"]).abs()
            assert torch.all(err <= bound), ("lse", slopes[h], n, m, float(err.max()), float((err / bound).max()))
            for name, got, most in (("out", out, 1.25), ("dq", dq, 3.0)):
                err = (got[q0:q0 + n, h].double() - r[name]).abs()
                assert torch.all(err <= most * U * b[name] + U * r[name].abs() + 2.0 ** -25), (name, slopes[h], n, m)
            for name in ("dk", "dv"):
                x, c = grads.get((name, g), (0, 0))
                grads[name, g] = (x + r[name], c + b[name])
        for (name, g), (want, size) in grads.items():
            err = ((dk if name == "dk" else dv)[k0:k0 + m, g].double() - want).abs()
            assert torch.all(err <= 3.0 * U * size + U * want.abs() + 2.0 ** -25), (name, n, m, g)
        q0, k0 = q0 + n, k0 + m


SLOPED = [(64, [300, 1, 70], [300, 1, 70], 6), (128, [130], [200], 2), (80, [1, 2], [300, 70], 2), (64, [40], [400], 6),
          (64, [1, 1], [64, 640], 6), (64, [1, 2], [640, 65], 2), (128, [70, 33], [133, 64], 2), (96, [100], [131], 6)]       # a block's corner on the diagonal


@pytest.mark.parametrize("dim, lens_q, lens_k, kv", SLOPED)
def test_steep_slopes(dim, lens_q, lens_k, kv):
    """A slope's bias is within 2^-20 of itself at every distance, so that next to a query it stays what it is however steep the slope."""
    check_slopes(dim, lens_q, lens_k, kv, [0.35, -0.01, 30.3, 700.1, 5000.7, 20000.3])


@pytest.mark.parametrize("dim, lens_q, lens_k, kv", SLOPED)
def test_scores_that_slopes_take_far_from_zero(dim, lens_q, lens_k, kv):
    """Scores of 2^28 to 2^38 at the first keys of a row, which are met first: their rounded products are no exponents, and none of it stays."""
    check_slopes(dim, lens_q, lens_k, kv, [0.35, 7e5 + 0.3, 1.1e7, 1.0e8, 2.0 ** 30, 1.0e9])


@pytest.mark.parametrize("cap, buckets", [(0.0, 0), (20.0, 0), (20.0, 8)])
@pytest.mark.parametrize("queries", [1, 40])
def test_far_keys_alone(queries, cap, buckets):
    """Slopes that grow with the distance (or fall) so that a row's largest score is far from zero: lse within 2^-18 of itself, out that of the one key that
    is left, nothing that is not finite."""
    heads, dim, n = 4, 64, 700
    q, k, v = (torch.randn(m, heads, dim, device=DEV).half() for m in (queries, n, n))
    slope = torch.tensor([-2.0 ** 10, -2.0 ** 20, -2.0 ** 24, -2.0 ** 30], device=DEV)
    table = torch.randn(heads, buckets, device=DEV).half() if buckets else None
    scores = samo.Scores(cap=cap, slopes=slope, table=table, borders=samo.samo_bucket_borders(buckets, 40) if buckets else None)
    out, lse = torch.zeros_like(q), torch.zeros(heads, queries, device=DEV)
    samo.samo_attention(q, k, v, out, lse, scores=scores)
    want = -slope.double()[:, None] * (torch.arange(queries, device=DEV) + n - queries)[None, :]       # the first key, score and table aside
    assert torch.all((lse.double() - want).abs() <= 2.0 ** -18 * want.abs() + 64.0)
    assert float((out.double() - v[0].double()).abs().max()) <= 2.0 ** -10 * float(v[0].abs().max())


@pytest.mark.parametrize("cap", [2.0 ** -10, 1.0, 30.0, 256.0])
@pytest.mark.parametrize("into", [1.0, 2.0 ** -7, 2.0 ** 9])
def test_the_tanh(cap, into):
    """Of one key lse is its score, cap tanh(x / cap); x is exact, a single product.  Up to half the cap the tanh is within 2^-20 of itself: a polynomial
    off by 5.5e-7, its coefficients (scaled by powers of two here) and four operations by 2^-25 and 2^-24 each, the largest of them once.  Above it is
    within 2^-22.  The score goes into units of log 2 and back by four roundings, 2^-22 of itself."""
    n, dim = 8192, 16
    t = torch.cat([0.5 * 2.0 ** (-12 * torch.rand(n // 2, device=DEV)), 0.5 + 11.5 * torch.rand(n // 2, device=DEV)])
    q, k, v = (torch.zeros(n, 1, dim, device=DEV).half() for _ in range(3))
    q[:, 0, 3], k[:, 0, 3] = (t * 8).half() * (2 * torch.randint(0, 2, (n,), device=DEV) - 1), 0.125 / into
    starts = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    out, lse = torch.zeros_like(q), torch.zeros(1, n, device=DEV)
    samo.samo_attention(q, k, v, out, lse, scale=cap * into, q_start=starts, k_start=starts, max_q=1, max_k=1, scores=samo.Scores(cap=cap))
    x = q[:, 0, 3].double() / 8
    want = cap * torch.tanh(x)
    bound = 2.0 ** -22 * want.abs() + torch.where(x.abs() <= 0.5, 2.0 ** -20 * want.abs(), 2.0 ** -22 * cap)
    off = (lse[0].double() - want).abs()
    assert torch.all(off <= bound), float((off / bound).max())
    assert float(off.max()) <= 2.0 ** -21 * cap               # a score within 2^-13 at the largest cap
