"""Attention, forward and backward, against the definition in 64 bits.

Tolerances.  The tensors are fp16 (u = 2^-11 relative, rounding to nearest), the sums fp32 in some order.  P enters the second product
rounded to fp16, so a row of out is off by at most u sum_j P_j |v_j| + u |out| and the fp32 sums' share, for which a quarter of u is
granted: |d out| <= 1.25 u A + u |out| with A = sum_j P_j |v_j|.  lse: the scores are exact products summed in fp32: 2^-23 (dim + 8) S with
S the largest sum of magnitudes of a score, and a few operations at the end, 2^-20.  Gradients: P and dS are rounded to fp16, dP - delta is off by what
out's rounding to fp16 makes of delta (u sum_d |dO out|) and the fp32 sums; each bound is that of the products' terms taken as magnitudes, with
P (|dP| + |delta| + u-terms) in the place of |dS|: |d| <= 3 u B + u |result| + 2^-24 (the smallest fp16 step, for each of dS's roundings among
the subnormal numbers: times the sum of the other factor's magnitudes).  Every bound is element by element.
"""
import math

import numpy as np
import pytest
import torch

import paper_2302_05045_amd as samo
from gpu_util import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -11


def seen_of(n, m, causal, window):
    i = torch.arange(n, device=DEV)[:, None] + (m - n)
    j = torch.arange(m, device=DEV)[None, :]
    seen = torch.ones((n, m), dtype=torch.bool, device=DEV)
    if causal:
        seen = j <= i
        if window:
            seen &= j > i - window
    return seen


def reference(q, k, v, do, scale, seen):
    """One head of one sequence in 64 bits: results and the magnitudes of their bounds."""
    q, k, v, do = (t.double() for t in (q, k, v, do))
    s = torch.where(seen, q @ k.T * scale, -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.where(seen, torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)[:, None]), 0.0)
    out = p @ v
    dp = do @ v.T
    delta = (do * out).sum(1, keepdim=True)
    ds = p * (dp - delta)
    size = p * (do.abs() @ v.abs().T + (do * out).abs().sum(1, keepdim=True)) + 2.0 ** -25 / U * seen
    r = dict(out=out, lse=lse, dq=ds @ k * scale, dk=ds.T @ q * scale, dv=p.T @ do)
    b = dict(out=p @ v.abs() + 2.0 ** -25 / U * (seen.double() @ v.abs()), dq=size @ k.abs() * scale, dk=size.T @ q.abs() * scale,
             dv=(p + 2.0 ** -25 / U * seen).T @ do.abs(), s=(q.abs() @ k.abs().T * scale).amax(1) if k.shape[0] else torch.zeros(q.shape[0], device=DEV))
    return r, b


def check(lens_q, lens_k, heads, kv_heads, dim, causal, window, seed=0, layout="packed", std=1.0, dstd=1.0, slack=0, fix=None, scale=None):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    tq, tk = sum(lens_q), sum(lens_k)
    rnd = lambda *s, a=std: (torch.randn(s, generator=gen, device=DEV) * a).half()
    if layout == "packed" and lens_q == lens_k:
        qkv, dqkv = rnd(tq, (heads + 2 * kv_heads) * dim), torch.full((tq, (heads + 2 * kv_heads) * dim), float("nan"), device=DEV).half()
        cut = lambda t: (t[:, :heads * dim].view(tq, heads, dim), t[:, heads * dim:(heads + kv_heads) * dim].view(tq, kv_heads, dim),
                         t[:, (heads + kv_heads) * dim:].view(tq, kv_heads, dim))
        (q, k, v), (dq, dk, dv) = cut(qkv), cut(dqkv)
    elif layout == "heads first":
        q, k, v = rnd(heads, tq, dim).transpose(0, 1), rnd(kv_heads, tk, dim).transpose(0, 1), rnd(kv_heads, tk, dim).transpose(0, 1)
        dq, dk, dv = (torch.full((t.shape[1], t.shape[0], dim), float("nan"), device=DEV).half().transpose(0, 1) for t in (q, k, v))
    else:                                                    # rows further apart than they need to be
        wide = lambda t, h: rnd(t, h, dim + 24)[:, :, 8:8 + dim]
        q, k, v = wide(tq, heads), wide(tk, kv_heads), wide(tk, kv_heads)
        dq, dk, dv = (torch.full((t.shape[0], t.shape[1], dim + 8), float("nan"), device=DEV).half()[:, :, :dim] for t in (q, k, v))
    out, lse = torch.full((tq, heads, dim), float("nan"), device=DEV).half(), torch.full((heads, tq), float("nan"), device=DEV)
    do = rnd(tq, heads, dim, a=dstd)
    if fix:
        fix(q, k, v, do)
    scale = dim ** -0.5 if scale is None else scale
    starts = lambda ns: torch.tensor(np.concatenate([[0], np.cumsum(ns)]), dtype=torch.int32, device=DEV)
    args = dict(causal=causal, window=window, scale=scale)
    if len(lens_q) > 1 or layout == "starts":
        args.update(q_start=starts(lens_q), k_start=starts(lens_k), max_q=min(tq, max(lens_q) + slack))
    samo.samo_attention(q, k, v, out, lse, **args)
    if len(lens_q) > 1 or layout == "starts":
        args.update(max_k=min(tk, max(lens_k) + slack))
    samo.samo_attention_backward(do, q, k, v, out, lse, dq, dk, dv, **args)
    q0 = k0 = 0
    for n, m in zip(lens_q, lens_k):
        seen = seen_of(n, m, causal, window)
        grads = {}
        for h in range(heads):
            g = h * kv_heads // heads
            r, b = reference(q[q0:q0 + n, h], k[k0:k0 + m, g], v[k0:k0 + m, g], do[q0:q0 + n, h], scale, seen)
            got = dict(out=out[q0:q0 + n, h], dq=dq[q0:q0 + n, h])
            for name, most in (("out", 1.25), ("dq", 3.0)):
                d = (got[name].double() - r[name]).abs()
                bound = most * U * b[name] + U * r[name].abs() + 2.0 ** -25
                assert torch.all(d <= bound), (name, n, m, h, float((d - bound).max()))
            z, want = lse[h, q0:q0 + n].double(), r["lse"]
            empty = torch.isinf(want)
            assert torch.equal(torch.isneginf(z), empty)
            assert torch.all((z - want).abs()[~empty] <= (2.0 ** -23 * (dim + 8) * b["s"] + 2.0 ** -20 * (1 + want.abs()))[~empty])
            assert torch.all(out[q0:q0 + n, h][empty] == 0) and torch.all(dq[q0:q0 + n, h][empty] == 0)
            for name in ("dk", "dv"):
                a, c = grads.get((name, g), (0, 0))
                grads[name, g] = (a + r[name], c + b[name])
        for (name, g), (want, size) in grads.items():
            d = ((dk if name == "dk" else dv)[k0:k0 + m, g].double() - want).abs()
            bound = 3.0 * U * size + U * want.abs() + 2.0 ** -25
            assert torch.all(d <= bound), (name, n, m, g, float((d - bound).max()))
        q0, k0 = q0 + n, k0 + m


@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 48, 56, 64, 72, 80, 88, 96, 104, 112, 120, 128])
def test_every_head_dim(dim):
    check([130, 67], [130, 67], 4, 2, dim, True, 0, seed=dim)
    check([97], [97], 2, 2, dim, False, 0, seed=dim + 1, layout="wide")


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 640])
def test_lengths_around_the_tiles(n):
    check([n], [n], 2, 1, 64, True, 0, seed=n)
    check([n], [n], 1, 1, 128, False, 0, seed=n)


@pytest.mark.parametrize("layout", ["packed", "heads first", "wide", "starts"])
def test_layouts(layout):
    check([200], [200], 6, 2, 80, True, 0, layout=layout)


def test_sequences_of_no_and_one_token_among_others():
    check([0, 1, 200, 0, 3, 64, 1, 0], [0, 1, 200, 0, 3, 64, 1, 0], 4, 4, 64, True, 0, slack=77)
    check([0, 5, 0], [7, 0, 0], 2, 1, 64, False, 0)          # queries without keys, keys without queries


@pytest.mark.parametrize("window", [1, 2, 33, 64, 100, 5000])
def test_windows(window):
    check([300, 20], [300, 20], 2, 1, 96, True, window, seed=window)


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 50), (False, 0)])
def test_fewer_and_more_queries_than_keys(causal, window):
    check([70, 200], [333, 201], 4, 2, 128, causal, window)  # the last queries of longer contexts
    check([333, 130], [70, 1], 4, 2, 64, causal, window)     # the first queries see nothing


@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 1), (6, 3), (16, 16)])
def test_shared_heads(heads, kv):
    check([150], [150], heads, kv, 64, True, 0)


@pytest.mark.parametrize("dim", [24, 64])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 40), (False, 0)])
def test_many_workgroups(dim, causal, window):
    """8 sequences, 16 heads, 4 tiles of keys: enough for the form in which a wave has its keys for itself."""
    lens = [130, 0, 1, 64, 257, 200, 128, 65]
    check(lens, [n + 3 * i for i, n in enumerate(lens)], 16, 16, dim, causal, window, slack=230, seed=dim)


@pytest.mark.parametrize("dim", [80, 96, 104])
def test_more_workgroups(dim):
    """1024 workgroups of keys: the same form for the larger heads that have it."""
    lens = [130, 0, 1, 64, 257, 200, 128, 65]
    check(lens, [n + 3 * i for i, n in enumerate(lens)], 16, 16, dim, True, 0, slack=700, seed=dim)


@pytest.fixture
def parts(request):
    samo.samo_debug_set(samo.KNOB_ATTENTION_SPLIT, request.param)
    yield request.param
    samo.samo_debug_set(samo.KNOB_ATTENTION_SPLIT)


@pytest.mark.parametrize("parts", [1, 2, 3, 7, 16], indirect=True)
@pytest.mark.parametrize("dim", [32, 64, 72, 96, 128])
def test_keys_and_queries_in_parts(parts, dim):
    """Parts of one tile and of many, parts that hold nothing, sequences without any; the sums are fp32 whatever their order: the same bounds."""
    check([0, 1, 130, 300, 64], [7, 400, 131, 290, 0], 4, 2, dim, True, 0, seed=dim, slack=60)
    check([200, 70], [90, 515], 3, 1, dim, False, 0, seed=dim + 1)
    check([450, 20], [450, 20], 2, 2, dim, True, 70, seed=dim + 2)


@pytest.mark.parametrize("parts", [4], indirect=True)
def test_parts_of_large_scores(parts):
    """A part's exponents are taken against its own largest score: parts hundreds apart, either way round."""
    check([300], [300], 2, 2, 64, True, 0, std=6.0)

    def steps(sign):
        def fix(q, k, v, do):
            k.mul_((1 + sign * torch.arange(k.shape[0], device=DEV)[:, None, None].div(128).floor()).half())
        return fix
    check([64], [512], 1, 1, 64, False, 0, fix=steps(1.0))
    check([64], [512], 1, 1, 64, False, 0, fix=steps(-0.25))


@pytest.mark.parametrize("context", [1, 63, 1000, 9001])
def test_one_token_behind_a_context(context):
    """The form of generation: one query a sequence, split as the sizes make it."""
    check([1, 1, 1], [context, 5, max(1, context // 2)], 8, 2, 64, True, 0, seed=context)
    check([1], [context], 4, 4, 128, True, 300, seed=context)


def test_parts_where_there_is_no_memory_for_them():
    """An empty workspace: the forward pass by single workgroups; one of delta alone: the backward pass."""
    q, k, v, do = (torch.randn(2000, 2, 64, device=DEV).half() for _ in range(4))
    res = []
    for room in (None, 0, 4 * 2 * 2000):
        o, dq, dk, dv = (torch.full_like(q, float("nan")) for _ in range(4))
        lse = torch.zeros(2, 2000, device=DEV)
        ws = None if room is None else torch.empty(room, dtype=torch.uint8, device=DEV)
        samo.samo_attention(q, k, v, o, lse, workspace=ws)
        samo.samo_attention_backward(do, q, k, v, o, lse, dq, dk, dv, workspace=ws if room else None)
        res.append((o, dq, dk, dv))
    assert all(torch.equal(a, b) for a, b in zip(res[1][:1], res[2][:1]))
    for a, b in zip(res[0], res[2]):
        assert float((a.float() - b.float()).norm() / b.float().norm()) < 1e-2


def test_large_scores_and_small_gradients():
    """Scores of hundreds (one key takes all of a row), rows whose largest score comes last, gradients among fp16's small numbers."""
    check([300], [300], 2, 2, 64, True, 0, std=6.0)
    check([200], [200], 2, 2, 128, False, 0, dstd=2.0 ** -9)
    check([150], [150], 1, 1, 64, False, 0, std=1.0, scale=3.0)

    def rising(q, k, v, do):
        k.mul_(torch.linspace(0, 4, k.shape[0], device=DEV)[:, None, None].half())
        q.abs_()
        k.abs_()
    check([400], [400], 1, 1, 64, False, 0, fix=rising)


def test_far_keys_that_are_not_finite_do_not_reach_a_query():
    n, dim = 256, 64
    q, k, v = (torch.randn(n, 1, dim, device=DEV).half() for _ in range(3))
    out, lse, again, lse2 = torch.zeros_like(q), torch.zeros(1, n, device=DEV), torch.zeros_like(q), torch.zeros(1, n, device=DEV)
    samo.samo_attention(q, k, v, out, lse)
    k[192:] = float("nan")
    v[192:] = float("inf")
    samo.samo_attention(q, k, v, again, lse2)
    assert torch.equal(out[:192], again[:192]) and torch.equal(lse[:, :192], lse2[:, :192])
    assert torch.all(torch.isnan(again[192:]))
    # another sequence's, in the same tile
    k[:] = torch.randn(n, 1, dim, device=DEV).half()
    v[:] = torch.randn(n, 1, dim, device=DEV).half()
    starts = torch.tensor([0, 100, 256], dtype=torch.int32, device=DEV)
    samo.samo_attention(q, k, v, out, lse, causal=False, q_start=starts, k_start=starts)
    k[100:] = float("nan")
    v[100:] = float("nan")
    samo.samo_attention(q, k, v, again, lse2, causal=False, q_start=starts, k_start=starts)
    assert torch.equal(out[:100], again[:100])


def test_gradients_against_differences():
    """The loss sum(out * do): its change along a random direction of q, k and v against the gradients, in steps that fp16 holds exactly.
    The forward pass rounds to fp16 at 2^-11; over n * dim outputs those roundings add up as a random sum, 6 of whose deviations are granted."""
    n, dim, eps = 96, 64, 2.0 ** -4
    gen = torch.Generator(device=DEV)
    gen.manual_seed(4)
    grid = lambda: (torch.randn((n, 2, dim), generator=gen, device=DEV) * 16).round().div(16).half()
    q, k, v, do = grid(), grid(), grid(), grid()
    out, lse = torch.zeros_like(q), torch.zeros(2, n, device=DEV)
    samo.samo_attention(q, k, v, out, lse)
    grads = [torch.zeros_like(q) for _ in range(3)]
    samo.samo_attention_backward(do, q, k, v, out, lse, *grads)
    for which in range(3):
        way = torch.randint(0, 2, q.shape, generator=gen, device=DEV).half() * 2 - 1
        loss = []
        for sign in (1, -1):
            args = [q, k, v]
            args[which] = args[which] + sign * eps * way
            o = torch.zeros_like(q)
            samo.samo_attention(*args, o, lse)
            loss.append(float((o.double() * do.double()).sum()))
        slope = (loss[0] - loss[1]) / (2 * eps)
        want = float((grads[which].double() * way.double()).sum())
        noise = 6 * U * math.sqrt(float((out.double() * do.double()).square().sum()) * 2) / (2 * eps)
        third = 0.05 * float(grads[which].double().norm())           # the differences' own error, third order in eps
        assert abs(slope - want) <= noise + third, (which, slope, want)


def test_same_bits_again_other_stream_and_graph():
    n, dim = 500, 80
    q, k, v, do = (torch.randn(n, 4, dim, device=DEV).half() for _ in range(4))
    bufs = lambda: [torch.zeros(n, 4, dim, device=DEV).half() for _ in range(4)] + [torch.zeros(4, n, device=DEV)]

    def call(o, dq, dk, dv, lse, ws=None):
        samo.samo_attention(q, k, v, o, lse)
        samo.samo_attention_backward(do, q, k, v, o, lse, dq, dk, dv, workspace=ws)

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


def test_rows_past_two_gibibytes():
    """A key/value slice whose rows are so far apart that the last ones begin past 2^31 bytes."""
    n, dim, apart = 700, 64, 1 << 21
    room = torch.zeros((n, apart), dtype=torch.float16, device=DEV)
    k, v = room[:, :dim].unsqueeze(1), room[:, 64:64 + dim].unsqueeze(1)
    kk, vv, q = (torch.randn(n, 1, dim, device=DEV).half() for _ in range(3))
    k.copy_(kk)
    v.copy_(vv)
    a, b, lse = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(1, n, device=DEV)
    samo.samo_attention(q, k, v, a, lse)
    samo.samo_attention(q, kk, vv, b, lse)
    assert torch.equal(a, b)


def test_native_and_python_descriptors_agree():
    """The descriptor's fields of a tensor, written by native code and in Python, and the refusals of both."""
    import ctypes
    whole = torch.zeros(6, 5, 16, device=DEV).half()
    kinds = [whole, whole[:, :, :8], whole[:, 1:3], whole.transpose(0, 1), whole[:1], whole[:, :1], whole[:0], torch.nn.Parameter(whole), whole.float(),
             whole[0], whole[:, :, ::2], whole.cpu(), None, [1]]
    for t in kinds:
        for shape in ((-1, -1, -1), (6, 5, 16), (1, 5, 16)):
            made = samo.AttentionDesc()
            made.q.row = 77
            done = samo._marshal.heads(ctypes.addressof(made) + samo._HEADS_AT["q"], t, *shape)
            try:
                want = samo._heads(t, "q", None if shape[0] < 0 else shape)
            except (TypeError, ValueError):
                assert not done and made.q.row == 77
                continue
            if done:
                assert (made.q.d_data, made.q.row, made.q.head) == (want.d_data, want.row, want.head)
            samo._set_heads(made, "q", t, *shape)
            assert (made.q.d_data, made.q.row, made.q.head) == (want.d_data, want.row, want.head)


def reached(seen, bad_q, bad_k, block_k):
    """Which queries and keys share a block (32 queries, block_k keys) that holds a seen pair with one of the bad ones."""
    n, m = seen.shape
    qs, ks = -(-n // 32), -(-m // block_k)
    whole = torch.zeros((qs * 32, ks * block_k), dtype=torch.bool, device=DEV)
    whole[:n, :m] = seen
    meet = whole.view(qs, 32, ks, block_k).any(3).any(1)
    spread = lambda bad, count, size: torch.nn.functional.pad(bad, (0, count * size - bad.numel())).view(count, size).any(1)
    of_q = (meet & spread(bad_k, ks, block_k)[None]).any(1).repeat_interleave(32)[:n]
    of_k = (meet & spread(bad_q, qs, 32)[:, None]).any(0).repeat_interleave(block_k)[:m]
    return of_q, of_k


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,prefix,window,bad", [(200, 0, 0, 70), (200, 10, 0, 70), (200, 10, 16, 70), (200, 33, 100, 130), (160, 300, 20, 5), (300, 1, 0, 255)])
def test_what_is_not_finite_reaches_no_further_than_its_blocks(n, prefix, window, bad, dim):
    """A key, value, query or gradient that is not finite reaches the rows whose block of 32 queries and 64 keys (gradients: 32) holds a pair that the mask
    leaves, and no other; where a query does not see the key, lse is as it was."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n + prefix)
    m = n + prefix
    rnd = lambda t: torch.randn((t, 1, dim), generator=gen, device=DEV).half()
    q, k, v, do = rnd(n), rnd(m), rnd(m), rnd(n)
    seen = seen_of(n, m, True, window)

    def run(q, k, v, do):
        out, lse, dq, dk, dv = torch.zeros_like(q), torch.zeros(1, n, device=DEV), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        samo.samo_attention(q, k, v, out, lse, window=window)
        samo.samo_attention_backward(do, q, k, v, out, lse, dq, dk, dv, window=window)
        return out, lse[0], dq, dk, dv

    clean = run(q, k, v, do)
    assert all(torch.all(torch.isfinite(t)) for t in clean)
    bad_k = torch.zeros(m, dtype=torch.bool, device=DEV)
    bad_k[bad] = True
    k2, v2 = k.clone(), v.clone()
    k2[bad], v2[bad] = float("nan"), float("inf")
    for keys, values in ((k2, v2), (k, v2), (k2, v)):
        got = run(q, keys, values, do)
        bad_q, _ = reached(seen, torch.zeros(n, dtype=torch.bool, device=DEV), bad_k, 64)
        hidden = ~seen[:, bad]
        assert torch.equal(got[0][~bad_q], clean[0][~bad_q]) and torch.equal(got[2][~bad_q], clean[2][~bad_q])
        assert torch.all((got[1] - clean[1])[hidden].abs() <= 2.0 ** -19 * (1 + clean[1][hidden].abs()))
        assert not torch.isfinite(got[0][~hidden]).all(2).any()
        _, keys_hit = reached(seen, bad_q, bad_k, 32)
        for i in (3, 4):
            assert torch.equal(got[i][~keys_hit & ~bad_k], clean[i][~keys_hit & ~bad_k])
    hit = n // 2
    one = torch.zeros(n, dtype=torch.bool, device=DEV)
    one[hit] = True
    _, keys_hit = reached(seen, one, torch.zeros(m, dtype=torch.bool, device=DEV), 32)
    q2, do2 = q.clone(), do.clone()
    q2[hit], do2[hit] = float("nan"), float("inf")
    for queries, grads in ((q2, do), (q, do2)):
        got = run(queries, k, v, grads)
        assert torch.equal(got[0][~one], clean[0][~one]) or queries is q2
        for i in (3, 4):
            assert torch.equal(got[i][~keys_hit], clean[i][~keys_hit])


@pytest.mark.parametrize("dim", [64, 80, 128])
def test_gradients_of_large_losses(dim):
    """dP - delta of tens of thousands; from 65504 on dS, as any fp16 gradient, is infinite, and what is formed from it is no finite number."""
    check([2] * 12, [2] * 12, 8, 4, dim, False, 0, dstd=1500.0)
    q, k, v, do = (torch.zeros(2, 1, dim, device=DEV).half() for _ in range(4))
    k[0], k[1], v[0], v[1], do[:] = 0.5, -0.5, 60.0, -60.0, 60.0
    out, lse, dq, dk, dv = torch.zeros_like(q), torch.zeros(1, 2, device=DEV), torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    samo.samo_attention(q, k, v, out, lse, causal=False)
    samo.samo_attention_backward(do, q, k, v, out, lse, dq, dk, dv, causal=False)
    assert torch.all(out == 0) and torch.all(dv == 60.0)      # P is 1/2 everywhere, |dS| = 1800 dim
    assert not torch.isfinite(dq).any() and not torch.isfinite(dk).any()


@pytest.mark.parametrize("name", ["window", "max_q", "max_k"])
def test_numbers_that_do_not_fit_the_descriptor_are_refused(name):
    """2^32 and more would become small numbers in a 32-bit field: another window, rows that are not computed."""
    q = torch.zeros(6, 2, 16, device=DEV).half()
    out, lse = torch.full_like(q, 7.0), torch.zeros(2, 6, device=DEV)
    for value in (2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 32):
        with pytest.raises(ValueError):
            samo.samo_attention(q, q, q, out, lse, **{name: value})
        with pytest.raises(ValueError):
            samo.samo_attention_backward(q, q, q, q, out, lse, out, out, out, **{name: value})
    assert torch.all(out == 7.0)


@pytest.mark.parametrize("parts", [1, 3], indirect=True)
@pytest.mark.parametrize("heads,kv,lens", [(25, 25, [130, 40, 257]), (50, 25, [129, 1, 200]), (67, 67, [300])])
def test_heads_that_do_not_divide_among_the_xcds(heads, kv, lens, parts):
    """More than 64 heads and sequences, not a multiple of 8: the last XCD has fewer, and some of a launch's workgroups none."""
    check(lens, [n + 7 for n in lens], heads, kv, 64, True, 0, seed=heads)
    check(lens, lens, heads, kv, 128, False, 0, seed=heads + 1)


def within_bounds(q, k, v, do, scale, seen, out=None, dq=None, dk=None, dv=None):
    """One head's results element by element, as in check()."""
    r, b = reference(q, k, v, do, scale, seen)
    for name, got, most in (("out", out, 1.25), ("dq", dq, 3.0), ("dk", dk, 3.0), ("dv", dv, 3.0)):
        if got is not None:
            d = (got.double() - r[name]).abs()
            bound = most * U * b[name] + U * r[name].abs() + 2.0 ** -25
            assert torch.all(d <= bound), (name, float((d - bound).max()))


@pytest.mark.parametrize("room", [None, 0, 4 * 2 * 2000])
def test_parts_and_no_memory_for_them_element_by_element(room):
    """With the memory for parts and without it: every element of out and of the gradients."""
    q, k, v, do = (torch.randn(2000, 2, 64, device=DEV).half() for _ in range(4))
    out, dq, dk, dv = (torch.full_like(q, float("nan")) for _ in range(4))
    lse = torch.zeros(2, 2000, device=DEV)
    ws = None if room is None else torch.empty(room, dtype=torch.uint8, device=DEV)
    samo.samo_attention(q, k, v, out, lse, workspace=ws)
    samo.samo_attention_backward(do, q, k, v, out, lse, dq, dk, dv, workspace=ws if room else None)
    for h in range(2):
        within_bounds(*(t[:, h] for t in (q, k, v, do)), 0.125, seen_of(2000, 2000, True, 0), out[:, h], dq[:, h], dk[:, h], dv[:, h])


@pytest.mark.parametrize("n,apart", [(700, 1 << 21), (200, 1 << 24)])
def test_rows_past_two_gibibytes_backward(n, apart):
    """Every tensor a slice whose rows lie so far apart that the last ones begin past 2^31 bytes, read and written."""
    dim = 64
    room = torch.full((n, apart), float("nan"), dtype=torch.float16, device=DEV)
    q, k, v, do, out, dq, dk, dv = (room[:, 64 * i:64 * i + dim].unsqueeze(1) for i in range(8))
    near = [torch.randn(n, 1, dim, device=DEV).half() for _ in range(4)]
    for far, t in zip((q, k, v, do), near):
        far.copy_(t)
    lse = torch.zeros(1, n, device=DEV)
    samo.samo_attention(q, k, v, out, lse)
    samo.samo_attention_backward(do, q, k, v, out, lse, dq, dk, dv)
    a, b, c, d, lse2 = *(torch.zeros_like(t) for t in near), torch.zeros(1, n, device=DEV)
    samo.samo_attention(*near[:3], a, lse2)
    samo.samo_attention_backward(near[3], *near[:3], a, lse2, b, c, d)
    assert torch.equal(lse, lse2)
    for far, t in zip((out, dq, dk, dv), (a, b, c, d)):
        assert torch.equal(far, t)
    assert torch.isnan(room[:, 512:520]).all()
