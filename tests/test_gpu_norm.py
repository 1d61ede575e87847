"""The norms around a block, forward and backward, against the definition in 64 bits (its gradients by torch's autograd).

Tolerances (u = 2^-11: fp16's rounding; e = 2^-24: fp32's).  A statistic is a sum of squares of `hidden` terms in fp32: within (hidden / threads + 20) e
<= 2^-18 of itself; the differences from the mean are within 2^-18 of the row's spread.  So a normed value is within 2^-17 (|x| + 1) and
    |d s'| <= u_s |s'| + 2^-16 |scale gate| (|n| + |wy|),        u_s: u, or e for a stream in fp32
    |d out| <= u |out| + 2^-15 (|w| (|x| + 1)) + what y's norm brings: 2^-16 |scale gate| (|n| + |wy|) r |w|
Backward: the norm of s' is formed from the stored s', so x is off by u_s |s'| r besides.  The gradient through a norm is off by the terms' magnitudes
times the offs of x, and by 2^-15 of them: with G = |g| + (|g| mean |x|) + |x| mean |g x| in magnitudes,
    |d D| <= u_s |D| + r (2^-15 G + dx-terms),      dx-terms = |off x| mean |g x| + |x| mean(|g| off x)
and so on through y's norm, whose input is exact.  The vectors' sums: the terms' offs added, 2^-15 of the terms' magnitudes, rounded once by u.
fp16 results among the subnormal numbers: 2^-25 more.  Every bound is element by element.
"""
import pytest
import torch

import paper_2302_05045_amd as samo
from gpu_util import DEV

pytestmark = pytest.mark.gpu
U, E = 2.0 ** -11, 2.0 ** -24
EPS = 1e-5


def normed(x, kind):
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    r = (x.square().mean(1, keepdim=True) + EPS).rsqrt()
    return x * r, r


def through(g, x, r, kind):
    if kind == "layer":
        g = g - g.mean(1, keepdim=True)
    return r * (g - x * (g * x).mean(1, keepdim=True))


def magnitudes(g, x, r, off_x):
    """Of what goes into the gradient through a norm, and how far x's offs take it."""
    mean = lambda t: t.mean(1, keepdim=True)
    g, x = g.abs(), x.abs()
    return r * (g + mean(g) + x * mean(g * x)), r * (off_x * mean(g * x) + x * mean(g * off_x))


def check(tokens, hidden, kind="rms", after="norm", vectors="wbWBg", scale=0.5, stream32=False, seed=0, std=2.0, mean=0.1, dnew=True, in_place=False, fix=None):
    """vectors: which of weight, bias, y_weight (W), y_bias (B) and gate there are."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rnd = lambda *s, a=1.0, m=0.0: (torch.randn(s, generator=gen, device=DEV) * a + m).half()
    kept = dict(weight=rnd(hidden, a=0.2, m=1.0), bias=rnd(hidden, a=0.3), y_weight=rnd(hidden, a=0.2, m=1.0), y_bias=rnd(hidden, a=0.3), gate=rnd(hidden, a=0.5))
    letters = dict(zip("wbWBg", kept))
    names = [letters[c] for c in vectors if (c in "wb" or after) and (c not in "WB" or after == "norm")]
    vec = {n: kept[n] if n in names else None for n in kept}
    dtype, us = (torch.float32, E) if stream32 else (torch.float16, U)
    stream = rnd(tokens, hidden, a=std, m=mean).to(dtype)
    y = rnd(tokens, hidden, a=1.5, m=mean) if after else None
    if fix:
        fix(stream, y)
    dout, dn_in = rnd(tokens, hidden), rnd(tokens, hidden).to(dtype) if dnew else None
    norm = samo.Norm(kind=kind, eps=EPS, y_norm=after == "norm", scale=scale, **vec)
    nan = lambda t, like=None: torch.full(t.shape, float("nan"), device=DEV, dtype=like or t.dtype)
    first = stream.clone()
    new = (first if in_place else nan(stream)) if after else None
    out, stats = nan(stream, torch.float16), torch.full((tokens, 4), float("nan"), device=DEV)
    samo.samo_norm(norm, first, out, y=y, new_stream=new, stats=stats)
    again = nan(out)
    samo.samo_norm(norm, stream, again, y=y, new_stream=nan(stream) if after else None)          # without stats: the same bits
    assert torch.equal(again, out)
    grads = samo.NormGrads(**{n: nan(vec[n]) for n in names})
    held = dn_in.clone() if in_place and dnew else None
    dstream, dy = held if held is not None else nan(stream), nan(y) if after else None
    samo.samo_norm_backward(norm, dout, new if after else first, stats, dstream, dnew=held if held is not None else dn_in, y=y, dy=dy, grads=grads)

    d = lambda t, other: other if t is None else t.double()
    w, b, wy, by = d(vec["weight"], 1.0), d(vec["bias"], 0.0), d(vec["y_weight"], 1.0), d(vec["y_bias"], 0.0)
    f = scale * d(vec["gate"], 1.0)
    ones = torch.ones(hidden, device=DEV, dtype=torch.float64)
    s, off_s = stream.double(), torch.zeros_like(stream, dtype=torch.float64)
    if after:
        yn, ry = normed(y.double(), kind) if after == "norm" else (y.double(), None)
        n = yn * wy + by if after == "norm" else yn
        s = s + f * n
        off_s = 2.0 ** -16 * abs(f * ones) * (n.abs() + abs(wy * ones) if after == "norm" else n.abs())
        off = (new.double() - s).abs()
        assert torch.all(off <= us * s.abs() + off_s + 2.0 ** -25), ("new stream", float((off - us * s.abs() - off_s).max()))
    x, r = normed(s, kind)
    want = x * w + b
    off, bound = (out.double() - want).abs(), U * want.abs() + 2.0 ** -15 * abs(w * ones) * (x.abs() + 1) + off_s * r * abs(w * ones) + 2.0 ** -25
    assert torch.all(off <= bound), ("out", float((off / bound).max()))

    g = dout.double()
    off_x = 2.0 ** -17 * (x.abs() + 1) + (us * s.abs() + off_s) * r
    size, through_off = magnitudes(g * w, x, r, off_x)
    D = d(dn_in, 0.0) + through(g * w, x, r, kind)
    off_D = 2.0 ** -15 * size + through_off
    got = {"dstream": dstream, "weight": grads.weight, "bias": grads.bias, "dy": dy, "y_weight": grads.y_weight, "y_bias": grads.y_bias, "gate": grads.gate}
    result = {"dstream": (D, us * D.abs() + off_D + (0 if stream32 else 2.0 ** -25))}
    vector = lambda t, off, terms: (t.sum(0), U * t.sum(0).abs() + off.sum(0) + 2.0 ** -15 * terms.abs().sum(0) + 2.0 ** -25)
    result["weight"], result["bias"] = vector(g * x, g.abs() * off_x, g * x), vector(g, 0 * g, g)
    if after:
        dn, off_dn = f * D, abs(f * ones) * off_D
        result["gate"] = vector(scale * n * D, abs(scale) * (n.abs() * off_D + 2.0 ** -16 * (n.abs() + abs(wy * ones)) * D.abs()),
                                abs(scale) * D.abs() * (yn.abs() * abs(wy * ones) + abs(by * ones) if after == "norm" else yn.abs()))
        if after == "norm":
            off_y = 2.0 ** -17 * (yn.abs() + 1)
            size, through_off = magnitudes(dn * wy, yn, ry, off_y)
            dy_want = through(dn * wy, yn, ry, kind)
            off_dy = 2.0 ** -15 * size + through_off + magnitudes(off_dn * wy, yn, ry, off_y)[0]
            result["y_weight"] = vector(dn * yn, off_dn * yn.abs() + dn.abs() * off_y, dn * yn)
            result["y_bias"] = vector(dn, off_dn, dn)
        else:
            dy_want, off_dy = dn, off_dn
        result["dy"] = (dy_want, U * dy_want.abs() + off_dy + 2.0 ** -16 * dy_want.abs() + 2.0 ** -25)
    for name, t in got.items():
        if t is None:
            continue
        want, bound = result[name]
        off = (t.double() - want).abs()
        assert torch.all(off <= bound), (name, float((off / bound).max()), float((off - bound).max()))
    return out, new, dstream, dy, grads


KINDS = [("rms", "norm"), ("layer", "norm"), ("rms", "plain"), ("layer", "plain"), ("rms", ""), ("layer", "")]


@pytest.mark.parametrize("kind,after", KINDS)
@pytest.mark.parametrize("hidden", [8, 64, 72, 512, 520, 1000, 1024, 2560, 4096, 4104, 5120, 8192, 8200, 16376, 16384])
def test_every_width(hidden, kind, after):
    check(5, hidden, kind, after, seed=hidden)
    check(3, hidden, kind, after, seed=hidden + 1, stream32=True)


@pytest.mark.parametrize("kind,after", KINDS)
@pytest.mark.parametrize("tokens", [1, 2, 255, 513, 1030, 2100])
def test_numbers_of_tokens(tokens, kind, after):
    """One row to a workgroup and several, an uneven number of them."""
    check(tokens, 136, kind, after, seed=tokens)
    check(tokens, 136, kind, after, seed=tokens, stream32=True, in_place=True)


@pytest.mark.parametrize("vectors", ["", "w", "b", "W", "B", "g", "wg", "Bg", "WB", "bWB"])
@pytest.mark.parametrize("kind,after", KINDS)
def test_vectors_that_are_not_there(vectors, kind, after):
    check(40, 256, kind, after, vectors)


@pytest.mark.parametrize("kind,after", KINDS)
@pytest.mark.parametrize("stream32", [False, True])
def test_in_place_and_without_a_gradient_from_further_on(kind, after, stream32):
    plain = check(70, 320, kind, after, stream32=stream32)
    placed = check(70, 320, kind, after, stream32=stream32, in_place=True)
    for a, b in zip(plain[:4], placed[:4]):
        assert (a is None and b is None) or torch.equal(a, b)
    check(70, 320, kind, after, stream32=stream32, dnew=False)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_rows_of_zeros_of_one_value_and_far_from_zero(kind):
    def fix(stream, y):
        stream[0], y[0] = 0.0, 0.0                           # eps alone
        y[1] = 3.0                                           # nothing but a mean
        stream[2, 5] = 300.0                                 # one channel above all others
        y[3, 0] = -200.0
    check(6, 512, kind, "norm", fix=fix)
    check(6, 512, kind, "plain", fix=fix)
    check(20, 1024, kind, "norm", mean=30.0, stream32=True)  # a mean 15 times the spread: what a variance by differences of squares would lose


@pytest.mark.parametrize("scale", [0.0, -1.5, 0.01])
def test_scales(scale):
    check(30, 264, "rms", "norm", scale=scale)
    check(30, 264, "layer", "plain", scale=scale)


def test_vectors_that_are_not_wanted():
    """Each gradient by itself, some, none (no workspace, no second kernel): the same bits as all of them."""
    t, h = 100, 264
    rnd = lambda *s: torch.randn(s, device=DEV).half()
    vec = dict(weight=rnd(h), bias=rnd(h), y_weight=rnd(h), y_bias=rnd(h), gate=rnd(h))
    norm = samo.Norm(kind="layer", y_norm=True, **vec)
    s, y, dout, dnew = rnd(t, h), rnd(t, h), rnd(t, h), rnd(t, h)
    new, out, stats = torch.zeros_like(s), torch.zeros_like(s), torch.zeros(t, 4, device=DEV)
    samo.samo_norm(norm, s, out, y=y, new_stream=new, stats=stats)

    def back(names):
        g = {n: torch.full((h,), float("nan"), device=DEV).half() for n in names}
        ds, dy = torch.zeros_like(s), torch.zeros_like(s)
        samo.samo_norm_backward(norm, dout, new, stats, ds, dnew=dnew, y=y, dy=dy, grads=samo.NormGrads(**g) if names else None)
        return ds, dy, g

    every = back(list(vec))
    for names in [[n] for n in vec] + [["weight", "gate"], ["y_bias", "bias"], []]:
        got = back(names)
        assert torch.equal(got[0], every[0]) and torch.equal(got[1], every[1])
        assert all(torch.equal(got[2][n], every[2][n]) for n in names)


def test_no_tokens():
    h = 64
    norm = samo.Norm(weight=torch.ones(h, device=DEV).half())
    none, stats = torch.zeros(0, h, device=DEV).half(), torch.zeros(0, 4, device=DEV)
    samo.samo_norm(norm, none, none, stats=stats)
    grad = torch.full((h,), float("nan"), device=DEV).half()
    samo.samo_norm_backward(norm, none, none, stats, none, grads=samo.NormGrads(weight=grad))
    assert torch.all(grad == 0)


def test_what_is_not_finite_stays_in_its_row():
    t, h = 600, 264
    rnd = lambda *s: torch.randn(s, device=DEV).half()
    norm = samo.Norm(y_norm=True, weight=rnd(h))
    s, y, dout = rnd(t, h), rnd(t, h), rnd(t, h)

    def run(s, y, dout):
        new, out, ds, dy = (torch.zeros_like(s) for _ in range(4))
        stats, gw = torch.zeros(t, 4, device=DEV), torch.zeros(h, device=DEV).half()
        samo.samo_norm(norm, s, out, y=y, new_stream=new, stats=stats)
        samo.samo_norm_backward(norm, dout, new, stats, ds, y=y, dy=dy, grads=samo.NormGrads(weight=gw))
        return new, out, ds, dy

    clean = run(s, y, dout)
    for which in range(3):
        bad = [a.clone() for a in (s, y, dout)]
        bad[which][77, 3], bad[which][400, 0] = float("nan"), float("inf")
        rows = torch.ones(t, dtype=torch.bool, device=DEV)
        rows[[77, 400]] = False
        for a, b in zip(run(*bad), clean):
            assert torch.equal(a[rows], b[rows])


def test_gradients_against_differences():
    """The loss sum(out dout + s' dnew) along a random direction of every input; a stream in fp32, steps that fp16 holds exactly.  out's roundings add
    up as a random sum, 6 of whose deviations are granted, and the differences' own error is of third order in the step."""
    t, h, eps = 48, 64, 2.0 ** -5
    gen = torch.Generator(device=DEV)
    gen.manual_seed(9)
    grid = lambda *s, m=0: ((torch.randn(s, generator=gen, device=DEV) * 16).round().div(16) + m).half()
    args = dict(stream=grid(t, h).float(), y=grid(t, h), weight=grid(h, m=1), bias=grid(h), y_weight=grid(h, m=1), y_bias=grid(h), gate=grid(h))
    dout, dnew = grid(t, h), grid(t, h).float()

    def forward(a):
        norm = samo.Norm(kind="layer", y_norm=True, scale=0.5, **{n: a[n] for n in ("weight", "bias", "y_weight", "y_bias", "gate")})
        new, out, stats = torch.zeros_like(a["stream"]), torch.zeros_like(dout), torch.zeros(t, 4, device=DEV)
        samo.samo_norm(norm, a["stream"], out, y=a["y"], new_stream=new, stats=stats)
        return norm, new, out, stats

    norm, new, out, stats = forward(args)
    ds, dy, g = torch.zeros_like(new), torch.zeros_like(out), {n: torch.zeros(h, device=DEV).half() for n in ("weight", "bias", "y_weight", "y_bias", "gate")}
    samo.samo_norm_backward(norm, dout, new, stats, ds, dnew=dnew, y=args["y"], dy=dy, grads=samo.NormGrads(**g))
    grads = dict(g, stream=ds, y=dy)
    for name, x in args.items():
        way = (torch.randint(0, 2, x.shape, generator=gen, device=DEV) * 2 - 1).to(x.dtype)
        loss = []
        for sign in (1, -1):
            _, s2, o2, _ = forward(dict(args, **{name: x + sign * eps * way}))
            loss.append(float((o2.double() * dout.double()).sum() + (s2.double() * dnew.double()).sum()))
        slope, want = (loss[0] - loss[1]) / (2 * eps), float((grads[name].double() * way.double()).sum())
        noise = 6 * U * float((out.double() * dout.double()).square().sum() * 2) ** 0.5 / (2 * eps)
        assert abs(slope - want) <= noise + 0.05 * float(grads[name].double().norm()), (name, slope, want)


def test_same_bits_again_other_stream_and_graph():
    t, h = 1100, 520
    rnd = lambda *s: torch.randn(s, device=DEV).half()
    norm = samo.Norm(kind="layer", y_norm=True, weight=rnd(h), bias=rnd(h), y_weight=rnd(h), gate=rnd(h))
    s, y, dout, dnew = rnd(t, h), rnd(t, h), rnd(t, h), rnd(t, h)
    bufs = lambda: [torch.zeros(t, h, device=DEV).half() for _ in range(4)] + [torch.zeros(t, 4, device=DEV)] + [torch.zeros(h, device=DEV).half() for _ in range(4)]

    def call(new, out, ds, dy, stats, gw, gb, gy, gg):
        samo.samo_norm(norm, s, out, y=y, new_stream=new, stats=stats)
        samo.samo_norm_backward(norm, dout, new, stats, ds, dnew=dnew, y=y, dy=dy, grads=samo.NormGrads(weight=gw, bias=gb, y_weight=gy, gate=gg))

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
        for x in third:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(first, second, third):
            assert torch.equal(a, b) and torch.equal(a, c)
        call(*bufs())


@pytest.mark.parametrize("stream32", [False, True])
def test_rows_past_two_gibibytes(stream32):
    """More than 2^31 bytes in each tensor: the last rows are those of a call of their own."""
    t, h = 140000, 8192
    dtype = torch.float32 if stream32 else torch.float16
    s = torch.randn(2000, h, device=DEV).to(dtype).repeat(t // 2000, 1)
    out, stats, ds = torch.empty(t, h, dtype=torch.float16, device=DEV), torch.empty(t, 4, device=DEV), torch.empty_like(s)
    norm = samo.Norm(weight=torch.randn(h, device=DEV).half())
    samo.samo_norm(norm, s, out, stats=stats)
    samo.samo_norm_backward(norm, out, s, stats, ds)
    o2, st2, d2 = torch.empty(2000, h, dtype=torch.float16, device=DEV), torch.empty(2000, 4, device=DEV), torch.empty_like(s[:2000])
    samo.samo_norm(norm, s[:2000], o2, stats=st2)
    samo.samo_norm_backward(norm, o2, s[:2000], st2, d2)
    for first in (0, t // 2, t - 2000):
        assert torch.equal(out[first:first + 2000], o2) and torch.equal(ds[first:first + 2000], d2)


def test_workspaces_of_the_callers_own():
    import ctypes
    t, h = 900, 136
    rnd = lambda *s: torch.randn(s, device=DEV).half()
    norm = samo.Norm(weight=rnd(h), bias=rnd(h))
    s, dout = rnd(t, h), rnd(t, h)
    out, stats, ds, gw, gb = torch.zeros_like(s), torch.zeros(t, 4, device=DEV), torch.zeros_like(s), rnd(h), rnd(h)
    samo.samo_norm(norm, s, out, stats=stats)
    d = samo._norm_desc(norm, None, None, norm.weight, norm.bias, None, None, None, s, None, stats, dout, None, ds, None, gw, gb, None, None, None)
    need = ctypes.c_size_t()
    assert samo.lib().samo_norm_workspace_bytes(ctypes.byref(d), ctypes.byref(need)) == 0 and need.value > 0
    res = []
    for room in (None, need.value, need.value + 1000):
        ws = None if room is None else torch.full((room,), 255, dtype=torch.uint8, device=DEV)
        samo.samo_norm_backward(norm, dout, s, stats, ds, grads=samo.NormGrads(weight=gw, bias=gb), workspace=ws)
        res.append((gw.clone(), gb.clone()))
        assert ws is None or torch.all(ws[need.value:] == 255)
    assert all(torch.equal(a, b) for r in res[1:] for a, b in zip(res[0], r))
    with pytest.raises(samo.SamoError):
        samo.samo_norm_backward(norm, dout, s, stats, ds, grads=samo.NormGrads(weight=gw, bias=gb), workspace=torch.empty(need.value - 1, dtype=torch.uint8, device=DEV))


def test_refusals_of_the_binding():
    t, h = 4, 16
    s, w = torch.full((t, h), 7.0, device=DEV).half(), torch.ones(h, device=DEV).half()
    out, stats = torch.full_like(s, 7.0), torch.zeros(t, 4, device=DEV)
    new = torch.full_like(s, 7.0)
    for norm, kw, what in ((samo.Norm(kind="batch"), {}, ValueError), (samo.Norm(weight=w[:8]), {}, ValueError), (samo.Norm(weight=w.float()), {}, TypeError),
                           (samo.Norm(weight=w.cpu()), {}, TypeError), (samo.Norm(eps=0.0), {}, samo.SamoError), (samo.Norm(eps=float("nan")), {}, samo.SamoError),
                           (samo.Norm(), dict(y=s), ValueError), (samo.Norm(), dict(new_stream=new), ValueError), (samo.Norm(), dict(y=s[:2], new_stream=new), ValueError),
                           (samo.Norm(), dict(y=s.float(), new_stream=new), TypeError), (samo.Norm(), dict(y=s, new_stream=new.float()), TypeError),
                           (samo.Norm(), dict(y=s, new_stream=out), samo.SamoError), (samo.Norm(scale=float("inf")), dict(y=s, new_stream=new), samo.SamoError),
                           (samo.Norm(), dict(stats=stats[:, :3]), TypeError), (samo.Norm(), dict(stats=stats[:2]), ValueError)):
        with pytest.raises(what):
            samo.samo_norm(norm, s, out, **kw)
    with pytest.raises(TypeError):
        samo.samo_norm(samo.Norm(), s.bfloat16(), out)
    with pytest.raises(TypeError):
        samo.samo_norm(samo.Norm(), s.t(), out)
    with pytest.raises(samo.SamoError):
        samo.samo_norm(samo.Norm(), s[:, :12].contiguous(), out[:, :12].contiguous())
    with pytest.raises(TypeError):
        samo.samo_norm(samo.Norm(), s, out.cpu())
    ds = torch.full_like(s, 7.0)
    for kw in (dict(y=s), dict(dy=new), dict(dnew=s.float()), dict(dnew=s[:2]), dict(grads=samo.NormGrads(weight=w[:8]))):
        with pytest.raises((ValueError, TypeError)):
            samo.samo_norm_backward(samo.Norm(), s, s, stats, ds, **kw)
    for kw in (dict(grads=samo.NormGrads(gate=w)), dict(grads=samo.NormGrads(y_weight=w)), dict(y=s, dy=ds)):
        with pytest.raises(samo.SamoError):
            samo.samo_norm_backward(samo.Norm(), s, s, stats, ds, **kw)
    assert torch.all(out == 7.0) and torch.all(new == 7.0) and torch.all(ds == 7.0)


def test_native_and_python_descriptors_agree():
    """The descriptor's fields by native code and in Python, for what both take; what one refuses the other refuses."""
    import ctypes
    t, h = 6, 16
    m, v = torch.zeros(t, h, device=DEV).half(), torch.zeros(h, device=DEV).half()
    good = [m] * 2 + [v] * 5 + [m] * 2 + [torch.zeros(t, 4, device=DEV)] + [m] * 4 + [v] * 5
    others = [None, m.float(), m[:3], m[:, :8], m.t(), m.cpu(), v.float(), v[:8], v[::2], m[:0], torch.zeros(t, 4, device=DEV), torch.nn.Parameter(m), [1], m[None]]
    fields = [name for name, _ in samo.NormDesc._fields_]
    for at in range(-1, len(good)):
        for other in others if at >= 0 else [None]:
            tensors = list(good)
            if at >= 0:
                tensors[at] = other
            native, python = samo.NormDesc(), samo.NormDesc()
            done = samo._marshal.norm(ctypes.addressof(native), tuple(tensors))
            try:
                samo._norm_pointers(python, tuple(tensors))
            except (TypeError, ValueError):
                assert not done, (at, other)
                continue
            if done:
                assert all(getattr(native, name) == getattr(python, name) for name in fields), at


@pytest.mark.parametrize("kind,after", KINDS)
def test_no_tokens_give_vectors_of_zeros(kind, after):
    """A micro-batch without tokens, whatever is around it: zeros, also where a vector holds what is not finite; by native code and in Python."""
    h = 72
    some = lambda *at: torch.ones(h, device=DEV).half().index_fill_(0, torch.tensor(at, device=DEV, dtype=torch.long), float("inf"))
    names = ["weight", "bias"] + ["gate"] * bool(after) + ["y_weight", "y_bias"] * (after == "norm")
    norm = samo.Norm(kind=kind, y_norm=after == "norm", scale=0.5, **{n: some(3, 5) for n in names})
    for stream32 in (False, True):
        rows, stats = torch.zeros(0, h, device=DEV).half(), torch.zeros(0, 4, device=DEV)
        stream = rows.float() if stream32 else rows
        y = rows if after else None
        samo.samo_norm(norm, stream, rows, y=y, new_stream=stream if after else None, stats=stats)
        for native in (samo._marshal, None):
            grads = samo.NormGrads(**{n: torch.full((h,), float("nan"), device=DEV).half() for n in names})
            kept, samo._marshal = samo._marshal, native
            try:
                samo.samo_norm_backward(norm, rows, stream, stats, stream, dnew=stream, y=y, dy=y, grads=grads)
            finally:
                samo._marshal = kept
            assert all(torch.all(getattr(grads, n) == 0) for n in names)
