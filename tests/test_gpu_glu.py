"""The gated feed-forward block, forward and backward, against the definition in 64 bits.

Tolerances.  Operands are fp16, their products exact in fp32, a sum over n terms in any order is within n 2^-24 of the sum of the terms'
magnitudes (S) of the exact one.  gate and up are that, rounded once to fp16 (u = 2^-11).  h: act has a slope below 1.13 everywhere, its
fp32 evaluation is within 2^-20 of max(1, |z|) (the error function's approximation is the largest part, 1.5e-7 |z| / 2), so
|dh| <= 1.13 e_G |U| + |act(G)| e_U + e_G e_U + 2^-20 max(1, |G|) |U| + u |h|, e the sums' bounds.  The backward pass starts from the gate and up that
were kept: dgate and dup are pointwise, within 2^-19 max(1, |z|)^2 of the factors' magnitudes and one rounding.  dx is a sum over both products of
the rounded dgate and dup (its reference takes those), within 2 ffn 2^-24 S, and one rounding.  The smallest fp16 step, 2^-24, is granted once.
"""
import math

import pytest
import torch

import paper_2302_05045_amd as samo
from gpu_util import DEV

pytestmark = pytest.mark.gpu
U = 2.0 ** -11
TINY = 2.0 ** -24

ACTS = {
    "silu": lambda z: z * torch.sigmoid(z),
    "gelu": lambda z: 0.5 * z * torch.erfc(-z / math.sqrt(2.0)),
    "gelu_tanh": lambda z: z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)),
    "relu": torch.relu,
}


def rnd(gen, *shape, std=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * std).half()


def make(tokens, features, ffn, seed, pruned=0.0, std=1.0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    x = rnd(gen, tokens, features, std=std)
    w = [rnd(gen, ffn, features, std=1.5 / math.sqrt(features * (1 - pruned))) * (torch.rand((ffn, features), generator=gen, device=DEV) >= pruned)
         for _ in range(2)]
    return gen, x, w[0], w[1]


def nan16(*shape):
    return torch.full(shape, float("nan"), device=DEV).half()


def within(got, want, bound, what):
    d = (got.double() - want).abs()
    assert torch.all(d <= bound + TINY), (what, float((d - bound).max()))


def check_forward(x, wg, wu, h, gate, up, act):
    z, v = x.double() @ wg.double().T, x.double() @ wu.double().T
    eps = (x.shape[1] + 2) * 2.0 ** -24
    ez, ev = eps * (x.double().abs() @ wg.double().abs().T), eps * (x.double().abs() @ wu.double().abs().T)
    a = ACTS[act](z)
    want = a * v
    within(h, want, 1.13 * ez * v.abs() + a.abs() * ev + ez * ev + 2.0 ** -20 * z.abs().clamp(min=1) * v.abs() + U * want.abs(), "h")
    if gate is not None:
        within(gate, z, ez + U * z.abs(), "gate")
        within(up, v, ev + U * v.abs(), "up")


def check_backward(dh, gate, up, wg, wu, dgate, dup, dx, act):
    z = gate.double().requires_grad_(True)
    a = ACTS[act](z)
    slope = torch.autograd.grad(a.sum(), z)[0]
    a, z = a.detach(), z.detach()
    dz, dv = dh.double() * up.double() * slope, dh.double() * a
    size = z.abs().clamp(min=1) ** 2 * 2.0 ** -19
    within(dgate, dz, size * (dh.double() * up.double()).abs() + U * dz.abs(), "dgate")
    within(dup, dv, size * dh.double().abs() + U * dv.abs(), "dup")
    if dx is not None:
        g, u = dgate.double(), dup.double()
        want = g @ wg.double() + u @ wu.double()
        magnitude = g.abs() @ wg.double().abs() + u.abs() @ wu.double().abs()
        within(dx, want, (2 * wg.shape[0] + 2) * 2.0 ** -24 * magnitude + U * want.abs(), "dx")


def run(tokens, features, ffn, act, seed=0, pruned=0.0, workspace=None, keep=True):
    gen, x, wg, wu = make(tokens, features, ffn, seed, pruned)
    h, gate, up = nan16(tokens, ffn), nan16(tokens, ffn), nan16(tokens, ffn)
    samo.samo_glu(x, wg, wu, h, gate, up, act)
    check_forward(x, wg, wu, h, gate, up, act)
    alone = nan16(tokens, ffn)
    samo.samo_glu(x, wg, wu, alone, act=act)
    assert torch.equal(alone, h)
    dh = rnd(gen, tokens, ffn)
    dgate, dup, dx = nan16(tokens, ffn), nan16(tokens, ffn), nan16(tokens, features)
    samo.samo_glu_backward(dh, gate, up, wg, wu, dgate, dup, dx, act, workspace=workspace)
    check_backward(dh, gate, up, wg, wu, dgate, dup, dx, act)
    return x, wg, wu, dh, gate, up, dgate, dup, dx


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("tokens", [1, 2, 16, 17, 32, 33, 127, 129, 257, 600])
def test_tokens_and_activations(tokens, act):
    run(tokens, 264, 520, act, seed=tokens, pruned=0.9)


@pytest.mark.parametrize("features,ffn", [(8, 8), (16, 24), (24, 1000), (64, 64), (72, 136), (1000, 40), (2056, 328), (256, 512), (520, 1288)])
@pytest.mark.parametrize("tokens", [3, 40, 300])
def test_sizes_that_fill_no_tile(features, ffn, tokens):
    run(tokens, features, ffn, "silu", seed=features + ffn)


@pytest.mark.parametrize("shape", [0, 1, 2, 3])
@pytest.mark.parametrize("tokens,features,ffn", [(513, 520, 264), (130, 32, 1032), (256, 96, 128), (700, 1096, 72)])
def test_every_tile_shape(shape, tokens, features, ffn):
    samo.samo_debug_set(samo.KNOB_GLU_SHAPE, shape)
    try:
        run(tokens, features, ffn, "gelu", seed=shape)
    finally:
        samo.samo_debug_set(samo.KNOB_GLU_SHAPE)


@pytest.mark.parametrize("shape", [0, 1, 2])
@pytest.mark.parametrize("splits", [1, 2, 3, 7, 16])
def test_split_sums(shape, splits):
    """Parts that end inside either product, at the border of the two, and a last one shorter than the others."""
    samo.samo_debug_set(samo.KNOB_GLU_SHAPE, shape)
    samo.samo_debug_set(samo.KNOB_GLU_SPLIT, splits)
    try:
        tokens, features, ffn = 150, 264, 1096
        need = samo.samo_glu_workspace_bytes(tokens, features, ffn)
        parts = need // (4 * tokens * features)                 # at most what was asked for: none may be empty or hold less than four stages
        assert need == 4 * tokens * features * parts and (parts == 0 if splits == 1 else 2 <= parts <= splits)
        ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device=DEV)
        run(tokens, features, ffn, "silu", workspace=ws)
        run(tokens, features, ffn, "silu", workspace=torch.empty(0, dtype=torch.uint8, device=DEV))      # none: unsplit
    finally:
        samo.samo_debug_set(samo.KNOB_GLU_SHAPE)
        samo.samo_debug_set(samo.KNOB_GLU_SPLIT)


def test_large_layers_agree_with_the_library_product():
    run(2048, 1024, 2736, "silu", pruned=0.9)
    run(1003, 2560, 1368, "gelu_tanh")


def test_without_dx():
    x, wg, wu, dh, gate, up, dgate, dup, dx = run(70, 128, 256, "silu")
    a, b = nan16(70, 256), nan16(70, 256)
    samo.samo_glu_backward(dh, gate, up, wg, wu, a, b, None, "silu")
    assert torch.equal(a, dgate) and torch.equal(b, dup)


def test_gradients_against_differences():
    """sum(h * dh) along a random direction of x, by central differences in 64 bits of the definition at the fp16 inputs: the gradient
    of the kernels is off by its roundings alone (2^-11 of the terms, as a random sum, 6 deviations) and the differences' third order."""
    gen, x, wg, wu = make(64, 128, 192, 5)
    h, gate, up = nan16(64, 192), nan16(64, 192), nan16(64, 192)
    samo.samo_glu(x, wg, wu, h, gate, up, "gelu_tanh")
    dh = rnd(gen, 64, 192)
    dgate, dup, dx = nan16(64, 192), nan16(64, 192), nan16(64, 128)
    samo.samo_glu_backward(dh, gate, up, wg, wu, dgate, dup, dx, "gelu_tanh")
    way = torch.randn((64, 128), generator=gen, device=DEV, dtype=torch.float64)
    f = lambda t: (ACTS["gelu_tanh"](t @ wg.double().T) * (t @ wu.double().T) * dh.double()).sum()
    eps = 1e-4
    slope = float((f(x.double() + eps * way) - f(x.double() - eps * way)) / (2 * eps))
    got = float((dx.double() * way).sum())
    terms = float((dx.double() * way).norm()) + float(((dgate.double().abs() @ wg.double().abs() + dup.double().abs() @ wu.double().abs()) * way).norm())
    assert abs(slope - got) <= 6 * 2 * U * terms + 1e-6 * abs(slope)


def test_weight_gradients_come_from_the_compressed_weight_gradient():
    """dgate and dup are the dY of samo_wgrad_gather_batched: the whole backward pass of the block's pruned matrices."""
    tokens, features, ffn = 300, 256, 512
    x, wg, wu, dh, gate, up, dgate, dup, dx = run(tokens, features, ffn, "silu", pruned=0.9)
    jobs, wants = [], []
    for w, d in ((wg, dgate), (wu, dup)):
        index = samo.samo_build_index((w.view(-1) != 0).to(torch.uint8))
        jobs.append((d, x, index.idx, index.seg_ptr, torch.empty(index.nnz, device=DEV)))
        dw = d.double().T @ x.double()
        wants.append((dw.view(-1)[index.idx.long()], (d.double().abs().T @ x.double().abs()).view(-1)[index.idx.long()]))
    samo.samo_wgrad_gather_batched(jobs, 1.0)
    for (_, _, _, _, gc), (want, size) in zip(jobs, wants):
        within(gc, want, tokens * 2.0 ** -23 * size + U * want.abs(), "dW")


def test_values_at_the_ends_of_fp16():
    """Pre-activations of thousands, an infinite one and a NaN keep to their rows."""
    gen, x, wg, wu = make(40, 64, 128, 3)
    x[1] *= 100
    x[2, 5] = float("inf")
    x[3, 7] = float("nan")
    for act in ACTS:
        h = nan16(40, 128)
        samo.samo_glu(x, wg, wu, h, act=act)
        assert torch.all(torch.isnan(h[3])) and torch.all(torch.isfinite(h[[0] + list(range(4, 40))]))
        check_forward(x[4:], wg, wu, h[4:], None, None, act)
        z, v = x[1].double() @ wg.double().T, x[1].double() @ wu.double().T
        want = (ACTS[act](z) * v).half()
        same = torch.isfinite(want) & (want.abs() > 1e-3)
        assert torch.all(((h[1].double() - want.double()).abs() <= 1e-2 * want.double().abs())[same])


def test_same_bits_again_other_stream_and_graph():
    gen, x, wg, wu = make(200, 520, 648, 9, 0.9)
    dh = rnd(gen, 200, 648)
    bufs = lambda: [torch.zeros(200, 648, device=DEV).half() for _ in range(5)] + [torch.zeros(200, 520, device=DEV).half()]

    def call(h, gate, up, dgate, dup, dx):
        samo.samo_glu(x, wg, wu, h, gate, up)
        samo.samo_glu_backward(dh, gate, up, wg, wu, dgate, dup, dx)

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


def exact_sums(tokens, features, ffn, seed):
    """Inputs whose sums are multiples of 2^-9 below 2^10, exact in fp32 in every order, and features whose gate is 2^-26, -2^-26 and 0 exactly."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    whole = lambda *s: torch.randint(-32, 33, s, generator=gen, device=DEV).float()
    x = whole(tokens, features) / 8
    wg, wu = (whole(ffn, features) / 64 * (torch.rand((ffn, features), generator=gen, device=DEV) < 0.1) for _ in range(2))
    x[:, -1], wg[:, -1], wu[:, -1] = 2.0 ** -13, 0.0, 0.0
    for first, small in ((1, 2.0 ** -13), (2, -2.0 ** -13), (3, 0.0)):
        wg[first::4] = 0.0
        wg[first::4, -1] = small
    return gen, x.half(), wg.half(), wu.half()


@pytest.mark.parametrize("tokens,shape", [(5, None), (20, None), (40, None), (300, 0), (300, 1), (300, 2), (300, 3)])
def test_relu_gradients_from_the_inputs(tokens, shape):
    """relu's slope jumps at zero: the gradients against those of X, Wg, Wu and dh in 64 bits, with gates as small as 2^-26.  up is rounded once, dgate
    once more: 2.01 u of the result.  A gate is kept within 2^-24, fp16's smallest number, which dup sees times dh."""
    features, ffn = 264, 520
    gen, x, wg, wu = exact_sums(tokens, features, ffn, tokens)
    dh = rnd(gen, tokens, ffn)
    h, gate, up, dgate, dup, dx = (nan16(tokens, n) for n in (ffn, ffn, ffn, ffn, ffn, features))
    if shape is not None:
        samo.samo_debug_set(samo.KNOB_GLU_SHAPE, shape)
    try:
        samo.samo_glu(x, wg, wu, h, gate, up, "relu")
        samo.samo_glu_backward(dh, gate, up, wg, wu, dgate, dup, dx, "relu")
    finally:
        samo.samo_debug_set(samo.KNOB_GLU_SHAPE)
    check_forward(x, wg, wu, h, gate, up, "relu")
    z, v, d = x.double() @ wg.double().T, x.double() @ wu.double().T, dh.double()
    assert torch.all(z[:, 1::4] == 2.0 ** -26) and torch.all(z[:, 2::4] == -2.0 ** -26) and torch.all(z[:, 3::4] == 0)
    dz, dv = d * v * (z > 0), d * torch.relu(z)
    within(dgate, dz, 2.01 * U * dz.abs(), "dgate")
    within(dup, dv, 2.01 * U * dv.abs() + TINY * d.abs(), "dup")
    want = dz @ wg.double() + dv @ wu.double()
    terms = dz.abs() @ wg.double().abs() + dv.abs() @ wu.double().abs()
    least = TINY * (wg.double().abs().sum(0) + (1 + d.abs()) @ wu.double().abs())
    within(dx, want, (2.01 * U + (2 * ffn + 2) * 2.0 ** -24) * terms + least + U * want.abs(), "dx")


@pytest.mark.parametrize("act", list(ACTS))
def test_gates_beyond_fp16_have_the_limits_of_the_slope(act):
    """Sums of 70000 and -70000 are kept as infinities.  The slope there is 1 and 0, act(-70000) is 0: a gradient is finite wherever it does not contain act(70000)."""
    tokens, features, ffn = 40, 64, 128
    gen, x, wg, wu = make(tokens, features, ffn, 12)
    x[:, :3] = 0
    wg[:, :3], wu[:, :3] = 0, 0
    wg[0::2, 0], wg[1::2, 0], wu[:, 1], wg[:, 2] = 200.0, -200.0, torch.linspace(-0.75, 0.75, ffn, device=DEV).half(), -200.0
    x[1], x[2] = 0, 0
    x[1, 0], x[1, 1] = 350.0, 1.0                            # both signs in turn
    x[2, 2], x[2, 1] = 350.0, 1.0                            # -70000 everywhere
    dh = rnd(gen, tokens, ffn)
    dh[dh == 0] = 1
    h, gate, up, dgate, dup, dx = (nan16(tokens, n) for n in (ffn, ffn, ffn, ffn, ffn, features))
    samo.samo_glu(x, wg, wu, h, gate, up, act)
    check_forward(x, wg, wu, h, None, None, act)
    assert torch.all(torch.isposinf(gate[1, 0::2])) and torch.all(torch.isneginf(gate[1, 1::2])) and torch.all(torch.isneginf(gate[2]))
    samo.samo_glu_backward(dh, gate, up, wg, wu, dgate, dup, dx, act)
    want = dh[1].double() * up[1].double()
    want[1::2] = 0
    within(dgate[1], want, 1.01 * U * want.abs(), "dgate")
    assert torch.equal(dup[1, 0::2], torch.copysign(torch.full_like(dh[1, 0::2], math.inf), dh[1, 0::2])) and torch.all(dup[1, 1::2] == 0)
    assert torch.all(dgate[2] == 0) and torch.all(dup[2] == 0) and torch.all(dx[2] == 0)
    rest = [0] + list(range(3, tokens))
    check_backward(dh[rest], gate[rest], up[rest], wg, wu, dgate[rest], dup[rest], dx[rest], act)


@pytest.mark.parametrize("act", list(ACTS))
def test_a_gate_that_is_no_number_stays_one(act):
    gen, x, wg, wu = make(40, 64, 128, 13)
    gate, up, dh = (rnd(gen, 40, 128) for _ in range(3))
    gate[3, 5] = float("nan")
    dgate, dup = nan16(40, 128), nan16(40, 128)
    samo.samo_glu_backward(dh, gate, up, wg, wu, dgate, dup, None, act)
    hit = torch.isnan(gate)
    assert torch.equal(torch.isnan(dup), hit) and torch.all(torch.isfinite(dgate[~hit])) and (act == "relu" or torch.isnan(dgate[3, 5]))
