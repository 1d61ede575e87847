"""Refusals of the norms around a block on the host, before anything is launched, and the size of their workspace."""
import ctypes

import pytest

import paper_2302_05045_amd as samo
from test_operators_cpu import ALIGN, ARG, FAKE, NULL, OK, SIZE, WORKSPACE

POINTERS = [name for name, kind in samo.NormDesc._fields_ if name.startswith("d_")]


def norm(**kw):
    """Every pointer its own: results may not be one another."""
    d = samo.NormDesc()
    d.tokens, d.hidden, d.kind, d.y_norm, d.eps, d.scale = 10, 64, 0, 1, 1e-5, 1.0
    for i, name in enumerate(POINTERS):
        setattr(d, name, FAKE * (1 + i))
    for name, value in kw.items():
        setattr(d, name, value)
    return d


@pytest.mark.parametrize("kw,want", [
    (dict(tokens=-1), SIZE), (dict(tokens=2 ** 31), SIZE), (dict(hidden=0), SIZE), (dict(hidden=12), SIZE), (dict(hidden=16392), SIZE), (dict(hidden=-8), SIZE),
    (dict(kind=2), ARG), (dict(kind=-1), ARG), (dict(eps=0.0), ARG), (dict(eps=2.0 ** -127), ARG), (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG),
    (dict(scale=float("nan")), ARG),
])
def test_norm_refuses(kw, want):
    L, need = samo.lib(), ctypes.c_size_t(7)
    assert L.samo_norm(ctypes.byref(norm(**kw)), None) == want
    assert L.samo_norm_backward(ctypes.byref(norm(**kw)), FAKE, 1 << 40, None) == want
    assert L.samo_norm_workspace_bytes(ctypes.byref(norm(**kw)), ctypes.byref(need)) == want and need.value == 7


def test_norm_refuses_pointers():
    L = samo.lib()
    forward = lambda **kw: L.samo_norm(ctypes.byref(norm(**kw)), None)
    back = lambda room=1 << 40, at=FAKE, **kw: L.samo_norm_backward(ctypes.byref(norm(**kw)), at, room, None)
    for name in POINTERS:
        assert back(**{name: FAKE + 8}) == ALIGN, name
        if POINTERS.index(name) < POINTERS.index("d_dout"):
            assert forward(**{name: FAKE + 4}) == ALIGN, name
    for name in ("d_stream", "d_out", "d_new_stream"):
        assert forward(**{name: None}) == NULL, name
    for name in ("d_dout", "d_new_stream", "d_stats", "d_dstream", "d_dy"):
        assert back(**{name: None}) == NULL, name
    assert forward(d_out=FAKE, d_new_stream=FAKE) == ARG and back(d_dy=FAKE, d_dstream=FAKE) == ARG
    # gradients of what is not there
    assert back(y_norm=0) == ARG
    assert back(d_y=None, d_dy_weight=None, d_dy_bias=None, d_dgate=None) == ARG and back(d_y=None, d_dy_weight=None, d_dy_bias=None, d_dy=None) == ARG
    assert back(at=FAKE + 8) == ALIGN and back(room=0) == WORKSPACE and back(at=None) == WORKSPACE
    assert L.samo_norm(None, None) == NULL and L.samo_norm_backward(None, FAKE, 1 << 20, None) == NULL
    assert L.samo_norm_workspace_bytes(ctypes.byref(norm()), None) == NULL
    # nothing to do: no launch, so it needs no device
    assert forward(tokens=0, d_stream=None, d_out=None, d_new_stream=None) == OK
    none = {n: None for n in ("d_dweight", "d_dbias", "d_dy_weight", "d_dy_bias", "d_dgate")}
    assert back(tokens=0, at=None, room=0, d_dout=None, **none) == OK


def test_norm_workspace():
    """A row of fp32 for each workgroup and sum that the wanted vectors need, at most one workgroup a token."""
    L, need = samo.lib(), ctypes.c_size_t()
    none = {n: None for n in ("d_dweight", "d_dbias", "d_dy_weight", "d_dy_bias", "d_dgate")}

    def ask(**kw):
        assert L.samo_norm_workspace_bytes(ctypes.byref(norm(**dict(none, **kw))), ctypes.byref(need)) == OK
        return need.value

    row = 4 * 64 * 10
    assert ask() == 0 and ask(d_dweight=FAKE) == row and ask(d_dweight=FAKE, d_dbias=FAKE) == 2 * row
    assert ask(d_dgate=FAKE, d_y_bias=None) == row and ask(d_dgate=FAKE) == 2 * row       # y's bias takes the sum of D besides
    assert ask(d_dgate=FAKE, d_dy_weight=FAKE, d_dy_bias=FAKE, d_dweight=FAKE, d_dbias=FAKE) == 4 * row
    assert ask(d_dgate=FAKE, y_norm=0) == row and ask(d_dweight=FAKE, tokens=0) == 0
    assert ask(d_dweight=FAKE, tokens=1 << 20) <= 4 * 64 * 4096


@pytest.mark.parametrize("y_norm", [0, 1])
def test_no_tokens_refuse_no_gradient_of_the_block(y_norm):
    """Tensors of no elements have no address: a block's output that is empty is not one that is missing, and no workspace is needed."""
    L, need = samo.lib(), ctypes.c_size_t()
    vectors = ["d_dweight", "d_dbias", "d_dgate", "d_dy_weight", "d_dy_bias"]
    none = {n: None for n in ["d_stream", "d_y", "d_new_stream", "d_out", "d_stats", "d_dout", "d_dnew", "d_dstream", "d_dy"] + vectors}

    def ask(wanted):
        need.value = 7
        kw = dict(none, **{n: FAKE * (50 + i) for i, n in enumerate(wanted)})
        return L.samo_norm_workspace_bytes(ctypes.byref(norm(tokens=0, y_norm=y_norm, **kw)), ctypes.byref(need))

    there = vectors if y_norm else vectors[:3]
    for wanted in [[n] for n in there] + [there]:
        assert ask(wanted) == OK and need.value == 0, wanted
    for name in () if y_norm else vectors[3:]:               # there is no norm behind the block, with tokens or without
        assert ask([name]) == ARG and need.value == 7, name
