"""Refusals of attention with scores of another form on the host, before anything is launched, and the sizes of its workspaces."""
import concurrent.futures
import ctypes

import pytest
import torch

import paper_2302_05045_amd as samo
import test_operators_cpu
from test_operators_cpu import ALIGN, ARG, FAKE, NULL, OK, SIZE, WORKSPACE, attention


def scores(**kw):
    c = samo.ScoresDesc()
    c.cap, c.d_slopes, c.d_table, c.d_borders, c.buckets = 30.0, FAKE, FAKE, FAKE, 32
    for name, value in kw.items():
        setattr(c, name, value)
    return c


@pytest.mark.parametrize("kw,want", [
    (dict(cap=-1.0), ARG), (dict(cap=float("nan")), ARG), (dict(cap=float("inf")), ARG), (dict(cap=2.0 ** -11), ARG), (dict(cap=256.5), ARG),
    (dict(buckets=0), SIZE), (dict(buckets=65), SIZE), (dict(buckets=-3), SIZE), (dict(d_borders=None), NULL), (dict(d_slopes=FAKE + 2), ALIGN),
    (dict(d_borders=FAKE + 1), ALIGN), (dict(d_first_keys=FAKE + 2), ALIGN), (dict(d_table=FAKE + 1), ALIGN), (dict(d_dtable=FAKE + 1), ALIGN),
])
def test_scored_attention_refuses(kw, want):
    L = samo.lib()
    d, c, need = attention(), scores(**kw), ctypes.c_size_t(7)
    assert L.samo_attention_scored(ctypes.byref(d), ctypes.byref(c), None) == want
    assert L.samo_attention_scored_backward(ctypes.byref(d), ctypes.byref(c), FAKE, 1 << 20, None) == want
    assert L.samo_attention_scored_sums_bytes(ctypes.byref(d), ctypes.byref(c), 1, ctypes.byref(need)) == want
    assert L.samo_attention_scored_workspace_bytes(ctypes.byref(d), ctypes.byref(c), ctypes.byref(need)) == want and need.value == 7


def test_scored_attention_refuses_what_plain_attention_refuses():
    L = samo.lib()
    for kw, want in ((dict(dim=12), SIZE), (dict(heads=3), SIZE), (dict(scale=0.0), ARG), (dict(d_lse=None), NULL), (dict(q=samo.Heads(None, 256, 64)), NULL),
                     (dict(window=5, causal=0), ARG), (dict(d_sums=FAKE + 8), ALIGN)):
        assert L.samo_attention_scored(ctypes.byref(attention(**kw)), ctypes.byref(scores()), None) == want, kw
        assert L.samo_attention_scored_backward(ctypes.byref(attention(**kw)), ctypes.byref(scores()), FAKE, 1 << 20, None) == want, kw
    c, need = scores(), ctypes.c_size_t()
    assert L.samo_attention_scored(ctypes.byref(attention()), None, None) == NULL and L.samo_attention_scored(None, ctypes.byref(c), None) == NULL
    assert L.samo_attention_scored_backward(ctypes.byref(attention()), None, FAKE, 1 << 20, None) == NULL
    assert L.samo_attention_scored_sums_bytes(ctypes.byref(attention()), ctypes.byref(c), 0, None) == NULL
    assert L.samo_attention_scored_workspace_bytes(ctypes.byref(attention()), None, ctypes.byref(need)) == NULL
    # the first keys are those of a causal mask
    assert L.samo_attention_scored(ctypes.byref(attention(causal=0)), ctypes.byref(scores(d_first_keys=FAKE)), None) == ARG
    for scale in (2.0 ** -61, 2.0 ** 61):
        assert L.samo_attention_scored(ctypes.byref(attention(scale=scale)), ctypes.byref(c), None) == ARG
    # a table's gradient needs a table; results that overlap
    assert L.samo_attention_scored_backward(ctypes.byref(attention()), ctypes.byref(scores(d_table=None, d_dtable=FAKE)), FAKE, 1 << 20, None) == NULL
    assert L.samo_attention_scored(ctypes.byref(attention(out=samo.Heads(FAKE, 0, 64))), ctypes.byref(c), None) == SIZE
    assert L.samo_attention_scored_backward(ctypes.byref(attention(dk=samo.Heads(FAKE, 256, 0))), ctypes.byref(c), FAKE, 1 << 20, None) == SIZE
    # one bucket has no border, without a table nothing is asked of buckets and borders
    quiet = dict(max_q=0, max_k=0)
    for kw in (dict(buckets=1, d_borders=None), dict(d_table=None, d_borders=None, buckets=0), dict(cap=0.0, d_slopes=None)):
        assert L.samo_attention_scored(ctypes.byref(attention(**quiet)), ctypes.byref(scores(**kw)), None) == OK, kw


def test_scored_workspace():
    """delta, and behind it a float for every column, 128 queries of a head and part."""
    L, need = samo.lib(), ctypes.c_size_t()
    ask = lambda c, **kw: L.samo_attention_scored_workspace_bytes(ctypes.byref(attention(**kw)), ctypes.byref(c), ctypes.byref(need))
    assert ask(scores()) == OK and need.value == 4 * 4 * 10
    assert ask(scores(d_dtable=FAKE)) == OK and need.value == 160 + 4 * 4 * 32
    assert ask(scores(d_dtable=FAKE, two_sided=1), q_tokens=301, max_q=300) == OK and need.value == 4 * 4 * 301 + 4 * 3 * 4 * 64
    assert L.samo_attention_scored_backward(ctypes.byref(attention()), ctypes.byref(scores(d_dtable=FAKE)), FAKE, 160 + 4 * 4 * 32 - 1, None) == WORKSPACE
    assert L.samo_attention_scored_backward(ctypes.byref(attention()), ctypes.byref(scores()), None, 0, None) == WORKSPACE
    assert L.samo_attention_scored_backward(ctypes.byref(attention()), ctypes.byref(scores()), FAKE + 8, 1 << 20, None) == ALIGN
    try:
        samo.samo_debug_set(samo.KNOB_ATTENTION_SPLIT, 5)
        assert ask(scores(d_dtable=FAKE)) == OK and need.value == 160 + 4 * 4 * 5 * 32
    finally:
        samo.samo_debug_set(samo.KNOB_ATTENTION_SPLIT)


def test_bucket_borders():
    cpu = lambda b, f: samo.samo_bucket_borders(b, f, device="cpu")
    assert cpu(1, 0) is None and cpu(2, 5).tolist() == [1]
    assert cpu(32, 128).tolist() == list(range(1, 17)) + [19, 21, 24, 27, 31, 35, 40, 46, 52, 59, 67, 77, 87, 99, 113]
    assert cpu(16, 128).tolist() == [1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91]     # powers of 2 by halves: 8, 8 sqrt 2, 16 ...
    assert cpu(64, 2000).dtype == torch.int32 and cpu(64, 2000).numel() == 63
    for buckets, far in ((0, 10), (65, 100), (8, 4), (8, 3), (8, 2 ** 30)):
        with pytest.raises(ValueError):
            cpu(buckets, far)


FORMS = ["keys", "cap", "slope", "table", "cap_slope", "cap_table", "all"]


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """What became of each form's source, compiled side by side."""
    with concurrent.futures.ThreadPoolExecutor(4) as pool:
        check = test_operators_cpu.test_m0_is_touched_only_by_the_copies_into_lds
        yield {form: pool.submit(check, tmp_path_factory.mktemp(form), "attention_%s.hip" % form) for form in FORMS}


@pytest.mark.parametrize("form", FORMS)
def test_m0_is_touched_only_by_the_copies_into_lds_in_the_forms_kernels(compiled, form):
    compiled[form].result()


def test_a_table_of_too_many_heads_is_refused():
    """Its gradient takes a workgroup of 1024 threads a head; a launch's threads are counted in 32 bits."""
    L, need = samo.lib(), ctypes.c_size_t()
    for heads, want in ((2 ** 21, SIZE), (2 ** 21 - 8, OK)):
        d = attention(heads=heads, kv_heads=heads)
        assert L.samo_attention_scored_workspace_bytes(ctypes.byref(d), ctypes.byref(scores(d_dtable=FAKE)), ctypes.byref(need)) == want, heads
    assert L.samo_attention_scored_workspace_bytes(ctypes.byref(attention(heads=2 ** 21, kv_heads=2 ** 21)), ctypes.byref(scores()), ctypes.byref(need)) == OK
