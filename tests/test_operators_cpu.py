"""Refusals of the attention, feed-forward and 8-bit state entries on the host, before anything is launched, and what the generated code
of the kernels with LDS copies has to hold."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import paper_2302_05045_amd as samo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # non-null, 16-byte aligned; never dereferenced on these paths
OK, NULL, SIZE, ARG = samo.SAMO_OK, samo.SAMO_ERR_NULL, samo.SAMO_ERR_SIZE, samo.SAMO_ERR_ARG
WORKSPACE, ALIGN, PLAN = samo.SAMO_ERR_WORKSPACE, samo.SAMO_ERR_ALIGN, samo.SAMO_ERR_PLAN


def attention(**kw):
    d = samo.AttentionDesc()
    view = lambda: samo.Heads(FAKE, 64 * 4, 64)
    for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        setattr(d, name, view())
    d.d_lse, d.q_tokens, d.k_tokens, d.batch, d.heads, d.kv_heads, d.dim = FAKE, 10, 10, 1, 4, 2, 64
    d.max_q, d.max_k, d.scale, d.causal, d.window = 10, 10, 0.125, 1, 0
    for name, value in kw.items():
        setattr(d, name, value)
    return d


@pytest.mark.parametrize("kw,want", [
    (dict(heads=3), SIZE), (dict(heads=0), SIZE), (dict(kv_heads=0), SIZE), (dict(dim=0), SIZE), (dict(dim=12), SIZE), (dict(dim=136), SIZE),
    (dict(batch=0), SIZE), (dict(q_tokens=-1), SIZE), (dict(k_tokens=2 ** 31), SIZE), (dict(max_q=11), SIZE), (dict(max_k=-1), SIZE),
    (dict(batch=2), ARG), (dict(d_q_start=FAKE), ARG), (dict(d_k_start=FAKE), ARG), (dict(scale=0.0), ARG), (dict(scale=float("nan")), ARG),
    (dict(scale=-1.0), ARG), (dict(scale=float("inf")), ARG), (dict(window=-1), ARG), (dict(window=5, causal=0), ARG), (dict(d_lse=None), NULL),
    (dict(d_lse=FAKE + 2), ALIGN), (dict(q=samo.Heads(None, 256, 64)), NULL), (dict(k=samo.Heads(FAKE + 8, 256, 64)), ALIGN),
    (dict(v=samo.Heads(FAKE, 252, 64)), SIZE), (dict(out=samo.Heads(FAKE, 256, 60)), SIZE), (dict(q=samo.Heads(FAKE, -256, 64)), SIZE),
    (dict(d_q_start=FAKE + 1, d_k_start=FAKE), ALIGN),
    (dict(q_tokens=2 ** 31 - 1, max_q=2 ** 31 - 1, batch=1, heads=512, kv_heads=1), SIZE),
])
def test_attention_refuses(kw, want):
    L = samo.lib()
    assert L.samo_attention(ctypes.byref(attention(**kw)), None) == want
    assert L.samo_attention_backward(ctypes.byref(attention(**kw)), FAKE, 1 << 20, None) == want


def test_attention_backward_refuses():
    L = samo.lib()
    for name in ("dout", "dq", "dk", "dv"):
        assert L.samo_attention_backward(ctypes.byref(attention(**{name: samo.Heads(None, 256, 64)})), FAKE, 1 << 20, None) == NULL
    assert L.samo_attention_backward(ctypes.byref(attention()), None, 0, None) == WORKSPACE
    assert L.samo_attention_backward(ctypes.byref(attention()), FAKE, 4 * 4 * 10 - 1, None) == WORKSPACE
    assert L.samo_attention_backward(ctypes.byref(attention()), FAKE + 4, 1 << 20, None) == ALIGN
    assert L.samo_attention(None, None) == NULL and L.samo_attention_backward(None, FAKE, 16, None) == NULL
    need = ctypes.c_size_t()
    assert L.samo_attention_workspace_bytes(ctypes.byref(attention()), ctypes.byref(need)) == OK and need.value == 160
    assert L.samo_attention_workspace_bytes(None, ctypes.byref(need)) == NULL
    assert L.samo_attention_workspace_bytes(ctypes.byref(attention()), None) == NULL
    # nothing to do: no launch, so it needs no device
    empty = attention(q_tokens=0, k_tokens=0, max_q=0, max_k=0, d_lse=None, **{n: samo.Heads(None, 0, 0) for n in ("q", "k", "v", "out")})
    assert L.samo_attention(ctypes.byref(empty), None) == OK


def test_glu_refuses():
    L = samo.lib()
    good = dict(x=FAKE, wg=FAKE, wu=FAKE, tokens=4, fin=16, ffn=32, act=0, h=FAKE, gate=None, up=None)

    def call(**kw):
        a = dict(good, **kw)
        return L.samo_glu(a["x"], a["wg"], a["wu"], a["tokens"], a["fin"], a["ffn"], a["act"], a["h"], a["gate"], a["up"], None)

    for kw, want in ((dict(tokens=-1), SIZE), (dict(fin=12), SIZE), (dict(fin=0), SIZE), (dict(ffn=4), SIZE), (dict(ffn=1 << 20), SIZE),
                     (dict(act=4), ARG), (dict(act=-1), ARG), (dict(x=None), NULL), (dict(wg=None), NULL), (dict(wu=None), NULL), (dict(h=None), NULL),
                     (dict(gate=FAKE), NULL), (dict(up=FAKE), NULL), (dict(x=FAKE + 2), ALIGN), (dict(h=FAKE + 8), ALIGN),
                     (dict(tokens=2 ** 31 - 1, ffn=(1 << 20) - 8), SIZE), (dict(tokens=0, x=None), OK)):
        assert call(**kw) == want, kw

    def back(**kw):
        a = dict(dh=FAKE, gate=FAKE, up=FAKE, wg=FAKE, wu=FAKE, tokens=4, fin=16, ffn=32, act=0, dgate=FAKE, dup=FAKE, dx=FAKE, ws=None)
        a.update(kw)
        return L.samo_glu_backward(a["dh"], a["gate"], a["up"], a["wg"], a["wu"], a["tokens"], a["fin"], a["ffn"], a["act"], a["dgate"],
                                   a["dup"], a["dx"], a["ws"], 0, None)

    for name in ("dh", "gate", "up", "wg", "wu", "dgate", "dup"):
        assert back(**{name: None}) == NULL, name
        assert back(**{name: FAKE + 4}) == ALIGN, name
    assert back(fin=9) == SIZE and back(act=7) == ARG and back(ws=FAKE + 8) == ALIGN and back(tokens=0, dh=None) == OK
    need = ctypes.c_size_t()
    assert L.samo_glu_workspace_bytes(4, 16, 32, None) == NULL and L.samo_glu_workspace_bytes(4, 15, 32, ctypes.byref(need)) == SIZE
    assert L.samo_glu_workspace_bytes(0, 16, 32, ctypes.byref(need)) == OK and need.value == 0


def layer8(**kw):
    d = samo.Layer8Desc(8, 4, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0, 0)
    for name, value in kw.items():
        setattr(d, name, value)
    return d


def test_step8_refuses():
    L = samo.lib()
    cfg = samo.adam_cfg(1)

    def call(source=0, scale=1.0, cfg=cfg, **kw):
        return L.samo_step8(ctypes.byref(layer8(**kw)), source, scale, None if cfg is None else ctypes.byref(cfg), 1, None)

    for kw, want in ((dict(n=-1), SIZE), (dict(nnz=9), SIZE), (dict(n=2 ** 31), SIZE), (dict(idx=None), NULL), (dict(seg_ptr=None), NULL),
                     (dict(idx=None, seg_ptr=None), SIZE), (dict(s8=None), NULL), (dict(q8=None), NULL), (dict(p=None), NULL), (dict(w=None), NULL),
                     (dict(g=None), NULL), (dict(source=1, gc16=None), NULL), (dict(q8=FAKE + 2), ALIGN), (dict(s8=FAKE + 1), ALIGN),
                     (dict(p=FAKE + 4), ALIGN), (dict(source=2), ARG), (dict(scale=0.0), ARG), (dict(cfg=None), NULL),
                     (dict(cfg=samo.adam_cfg(0)), ARG), (dict(cfg=samo.adam_cfg(1, eps=0.0)), ARG)):
        assert call(**kw) == want, kw
    assert L.samo_step8(None, 0, 1.0, ctypes.byref(cfg), 1, None) == NULL
    assert L.samo_step8_batched(None, 0, 1.0, ctypes.byref(cfg), 1, None, None) == NULL
    for entry in (L.samo_state8_pack, L.samo_state8_unpack):
        assert entry(None, None) == NULL and entry(ctypes.byref(layer8(m=None)), None) == NULL and entry(ctypes.byref(layer8(v=None)), None) == NULL
    plan = samo.Plan8Desc()                                         # a plan of nothing lacks every buffer
    assert L.samo_step8_batched(ctypes.byref(plan), 0, 1.0, ctypes.byref(cfg), 1, None, None) == PLAN
    assert L.samo_state8_unpack_batched(ctypes.byref(plan), None) == PLAN and L.samo_state8_pack_batched(None, None) == NULL


def test_plan8_sizes_and_refusals():
    """Descriptors of 104 bytes padded to 256, one 8-byte record for every four segments of a layer (16 of a large model's pruned layers)."""
    L = samo.lib()
    need, plan = ctypes.c_size_t(), samo.Plan8Desc()
    layers = (samo.Layer8Desc * 2)(layer8(n=5000, nnz=100), layer8(n=9000, nnz=9000, idx=None, seg_ptr=None))
    assert ctypes.sizeof(samo.Layer8Desc) == 104
    assert L.samo_plan8_workspace_bytes(layers, 2, ctypes.byref(need)) == OK and need.value == 256 + 8 * (2 + 3)
    layers[0].n = 2 ** 31 - 1
    assert L.samo_plan8_workspace_bytes(layers, 2, ctypes.byref(need)) == OK and need.value == 256 + 8 * (2 ** 21 // 16 + 3)
    assert L.samo_plan8_workspace_bytes(layers, -1, ctypes.byref(need)) == SIZE
    assert L.samo_plan8_workspace_bytes(None, 1, ctypes.byref(need)) == NULL and L.samo_plan8_workspace_bytes(layers, 1, None) == NULL
    layers[0].n = 5000
    assert L.samo_plan8_init(layers, 2, FAKE, 16, None, ctypes.byref(plan)) == WORKSPACE
    assert L.samo_plan8_init(layers, 2, None, 1 << 20, None, ctypes.byref(plan)) == WORKSPACE
    assert L.samo_plan8_init(layers, 2, FAKE + 8, 1 << 20, None, ctypes.byref(plan)) == ALIGN
    assert L.samo_plan8_init(layers, 2, FAKE, 1 << 20, None, None) == NULL
    layers[1].q8 = FAKE + 1
    assert L.samo_plan8_init(layers, 2, FAKE, 1 << 20, None, ctypes.byref(plan)) == ALIGN
    assert L.samo_plan8_init(layers, 0, None, 0, None, ctypes.byref(plan)) == OK


def test_binding_refuses_what_is_not_a_gpu_tensor():
    t = torch.zeros(4, 2, 64, dtype=torch.float16)
    with pytest.raises(TypeError):
        samo.samo_attention(t, t, t, t, torch.zeros(2, 4))
    with pytest.raises(TypeError):
        samo.samo_glu(t[0], t[0], t[0], t[0])
    with pytest.raises(ValueError):
        samo._act("tanh")
    with pytest.raises(TypeError):
        samo.samo_step8(samo.Layer8(8, None, None, torch.zeros(8), torch.zeros(16, dtype=torch.uint8), torch.zeros(2, dtype=torch.uint8)), 1.0,
                        samo.adam_cfg(1), 0)
    assert samo.samo_state8_scales_len(1025) == 4 and samo.samo_state8_scales_len(0) == 0


@pytest.mark.parametrize("source", ["attention.hip", "glu.hip"])
def test_m0_is_touched_only_by_the_copies_into_lds(tmp_path, source):
    """As in the weight gradient's kernels: the copies set M0 from inline assembly, which cannot declare it clobbered, so the compiler must not
    use it in these kernels.  Checked on the generated code of every build."""
    from paper_2302_05045_amd import _build
    asm = tmp_path / "out.s"
    subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + [f for f in _build.FLAGS if f not in ("-shared", "-fPIC")] +
                          ["-S", "--cuda-device-only", "-I", os.path.join(ROOT, "include"), "-I", _build.CSRC,
                           os.path.join(_build.CSRC, source), "-o", str(asm)], stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    lines = [ln.split(";")[0].strip() for ln in asm.read_text().splitlines()]
    code = [ln for ln in lines if ln and not ln.startswith(".") and not ln.endswith(":")]
    uses = [i for i, ln in enumerate(code) if re.search(r"\bm0\b", ln)]
    assert len(uses) >= 16
    for i in uses:
        assert re.fullmatch(r"s_mov_b32 m0, s\d+", code[i]), code[i]
        assert code[i + 1] == "s_nop 0" and re.match(r"global_load_lds_dword(x4)? ", code[i + 2]), code[i:i + 3]
    assert sum(ln.startswith("global_load_lds_") for ln in code) == len(uses)


def test_attention_memory_for_sums():
    """What calls can use beside their workspace: a query of NULL or of a refused descriptor, the sizes by the number of parts, misaligned memory."""
    L = samo.lib()
    need = ctypes.c_size_t(7)
    ask = lambda d, backward: L.samo_attention_sums_bytes(ctypes.byref(d), backward, ctypes.byref(need))
    assert L.samo_attention_sums_bytes(None, 0, ctypes.byref(need)) == NULL
    assert L.samo_attention_sums_bytes(ctypes.byref(attention()), 0, None) == NULL
    assert ask(attention(dim=12), 0) == SIZE and ask(attention(dq=samo.Heads(None, 256, 64)), 1) == NULL
    assert L.samo_attention(ctypes.byref(attention(d_sums=FAKE + 8, sums_bytes=1 << 20)), None) == ALIGN
    assert L.samo_attention_backward(ctypes.byref(attention(d_sums=FAKE + 4)), FAKE, 1 << 20, None) == ALIGN
    try:
        for parts in (1, 2, 16, 40):
            samo.samo_debug_set(samo.KNOB_ATTENTION_SPLIT, parts)
            slots = 0 if parts == 1 else min(parts, 16)       # of 128 rows, one tile of a head; more than 16 parts are 16
            assert ask(attention(), 0) == OK and need.value == 4 * slots * 128 * (4 * 64 + 8)
            assert ask(attention(), 1) == OK and need.value == slots * max(4 * 128 * 4 * 64, 2 * 2 * 128 * 4 * 64)
            assert ask(attention(dim=72), 0) == OK and need.value == 4 * slots * 128 * (4 * 96 + 8)
    finally:
        samo.samo_debug_set(samo.KNOB_ATTENTION_SPLIT)
    # a short call of this size has no use for any
    assert ask(attention(), 0) == OK and need.value == 0


def views_of(dim):
    return {name: samo.Heads(FAKE, 32 * dim, dim) for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")}


@pytest.mark.parametrize("kw,dkv_only", [
    (dict(batch=2 ** 19, heads=32, kv_heads=32, max_q=1), False),                              # 2^24 workgroups of 256 threads
    (dict(batch=512, heads=32, kv_heads=32, q_tokens=2 ** 18, k_tokens=2 ** 18, max_q=2 ** 18, max_k=2 ** 18), False),
    (dict(batch=2 ** 31 - 1, heads=2 ** 31 - 1, kv_heads=1, max_q=10), False),
    (dict(batch=2 ** 18, heads=32, kv_heads=32, dim=128, max_q=1, max_k=1), True),             # 2^23 of 512
    (dict(batch=2 ** 19, heads=32, kv_heads=32, max_q=0, max_k=1), True),
])
def test_attention_refuses_more_threads_than_a_launch_holds(kw, dkv_only):
    """A launch's threads are counted in 32 bits: refused before the first of the call's launches."""
    L = samo.lib()
    d = attention(d_q_start=FAKE, d_k_start=FAKE, **kw, **views_of(kw.get("dim", 64)))
    need = ctypes.c_size_t()
    room = 4 * d.heads * d.q_tokens
    assert L.samo_attention_backward(ctypes.byref(d), FAKE, room, None) == SIZE
    assert L.samo_attention_sums_bytes(ctypes.byref(d), 1, ctypes.byref(need)) == SIZE
    assert L.samo_attention_sums_bytes(ctypes.byref(d), 0, ctypes.byref(need)) == (OK if dkv_only else SIZE)
    if not dkv_only:
        assert L.samo_attention(ctypes.byref(d), None) == SIZE


@pytest.mark.parametrize("kw", [dict(batch=2 ** 19 - 1, heads=32, kv_heads=32, max_q=1, max_k=0), dict(batch=2 ** 19 - 1, heads=32, kv_heads=32, max_q=1, max_k=1),
                                dict(batch=2 ** 18 - 1, heads=32, kv_heads=32, dim=128, max_q=1, max_k=1)])
def test_attention_takes_what_a_launch_holds(kw):
    need = ctypes.c_size_t()
    for backward in (0, 1):
        assert samo.lib().samo_attention_sums_bytes(ctypes.byref(attention(d_q_start=FAKE, d_k_start=FAKE, **kw, **views_of(kw.get("dim", 64)))), backward, ctypes.byref(need)) == OK


@pytest.mark.parametrize("name", ["q_tokens", "k_tokens"])
def test_attention_refuses_tokens_whose_bounds_pass_32_bits(name):
    """Windows and masks are sums of two lengths and a window, which is 2^30 where there is none."""
    L = samo.lib()
    need = ctypes.c_size_t()
    for tokens, want in ((2 ** 30 - 127, SIZE), (2 ** 30, SIZE), (2 ** 31 - 1, SIZE), (2 ** 30 - 128, OK)):
        d = attention(**{name: tokens})
        assert L.samo_attention_sums_bytes(ctypes.byref(d), 0, ctypes.byref(need)) == want, tokens
        if want == SIZE:
            assert L.samo_attention(ctypes.byref(d), None) == SIZE and L.samo_attention_backward(ctypes.byref(d), FAKE, 1 << 40, None) == SIZE


@pytest.mark.parametrize("view", [samo.Heads(FAKE, 0, 64), samo.Heads(FAKE, 256, 0), samo.Heads(FAKE, 56, 640), samo.Heads(FAKE, 256, 56)])
def test_attention_refuses_results_that_overlap(view):
    """Rows or heads of a result less than dim apart are written by several workgroups; of what is only read they may be one and the same.  (max_q and
    max_k of 0: nothing is launched.)"""
    L = samo.lib()
    forward = lambda **kw: L.samo_attention(ctypes.byref(attention(**{**dict(max_q=0, max_k=0), **kw})), None)
    back = lambda **kw: L.samo_attention_backward(ctypes.byref(attention(**{**dict(max_q=0, max_k=0), **kw})), FAKE, 1 << 20, None)
    assert forward(out=view) == SIZE and all(back(**{name: view}) == SIZE for name in ("dq", "dk", "dv"))
    for name in ("q", "k", "v", "dq", "dk", "dv"):
        assert forward(**{name: view}) == OK, name
    for name in ("q", "k", "v", "dout", "out"):              # the backward pass reads out
        assert back(**{name: view}) == OK, name
    # strides of a dimension of one element are not looked at
    assert forward(out=samo.Heads(FAKE, 0, 64), q_tokens=1) == OK and forward(out=samo.Heads(FAKE, 64, 0), heads=1, kv_heads=1) == OK
    assert back(dk=samo.Heads(FAKE, 64, 0), kv_heads=1) == OK and back(dk=samo.Heads(FAKE, 0, 64), k_tokens=1) == OK


def test_glu_refuses_more_threads_than_a_launch_holds():
    L = samo.lib()
    forward = lambda tokens, fin, ffn: L.samo_glu(FAKE, FAKE, FAKE, tokens, fin, ffn, 0, FAKE, None, None, None)
    back = lambda tokens, fin, ffn: L.samo_glu_backward(FAKE, FAKE, FAKE, FAKE, FAKE, tokens, fin, ffn, 0, FAKE, FAKE, FAKE, None, 0, None)
    need = ctypes.c_size_t()
    assert forward(2 ** 27, 8, 2048) == SIZE                   # 2^19 by 16 tiles of 512 threads
    assert back(2 ** 24, 8, 2048) == SIZE                      # 2^35 elements, eight to a thread
    assert back(2 ** 27, 4096, 8) == SIZE and L.samo_glu_workspace_bytes(2 ** 27, 4096, 8, ctypes.byref(need)) == SIZE     # of dX: 2^19 by 16
    samo.samo_debug_set(samo.KNOB_GLU_SHAPE, 3)
    try:
        assert forward(2 ** 24, 8, 2048) == SIZE               # 2^17 by 64 tiles of 128 tokens x 32 features
    finally:
        samo.samo_debug_set(samo.KNOB_GLU_SHAPE)
    assert L.samo_glu_workspace_bytes(2 ** 24, 8, 2040, ctypes.byref(need)) == OK


def test_plan8_refuses_more_threads_than_a_launch_holds():
    """Unpruned layers have a workgroup of 256 threads for every four segments: 32 of the largest are 2^24."""
    L = samo.lib()
    need, plan = ctypes.c_size_t(), samo.Plan8Desc()
    n = 2 ** 31 - 1
    layers = (samo.Layer8Desc * 32)(*[layer8(n=n, nnz=n, idx=None, seg_ptr=None) for _ in range(32)])
    assert L.samo_plan8_workspace_bytes(layers, 31, ctypes.byref(need)) == OK
    assert L.samo_plan8_workspace_bytes(layers, 32, ctypes.byref(need)) == SIZE
    assert L.samo_plan8_init(layers, 32, FAKE, 1 << 40, None, ctypes.byref(plan)) == SIZE
