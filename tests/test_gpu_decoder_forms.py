"""The norms and the forms of scores together, as the example's decoder uses them: its gradients against plain operations in fp32 under autograd, the same bits
from the same training, and tokens one at a time against the whole sequence."""
import os
import sys

import pytest
import torch

import paper_2302_05045_amd as samo

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def plain_loss(model, weights, tokens, targets, starts):
    """The decoder's loss by plain operations; weights: an fp32 leaf for each of model.weights."""
    of = dict(zip(map(id, model.weights), weights))
    norm = lambda x: x * (x.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    vectors = [iter(w for w in weights[len(weights) - (3 * len(model.norms) - 2):])]
    tables = weights[5 * len(model.blocks) + 1:]
    stream = model.embedding[tokens].float()
    x = norm(stream) * next(vectors[0])
    scale = (2 * len(model.blocks)) ** -0.5

    def around(stream, y):
        w, wy, gate = next(vectors[0]), next(vectors[0]), next(vectors[0])
        stream = stream + scale * gate * (norm(y) * wy)
        return stream, norm(stream) * w

    h, hk, d = model.heads, model.kv_heads, model.dim
    for n, b in enumerate(model.blocks):
        q, k, v = (x @ of[id(b["qkv"])].T).view(-1, h + 2 * hk, d).split([h, hk, hk], dim=1)
        outs = []
        for a, e in zip(starts, starts[1:]):
            ks, vs = k[a:e].repeat_interleave(h // hk, 1), v[a:e].repeat_interleave(h // hk, 1)
            s = torch.stack([q[a:e, i] @ ks[:, i].T for i in range(h)]) * d ** -0.5
            cap = model.scores[n].cap
            s = cap * torch.tanh(s / cap)
            far = torch.arange(e - a, device=s.device)[:, None] - torch.arange(e - a, device=s.device)[None, :]
            column = (far.clamp(min=0)[..., None] >= model.scores[n].borders).sum(-1)
            s = (s + tables[n][:, column]).masked_fill(far < 0, float("-inf"))
            p = torch.softmax(s, 2)
            outs.append(torch.stack([p[i] @ vs[:, i] for i in range(h)], 1))
        stream, x = around(stream, torch.cat(outs).flatten(1) @ of[id(b["proj"])].T)
        gate = x @ of[id(b["gate"])].T
        stream, x = around(stream, (gate * torch.sigmoid(gate) * (x @ of[id(b["up"])].T)) @ of[id(b["down"])].T)
    return torch.nn.functional.cross_entropy(x @ of[id(model.head)].T, targets)


def test_gradients_of_the_decoder():
    """Every weight's gradient.  An fp16 rounding takes a tensor 2^-11 off at most, in its own 2-norm; from the embedding to a gradient there are at most 12
    rounded tensors a layer forward and as many backward (norms, projections, q k v, P, out, G, U, h; their gradients): 48 roundings for two layers, of gain 1
    relative to the tensor they are added to."""
    import pruned_decoder
    model = pruned_decoder.Decoder(2, 128, 264, 4, 2, 32, 0.4, cap=5.0, buckets=16, sandwich=True, seed=3)
    gen = torch.Generator()
    gen.manual_seed(1)
    for norm, _ in model.norms:                              # away from ones, so that every vector matters
        for t in (norm.weight, norm.y_weight, norm.gate):
            if t is not None:
                t.add_(torch.randn(t.shape, generator=gen).to(t) * 0.2)
    for scores in model.scores:
        scores.table.add_(torch.randn(scores.table.shape, generator=gen).to(scores.table) * 0.5)
    tokens, targets, batch = pruned_decoder.packed_batch(5, 60, 32, gen)
    loss = model.gradients(tokens, targets, batch)
    leaves = [w.dense.float().requires_grad_() for w in model.weights]
    want = plain_loss(model, [t if t.shape[0] > 1 else t.view(-1) for t in leaves], tokens, targets, batch["starts"].tolist())
    assert abs(float(loss.detach()) - float(want.detach())) < 48 * 2.0 ** -11 * float(want.detach())
    grads = torch.autograd.grad(want, leaves)
    for n, (w, g) in enumerate(zip(model.weights, grads)):
        g = g.reshape(-1) if w.idx is None else g.reshape(-1)[w.idx.long()]
        off = float((w.gc16.double() / pruned_decoder.LOSS_SCALE - g.double()).norm() / g.double().norm())
        assert off < 48 * 2.0 ** -11, (n, tuple(w.dense.shape), off)


def test_training_and_generation_with_every_form():
    import pruned_decoder
    args = dict(layers=2, hidden=64, ffn=96, heads=4, kv_heads=2, vocab=24, steps=6, sequences=3, longest=40, window=17, cap=10.0, buckets=8, sandwich=True)
    runs = [pruned_decoder.train(**args) for _ in range(2)]
    assert runs[0][1] == runs[1][1] and all(x == x for x in runs[0][1])
    for a, b in zip(runs[0][0].weights, runs[1][0].weights):
        assert torch.equal(a.p, b.p) and torch.equal(a.q8, b.q8) and torch.equal(a.dense, b.dense)
    model = runs[0][0]
    assert all(float(t.abs().max()) > 0 for t in model.tables) and any(float((n.gate - 1).abs().max()) > 0 for n, _ in model.norms[1:])
    # one token at a time through the cache, and the whole sequence at once
    prompt = [5, 9, 1, 3] * 5
    for both_ways in (False, True):
        made = model.generate(prompt, 6, both_ways=both_ways)
        seq = torch.tensor(prompt + made, device="cuda")
        first = torch.tensor([len(prompt)], dtype=torch.int32, device="cuda") if both_ways else None

        def attend(n, qkv, batch):
            q, k, v = qkv.split([model.heads, model.kv_heads, model.kv_heads], dim=1)
            out, lse = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty(model.heads, q.shape[0], device="cuda")
            samo.samo_attention(q, k, v, out, lse, window=model.window, scores=model.scores[n]._replace(first_keys=first))
            return out

        with torch.no_grad():
            logits = model.forward(seq, attend, None).float()
        for i, token in enumerate(made):
            row = logits[len(prompt) - 1 + i]
            assert float(row.max() - row[token]) < 0.05 * float(row.abs().max()), (both_ways, i)


def test_the_decoder_captured_and_replayed_beside_its_eager_self():
    """Forward and backward pass of attention with every form and of the norms in one graph, replayed between eager calls of the same tensors."""
    t, heads, dim = 300, 4, 64
    hidden = heads * dim
    rnd = lambda *s: torch.randn(s, device="cuda").half()
    qkv, dout, y, stream = rnd(t, 3 * heads, dim), rnd(t, hidden), rnd(t, hidden), torch.randn(t, hidden, device="cuda")
    table = rnd(heads, 32)
    scores = samo.Scores(cap=10.0, table=table, borders=samo.samo_bucket_borders(32, 128), slopes=torch.rand(heads, device="cuda"))
    norm = samo.Norm(kind="layer", y_norm=True, weight=rnd(hidden), bias=rnd(hidden), y_weight=rnd(hidden), gate=rnd(hidden))

    def run():
        q, k, v = qkv.split(heads, dim=1)
        out, lse, dqkv = torch.empty(t, heads, dim, dtype=torch.float16, device="cuda"), torch.empty(heads, t, device="cuda"), torch.empty_like(qkv)
        samo.samo_attention(q, k, v, out, lse, scores=scores)
        new, nxt, stats = torch.empty_like(stream), torch.empty_like(y), torch.empty(t, 4, device="cuda")
        samo.samo_norm(norm, stream, nxt, y=out.view(t, hidden), new_stream=new, stats=stats)
        ds, dy, dtable, dgate, dbias = torch.empty_like(stream), torch.empty_like(y), torch.empty_like(table), rnd_like(norm.gate), rnd_like(norm.bias)
        samo.samo_norm_backward(norm, dout, new, stats, ds, y=out.view(t, hidden), dy=dy, grads=samo.NormGrads(gate=dgate, bias=dbias))
        samo.samo_attention_backward(dy.view(t, heads, dim), q, k, v, out, lse, *dqkv.split(heads, dim=1), scores=scores, dtable=dtable)
        return out, lse, new, nxt, ds, dy, dqkv, dtable, dgate, dbias

    rnd_like = lambda x: torch.zeros_like(x)
    want = [x.clone() for x in run()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(run(), want))
