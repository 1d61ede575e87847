"""The example runs the operators together: a pruned decoder learns to repeat, and generates what its forward pass over whole sequences says."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def test_pruned_decoder_learns_and_generates():
    import pruned_decoder
    model, losses = pruned_decoder.train(layers=2, hidden=128, ffn=264, heads=4, kv_heads=2, vocab=32, kept=0.4, steps=80, sequences=8, longest=50)
    assert all(x == x and x < 20 for x in losses)
    assert sum(losses[-5:]) < 0.8 * sum(losses[:5]), losses
    for w in model.weights:                                  # what is pruned stays zero, what is kept is the fp16 of p
        dense = torch.zeros_like(w.dense).view(-1)
        if w.idx is None:
            dense.copy_(w.p)
        else:
            dense[w.idx.long()] = w.p.half()
        assert torch.equal(w.dense.view(-1), dense)
    # one token at a time through the cache, and the whole sequence at once: the same attention, other kernels' orders of sums
    prompt = [5, 9, 1, 30] * 5
    made = model.generate(prompt, 6)
    seq = torch.tensor(prompt + made, device="cuda")
    with torch.no_grad():
        logits = model.forward(seq, model.attend, dict(starts=torch.tensor([0, seq.numel()], dtype=torch.int32, device="cuda"), longest=seq.numel())).float()
    for i, token in enumerate(made):
        row = logits[len(prompt) - 1 + i]
        assert float(row.max() - row[token]) < 0.05 * float(row.abs().max()), i


def test_the_same_training_gives_the_same_bits():
    import pruned_decoder
    runs = [pruned_decoder.train(layers=1, hidden=64, ffn=96, heads=2, kv_heads=1, vocab=24, steps=4, sequences=3, longest=40, window=17) for _ in range(2)]
    assert runs[0][1] == runs[1][1]
    for a, b in zip(runs[0][0].weights, runs[1][0].weights):
        assert torch.equal(a.p, b.p) and torch.equal(a.q8, b.q8) and torch.equal(a.s8, b.s8) and torch.equal(a.dense, b.dense)
