"""A small pruned decoder trained on packed sequences, and asked for tokens one at a time.

Every weight matrix keeps a random share of its elements.  Its fp32 values, its two Adam states (a byte each) and its gradient
exist for those only; the fp16 matrix that the products read is dense with explicit zeros.  The pieces in the order of a step:

    samo_attention, samo_glu                        forward, between torch's plain products
    samo_attention_backward, samo_glu_backward      the gradients of activations
    samo_wgrad_gather_fp16_batched                  all weights' gradients, formed and compressed in one kernel
    Plan8.samo_step8_batched                        Adam on 8-bit states; writes the fp16 matrices of the next step

    python examples/pruned_decoder.py --layers 2 --hidden 256 --ffn 512 --heads 4 --steps 60
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2302_05045_amd as samo  # noqa: E402

DEV = "cuda"
LOSS_SCALE = 1024.0


class Attention(torch.autograd.Function):
    """qkv: tokens x (heads + 2 kv_heads) x dim, the projection's output; its gradient is written in place of slices of one tensor."""

    @staticmethod
    def forward(ctx, qkv, heads, kv_heads, starts, longest, window):
        q, k, v = qkv.split([heads, kv_heads, kv_heads], dim=1)
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        lse = torch.empty(heads, q.shape[0], device=qkv.device)
        samo.samo_attention(q, k, v, out, lse, window=window, q_start=starts, k_start=starts, max_q=longest, max_k=longest)
        ctx.save_for_backward(qkv, out, lse, starts)
        ctx.sizes = (heads, kv_heads, longest, window)
        return out

    @staticmethod
    def backward(ctx, dout):
        qkv, out, lse, starts = ctx.saved_tensors
        heads, kv_heads, longest, window = ctx.sizes
        parts = [heads, kv_heads, kv_heads]
        dqkv = torch.empty_like(qkv)
        samo.samo_attention_backward(dout.contiguous(), *qkv.split(parts, dim=1), out, lse, *dqkv.split(parts, dim=1), window=window,
                                     q_start=starts, k_start=starts, max_q=longest, max_k=longest)
        return dqkv, None, None, None, None, None


class Linear(torch.autograd.Function):
    """y = x w^T; the weight's gradient is left to the step: its operands join the model's list."""

    @staticmethod
    def forward(ctx, x, weight, todo):
        ctx.save_for_backward(x)
        ctx.weight, ctx.todo = weight, todo
        return x @ weight.dense.T

    @staticmethod
    def backward(ctx, dy):
        dy = dy.contiguous()
        ctx.todo.append((dy, ctx.saved_tensors[0], ctx.weight.idx, ctx.weight.seg_ptr, ctx.weight.gc16))
        return dy @ ctx.weight.dense, None, None


class Glu(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, todo):
        h, gate, up = (torch.empty(x.shape[0], w_gate.dense.shape[0], dtype=x.dtype, device=x.device) for _ in range(3))
        samo.samo_glu(x, w_gate.dense, w_up.dense, h, gate, up)
        ctx.save_for_backward(x, gate, up)
        ctx.weights, ctx.todo = (w_gate, w_up), todo
        return h

    @staticmethod
    def backward(ctx, dh):
        x, gate, up = ctx.saved_tensors
        dgate, dup, dx = torch.empty_like(gate), torch.empty_like(up), torch.empty_like(x)
        samo.samo_glu_backward(dh.contiguous(), gate, up, ctx.weights[0].dense, ctx.weights[1].dense, dgate, dup, dx)
        for w, dy in zip(ctx.weights, (dgate, dup)):
            ctx.todo.append((dy, x, w.idx, w.seg_ptr, w.gc16))
        return dx, None, None, None


class Weight:
    """One matrix: what is resident of it, and the dense fp16 form."""

    def __init__(self, rows, cols, kept, gen, first):
        w = torch.randn(rows, cols, device=DEV, generator=gen) * (kept * cols) ** -0.5
        self.idx = self.seg_ptr = None
        if kept < 1:
            mask = (torch.rand(rows, cols, device=DEV, generator=gen) < kept).to(torch.uint8)
            index = samo.samo_build_index(mask.view(-1))
            self.idx, self.seg_ptr = index.idx, index.seg_ptr
            w *= mask
        self.p = (w.view(-1) if self.idx is None else w.view(-1)[self.idx.long()]).contiguous()
        self.q8, self.s8 = samo.alloc_state8(rows * cols, self.p.numel(), DEV)
        self.gc16 = torch.empty(self.p.numel(), dtype=torch.float16, device=DEV)
        self.dense = w.half()
        self.layer = samo.Layer8(rows * cols, self.idx, self.seg_ptr, self.p, self.q8, self.s8, w=self.dense.view(-1), gc16=self.gc16, rng_offset=first)


class Decoder:
    def __init__(self, layers, hidden, ffn, heads, kv_heads, vocab, kept, window=0, seed=0):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.window = heads, kv_heads, hidden // heads, window
        self.weights, self.blocks, self.todo, self.steps = [], [], [], 0
        elements = 0

        def weight(rows, cols, share):
            nonlocal elements
            self.weights.append(Weight(rows, cols, share, gen, elements))
            elements += rows * cols
            return self.weights[-1]

        for _ in range(layers):
            self.blocks.append(dict(qkv=weight((heads + 2 * kv_heads) * self.dim, hidden, kept), proj=weight(hidden, heads * self.dim, kept),
                                    gate=weight(ffn, hidden, kept), up=weight(ffn, hidden, kept), down=weight(hidden, ffn, kept)))
        self.head = weight(vocab, hidden, 1.0)               # not pruned
        self.embedding = torch.randn(vocab, hidden, device=DEV, generator=gen).half()      # not trained
        self.plan = samo.Plan8([w.layer for w in self.weights])

    def attend(self, n, qkv, batch):
        return Attention.apply(qkv, self.heads, self.kv_heads, batch["starts"], batch["longest"], self.window)

    def forward(self, tokens, attend, batch):
        norm = lambda x: F.rms_norm(x.float(), x.shape[-1:]).half()
        x = self.embedding[tokens].requires_grad_(torch.is_grad_enabled())
        for n, b in enumerate(self.blocks):
            qkv = Linear.apply(norm(x), b["qkv"], self.todo).view(-1, self.heads + 2 * self.kv_heads, self.dim)
            x = x + Linear.apply(attend(n, qkv, batch).flatten(1), b["proj"], self.todo)
            x = x + Linear.apply(Glu.apply(norm(x), b["gate"], b["up"], self.todo), b["down"], self.todo)
        return Linear.apply(norm(x), self.head, self.todo)

    def step(self, tokens, targets, batch, lr):
        self.todo.clear()
        loss = F.cross_entropy(self.forward(tokens, self.attend, batch).float(), targets)
        (loss * LOSS_SCALE).backward()
        most = samo.SAMO_WGRAD_MAX_JOBS
        for first in range(0, len(self.todo), most):
            samo.samo_wgrad_gather_fp16_batched(self.todo[first:first + most])
        self.todo.clear()
        self.steps += 1
        self.plan.samo_step8_batched(1.0 / LOSS_SCALE, samo.adam_cfg(self.steps, lr=lr), seed=self.steps, source=1)
        return float(loss.detach())

    @torch.no_grad()
    def generate(self, prompt, count):
        """The tokens most likely to follow, one at a time: one query a step behind the cache's keys."""
        room = len(prompt) + count
        cache = torch.empty(len(self.blocks), 2, room, self.kv_heads, self.dim, dtype=torch.float16, device=DEV)
        done = 0

        def attend(n, qkv, batch):
            nonlocal done
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
            end = done + q.shape[0]
            cache[n, 0, done:end], cache[n, 1, done:end] = k, v
            out, lse = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty(self.heads, q.shape[0], device=DEV)
            samo.samo_attention(q, cache[n, 0, :end], cache[n, 1, :end], out, lse, window=self.window)
            return out

        tokens, result = torch.tensor(prompt, device=DEV), []
        for _ in range(count):
            logits = self.forward(tokens, attend, None)
            done += tokens.numel()
            tokens = logits[-1:].argmax(1)
            result.append(int(tokens))
        return result


def packed_batch(sequences, longest, vocab, gen):
    """Sequences of uneven lengths that repeat their first tokens over and over, end to end: a token's successor is to be looked up."""
    tokens, targets, starts = [], [], [0]
    for _ in range(sequences):
        n = int(torch.randint(longest // 2, longest + 1, (1,), generator=gen))
        period = int(torch.randint(2, 9, (1,), generator=gen))
        row = torch.randint(0, vocab, (period,), generator=gen).repeat(n // period + 2)[:n + 1]
        tokens.append(row[:-1])
        targets.append(row[1:])
        starts.append(starts[-1] + n)
    return (torch.cat(tokens).to(DEV), torch.cat(targets).to(DEV),
            dict(starts=torch.tensor(starts, dtype=torch.int32, device=DEV), longest=max(b - a for a, b in zip(starts, starts[1:]))))


def train(layers=2, hidden=256, ffn=512, heads=4, kv_heads=2, vocab=64, kept=0.3, window=0, steps=60, sequences=16, longest=96, lr=2e-3, seed=0,
          log=None):
    model = Decoder(layers, hidden, ffn, heads, kv_heads, vocab, kept, window, seed)
    gen = torch.Generator()
    gen.manual_seed(seed)
    losses = []
    for n in range(steps):
        tokens, targets, batch = packed_batch(sequences, longest, vocab, gen)
        losses.append(model.step(tokens, targets, batch, lr))
        if log and n % 10 == 9:
            log("step %d: loss %.4f" % (n + 1, losses[-1]))
    return model, losses


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("layers", 2), ("hidden", 256), ("ffn", 512), ("heads", 4), ("kv-heads", 2), ("vocab", 64), ("window", 0), ("steps", 300),
                        ("sequences", 16), ("longest", 96), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--kept", type=float, default=0.3)
    ap.add_argument("--lr", type=float, default=2e-3)
    args = vars(ap.parse_args())
    model, _ = train(**args, log=lambda line: print(line, flush=True))
    kept = sum(w.p.numel() for w in model.weights)
    print("%d of %d elements kept; 10 bytes each and their gradient" % (kept, sum(w.dense.numel() for w in model.weights)))
    prompt = [3, 14, 15, 9] * 4
    print("after", prompt, "->", model.generate(prompt, 8))


if __name__ == "__main__":
    main()
