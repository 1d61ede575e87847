"""A small pruned decoder trained on packed sequences, and asked for tokens one at a time.

Every weight matrix keeps a random share of its elements.  Its fp32 values, its two Adam states (a byte each) and its gradient
exist for those only; the fp16 matrix that the products read is dense with explicit zeros.  The pieces in the order of a step:

    samo_attention, samo_glu                        forward, between torch's plain products
    samo_norm                                       with sandwich: the norms before and after a block, its gate and the residual sum
    samo_attention_backward, samo_glu_backward, samo_norm_backward      the gradients of activations, of norms and of bias tables
    samo_wgrad_gather_fp16_batched                  all weights' gradients, formed and compressed in one kernel
    Plan8.samo_step8_batched                        Adam on 8-bit states; writes the fp16 matrices of the next step

Scores may be capped (cap) and get a learned bias by the distance's bucket (buckets); a prompt may be read in both directions (see generate).

    python examples/pruned_decoder.py --layers 2 --hidden 256 --ffn 512 --heads 4 --steps 60
    python examples/pruned_decoder.py --cap 30 --buckets 16 --sandwich
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
    def forward(ctx, qkv, heads, kv_heads, starts, longest, window, scores=None, dtable=None):
        q, k, v = qkv.split([heads, kv_heads, kv_heads], dim=1)
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        lse = torch.empty(heads, q.shape[0], device=qkv.device)
        samo.samo_attention(q, k, v, out, lse, window=window, q_start=starts, k_start=starts, max_q=longest, max_k=longest,
                            scores=scores)
        ctx.save_for_backward(qkv, out, lse, starts)
        ctx.sizes = (heads, kv_heads, longest, window, scores, dtable)
        return out

    @staticmethod
    def backward(ctx, dout):
        qkv, out, lse, starts = ctx.saved_tensors
        heads, kv_heads, longest, window, scores, dtable = ctx.sizes
        parts = [heads, kv_heads, kv_heads]
        dqkv = torch.empty_like(qkv)
        samo.samo_attention_backward(dout.contiguous(), *qkv.split(parts, dim=1), out, lse, *dqkv.split(parts, dim=1), window=window,
                                     q_start=starts, k_start=starts, max_q=longest, max_k=longest, scores=scores, dtable=dtable)
        return dqkv, None, None, None, None, None, None, None


class Norms(torch.autograd.Function):
    """(new stream, input of the next block) of the residual stream and a block's output y (None: the norm before the first block)."""

    @staticmethod
    def forward(ctx, stream, y, norm, grads):
        new, out = None if y is None else torch.empty_like(stream), torch.empty(stream.shape, dtype=torch.float16, device=stream.device)
        stats = torch.empty(stream.shape[0], 4, device=stream.device)
        samo.samo_norm(norm, stream, out, y=y, new_stream=new, stats=stats)
        new = stream.clone() if new is None else new
        ctx.save_for_backward(new, y, stats)
        ctx.norm, ctx.grads = norm, grads
        return new, out

    @staticmethod
    def backward(ctx, dnew, dout):
        new, y, stats = ctx.saved_tensors
        dstream, dy = torch.empty_like(new), None if y is None else torch.empty_like(y)
        samo.samo_norm_backward(ctx.norm, dout.contiguous(), new, stats, dstream, dnew=dnew.contiguous(), y=y, dy=dy, grads=ctx.grads)
        return dstream, dy, None, None


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

    def __init__(self, rows, cols, kept, gen, first, value=None):
        w = torch.randn(rows, cols, device=DEV, generator=gen) * (kept * cols) ** -0.5 if value is None else torch.full((rows, cols), value, device=DEV)
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
    def __init__(self, layers, hidden, ffn, heads, kv_heads, vocab, kept, window=0, seed=0, cap=0.0, buckets=0, sandwich=False):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.window = heads, kv_heads, hidden // heads, window
        self.weights, self.blocks, self.todo, self.steps = [], [], [], 0
        elements = 0

        def weight(rows, cols, share, value=None):
            nonlocal elements
            self.weights.append(Weight(rows, cols, share, gen, elements, value))
            elements += rows * cols
            return self.weights[-1]

        for _ in range(layers):
            self.blocks.append(dict(qkv=weight((heads + 2 * kv_heads) * self.dim, hidden, kept), proj=weight(hidden, heads * self.dim, kept),
                                    gate=weight(ffn, hidden, kept), up=weight(ffn, hidden, kept), down=weight(hidden, ffn, kept)))
        self.head = weight(vocab, hidden, 1.0)               # not pruned
        self.scores, self.tables = [None] * layers, [None] * layers
        if cap or buckets:
            borders = samo.samo_bucket_borders(buckets, 128) if buckets else None
            for n in range(layers):
                table = weight(heads, buckets, 1.0, value=0.0) if buckets else None
                self.tables[n] = table and table.gc16.view(heads, buckets)
                self.scores[n] = samo.Scores(cap=cap, table=table and table.dense, borders=borders)
        self.norms = []                                      # before the first block, then around every block
        if sandwich:
            for n in range(2 * layers + 1):
                own = dict(weight=weight(1, hidden, 1.0, value=1.0))
                if n:
                    own.update(y_weight=weight(1, hidden, 1.0, value=1.0), gate=weight(1, hidden, 1.0, value=1.0))
                self.norms.append((samo.Norm(y_norm=n > 0, scale=(2 * layers) ** -0.5, **{k: w.dense.view(-1) for k, w in own.items()}),
                                   samo.NormGrads(**{k: w.gc16 for k, w in own.items()})))
        self.embedding = torch.randn(vocab, hidden, device=DEV, generator=gen).half()      # not trained
        self.plan = samo.Plan8([w.layer for w in self.weights])

    def attend(self, n, qkv, batch):
        return Attention.apply(qkv, self.heads, self.kv_heads, batch["starts"], batch["longest"], self.window, self.scores[n], self.tables[n])

    def forward(self, tokens, attend, batch):
        norm = lambda x: F.rms_norm(x.float(), x.shape[-1:]).half()
        x = self.embedding[tokens].requires_grad_(torch.is_grad_enabled())
        if self.norms:
            stream, x = Norms.apply(x, None, *self.norms[0])
            for n, b in enumerate(self.blocks):
                qkv = Linear.apply(x, b["qkv"], self.todo).view(-1, self.heads + 2 * self.kv_heads, self.dim)
                y = Linear.apply(attend(n, qkv, batch).flatten(1), b["proj"], self.todo)
                stream, x = Norms.apply(stream, y, *self.norms[2 * n + 1])
                y = Linear.apply(Glu.apply(x, b["gate"], b["up"], self.todo), b["down"], self.todo)
                stream, x = Norms.apply(stream, y, *self.norms[2 * n + 2])
            return Linear.apply(x, self.head, self.todo)
        for n, b in enumerate(self.blocks):
            qkv = Linear.apply(norm(x), b["qkv"], self.todo).view(-1, self.heads + 2 * self.kv_heads, self.dim)
            x = x + Linear.apply(attend(n, qkv, batch).flatten(1), b["proj"], self.todo)
            x = x + Linear.apply(Glu.apply(norm(x), b["gate"], b["up"], self.todo), b["down"], self.todo)
        return Linear.apply(norm(x), self.head, self.todo)

    def gradients(self, tokens, targets, batch):
        """The loss; LOSS_SCALE times its gradient is left in the weights' gc16."""
        self.todo.clear()
        loss = F.cross_entropy(self.forward(tokens, self.attend, batch).float(), targets)
        (loss * LOSS_SCALE).backward()
        most = samo.SAMO_WGRAD_MAX_JOBS
        for first in range(0, len(self.todo), most):
            samo.samo_wgrad_gather_fp16_batched(self.todo[first:first + most])
        self.todo.clear()
        return loss

    def step(self, tokens, targets, batch, lr):
        loss = self.gradients(tokens, targets, batch)
        self.steps += 1
        self.plan.samo_step8_batched(1.0 / LOSS_SCALE, samo.adam_cfg(self.steps, lr=lr), seed=self.steps, source=1)
        return float(loss.detach())

    @torch.no_grad()
    def generate(self, prompt, count, both_ways=False):
        """The tokens most likely to follow, one at a time: one query a step behind the cache's keys.  both_ways: every token of the prompt sees all of it."""
        room = len(prompt) + count
        cache = torch.empty(len(self.blocks), 2, room, self.kv_heads, self.dim, dtype=torch.float16, device=DEV)
        done = 0
        first_keys = torch.tensor([len(prompt)], dtype=torch.int32, device=DEV) if both_ways else None

        def attend(n, qkv, batch):
            nonlocal done
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
            end = done + q.shape[0]
            cache[n, 0, done:end], cache[n, 1, done:end] = k, v
            out, lse = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty(self.heads, q.shape[0], device=DEV)
            scores = (self.scores[n] or samo.Scores())._replace(first_keys=first_keys) if both_ways else self.scores[n]
            samo.samo_attention(q, cache[n, 0, :end], cache[n, 1, :end], out, lse, window=self.window, scores=scores)
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
          cap=0.0, buckets=0, sandwich=False, log=None):
    model = Decoder(layers, hidden, ffn, heads, kv_heads, vocab, kept, window, seed, cap, buckets, sandwich)
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
                        ("sequences", 16), ("longest", 96), ("seed", 0), ("buckets", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--kept", type=float, default=0.3)
    ap.add_argument("--lr", type=float, default=2e-3)
    ap.add_argument("--cap", type=float, default=0.0)
    ap.add_argument("--sandwich", action="store_true")
    args = vars(ap.parse_args())
    model, _ = train(**args, log=lambda line: print(line, flush=True))
    kept = sum(w.p.numel() for w in model.weights)
    print("%d of %d elements kept; 10 bytes each and their gradient" % (kept, sum(w.dense.numel() for w in model.weights)))
    prompt = [3, 14, 15, 9] * 4
    print("after", prompt, "->", model.generate(prompt, 8))


if __name__ == "__main__":
    main()
