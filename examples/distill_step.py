"""Training steps of a small attention-only student that learns a teacher's next words from its top logits, with a part of its
tensors frozen in each step: the operators around the linear layers (embedding, norms, attention, distillation loss) with
the stage backward, the masked optimizer and the stability scores that pick the next step's frozen tensors.

    python3 examples/distill_step.py --steps 40 --freeze 0.5

The products of the forward pass and the additions of activations are torch's; everything else is the library's.  The words are synthetic:
a teacher that knows only the word before, and sequences of different lengths drawn from it, packed without padding between them.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2602_05754_amd as tf  # noqa: E402


class Task:
    """`vocabulary` words, each with `k` followers and the teacher's logits of those."""

    def __init__(self, vocabulary, k, seed=0):
        rs = np.random.default_rng(seed)
        self.followers = np.stack([rs.permutation(vocabulary)[:k] for _ in range(vocabulary)]).astype(np.int32)
        self.logits = (2 * rs.standard_normal((vocabulary, k))).astype(np.float32)
        self.vocabulary, self.rs = vocabulary, rs

    def batch(self, tokens, sequences):
        """(words, starts, weight): sequences drawn from the teacher; the last word of each has no follower to learn."""
        starts = np.concatenate([[0], np.sort(self.rs.choice(np.arange(1, tokens), sequences - 1, replace=False)), [tokens]])
        words, weight = np.empty(tokens, np.int32), np.ones(tokens, np.float32)
        for a, b in zip(starts, starts[1:]):
            words[a] = self.rs.integers(self.vocabulary)
            for t in range(a + 1, b):
                p = np.exp(self.logits[words[t - 1]].astype(np.float64))
                words[t] = self.rs.choice(self.followers[words[t - 1]], p=p / p.sum())
            weight[b - 1] = 0
        return words, starts.astype(np.int64), weight


class Student:
    """Embedding, `blocks` times x += attention(norm(x)), norm, products with the words.  Names of tensors: embedding, then of each
    block norm, q, k, v, o, then final, final_bias, head."""

    def __init__(self, ctx, vocabulary, d, heads, kv_heads, blocks, io="bf16", seed=1):
        self.ctx, self.d, self.heads, self.kv_heads, self.hd, self.blocks = ctx, d, heads, kv_heads, d // heads, blocks
        self.V, self.io, self.dtype = vocabulary, {"f32": tf.TF_F32, "bf16": tf.TF_BF16}[io], {"f32": torch.float32, "bf16": torch.bfloat16}[io]
        self.scale, self.embed_scale, self.tau, self.eps = self.hd ** -0.5, d ** 0.5, 1.0, 1e-6
        kv = kv_heads * self.hd
        self.shapes = {"embedding": (vocabulary, d)}
        for b in range(blocks):
            self.shapes.update({f"{b}.norm": (d,), f"{b}.q": (d, d), f"{b}.k": (d, kv), f"{b}.v": (d, kv), f"{b}.o": (d, d)})
        self.shapes.update({"final": (d,), "final_bias": (d,), "head": (d, vocabulary)})
        self.names = list(self.shapes)
        g = torch.Generator().manual_seed(seed)
        self.master, self.weight, self.grad = {}, {}, {}
        for n, s in self.shapes.items():
            if n == "final_bias":
                w = torch.zeros(s)
            elif len(s) == 1:
                w = torch.ones(s)
            else:
                w = torch.randn(s, generator=g) * (s[1] ** -0.5 if n == "embedding" else s[0] ** -0.5)
            self.master[n] = w.cuda()
            self.weight[n] = self.master[n] if io == "f32" else self.master[n].to(self.dtype)
            self.grad[n] = torch.zeros(s, device="cuda")
        zeros = lambda: [torch.zeros_like(self.master[n]) for n in self.names]
        self.m, self.v, self.ema, self.ema_abs = zeros(), zeros(), zeros(), zeros()
        self.steps = [1] * len(self.names)
        self.sums = torch.zeros(2 * len(self.names), dtype=torch.float64, device="cuda")

    def empty(self, *shape, dtype=None):
        return torch.empty(shape, dtype=dtype or self.dtype, device="cuda")

    def forward(self, words, starts):
        """logits, and what the backward pass reads again."""
        T, d, hd, w = len(words), self.d, self.hd, self.weight
        f32 = torch.float32
        x = self.empty(T, d)
        tf.tf_embedding_forward(self.ctx, T, self.V, d, self.io, words, w["embedding"], self.embed_scale, x)
        kept = []
        for b in range(self.blocks):
            n, rstd = self.empty(T, d), self.empty(T, dtype=f32)
            tf.tf_norm_forward(self.ctx, T, d, self.io, x, w[f"{b}.norm"], None, self.eps, False, n, None, rstd)
            q, k, v = (n @ w[f"{b}.{p}"] for p in "qkv")
            o, lse = self.empty(T, d), self.empty(T, self.heads, dtype=f32)
            tf.tf_attention_forward(self.ctx, starts, T, self.heads, self.kv_heads, hd, self.io, q, k, v, self.scale, o, lse)
            kept.append((x, n, rstd, q, k, v, o, lse))
            x = x + o @ w[f"{b}.o"]
        n, mean, rstd = self.empty(T, d), self.empty(T, dtype=f32), self.empty(T, dtype=f32)
        tf.tf_norm_forward(self.ctx, T, d, self.io, x, w["final"], w["final_bias"], self.eps, True, n, mean, rstd)
        return n @ w["head"], (kept, x, n, mean, rstd)

    def backward(self, words, starts, dlogits, kept, frozen):
        """Gradients of the tensors that are not frozen -> self.grad."""
        T, d, hd, io, w, ctx = len(words), self.d, self.hd, self.io, self.weight, self.ctx
        kept, x, n, mean, rstd = kept
        is_frozen = dict(zip(self.names, frozen))
        grad = {name: None if is_frozen[name] else g for name, g in self.grad.items()}

        def linear(names, X, dY):
            """The layers' dW; the gradient of the input that they share.  (One product for them all, tf_stage_backward_shared, in bf16 takes
            only the sizes of the matrix-core kernel, and these tokens and widths may be any.)"""
            dX = [torch.empty_like(X) for _ in names]
            tf.tf_stage_backward(ctx, [self.shapes[i] for i in names], T, io, [w[i] for i in names], [X] * len(names), dY,
                                 [is_frozen[i] for i in names], dX, [self.grad[i] for i in names], tf.TF_F32)
            return dX[0] if len(dX) == 1 else torch.stack(dX).float().sum(0).to(X.dtype)

        dn, dx = linear(["head"], n, [dlogits]), self.empty(T, d)
        tf.tf_norm_backward(ctx, T, d, io, x, w["final"], dn, mean, rstd, True, dx, grad["final"], grad["final_bias"], tf.TF_F32)
        for b in reversed(range(self.blocks)):
            x, n, rstd, q, k, v, o, lse = kept[b]
            do = linear([f"{b}.o"], o, [dx])
            dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
            tf.tf_attention_backward(ctx, starts, T, self.heads, self.kv_heads, hd, io, q, k, v, o, lse, do, self.scale, dq, dk, dv)
            dn = linear([f"{b}.{p}" for p in "qkv"], n, [dq, dk, dv])
            into = self.empty(T, d)
            tf.tf_norm_backward(ctx, T, d, io, x, w[f"{b}.norm"], dn, None, rstd, False, into, grad[f"{b}.norm"], None, tf.TF_F32)
            dx = dx + into
        if grad["embedding"] is not None:
            tf.tf_embedding_backward(ctx, T, self.V, d, io, words, dx, self.embed_scale, grad["embedding"], tf.TF_F32)

    def loss(self, logits, ids, teacher, weight):
        """Loss per token, and the gradient of its sum over the tokens' number."""
        T, K = ids.shape
        loss, dlogits = self.empty(T, dtype=torch.float32), torch.empty_like(logits)
        tf.tf_distill_loss(self.ctx, T, self.V, K, self.io, logits, ids, teacher, weight, self.tau, 1.0 / T, loss, dlogits)
        return loss, dlogits

    def update(self, frozen, lr):
        """The optimizer's step, the stability averages with it; scores of all tensors."""
        numel = [self.master[n].numel() for n in self.names]
        bf16 = self.io == tf.TF_BF16
        tf.tf_masked_adamw(self.ctx, numel, [self.master[n] for n in self.names], self.m, self.v, [self.grad[n] for n in self.names], tf.TF_F32,
                           self.steps, lr, 0.9, 0.95, 1e-8, 0.0, p_lowp=[self.weight[n] for n in self.names] if bf16 else None,
                           tensor_freeze_mask=frozen, ema=self.ema, ema_abs=self.ema_abs, ema_decay=0.9, score_sums=self.sums)
        self.steps = [s if f else s + 1 for s, f in zip(self.steps, frozen)]
        return tf.tf_stability_scores(self.sums.cpu().numpy())

    def step(self, batch, task_ids, task_logits, frozen, lr):
        """(mean loss, scores) of a step."""
        words, starts, weight = batch
        words, weight = torch.from_numpy(words).cuda(), torch.from_numpy(weight).cuda()
        logits, kept = self.forward(words, starts)
        loss, dlogits = self.loss(logits, task_ids[words.long()].contiguous(), task_logits[words.long()].contiguous(), weight)
        self.backward(words, starts, dlogits, kept, frozen)
        scores = self.update(frozen, lr)
        return float(loss.mean()), scores


def train(steps, freeze, io="bf16", vocabulary=512, k=8, d=256, heads=4, kv_heads=2, blocks=2, tokens=1024, sequences=7, lr=3e-3, say=lambda *a: None):
    """Mean loss of each step; from the second on the `freeze` share of tensors with the lowest scores is frozen."""
    ctx = tf.Context(torch.cuda.current_device())
    task, student = Task(vocabulary, k), Student(ctx, vocabulary, d, heads, kv_heads, blocks, io)
    ids, teacher = torch.from_numpy(task.followers).cuda(), torch.from_numpy(task.logits).cuda()
    frozen, losses = np.zeros(len(student.names), np.uint8), []
    for i in range(steps):
        loss, scores = student.step(task.batch(tokens, sequences), ids, teacher, frozen, lr)
        losses.append(loss)
        say(f"step {i}: loss {loss:.4f}, frozen {int(frozen.sum())} of {len(frozen)}")
        frozen = tf.tf_select_lowest(scores, tf.tf_num_frozen(freeze, len(frozen)))
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    parser.add_argument("--steps", type=int, default=40)
    parser.add_argument("--freeze", type=float, default=0.5)
    parser.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    args = parser.parse_args()
    train(args.steps, args.freeze, args.dtype, say=lambda line: print(line, flush=True))
