"""Both ends of a synchronisation, on one GPU: a trainer whose steps change a model, and a receiver that answers with it.

The model is the smallest that has the parts: an embedding, a norm weight and a head, logits = (scale * E[token] * g) H'.
Trainer, each step: rows of the embedding, the loss, the gradients (the embedding's through its tokens, two micro-batches
added up), clipping by the norm of all gradients, an update of the fp32 master weights, and an encode that finds what the
bf16 weights' bits changed in.  Receiver, two shards: apply, the head's shards rounded to 4-bit matrices, and logits for
prompts and for single tokens, each shard its rows of the embedding and its columns of the logits.

    python examples/train_and_serve.py [steps]
"""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

import paper_2605_06534_amd as R
from workloads import models

VOCAB, HIDDEN, TP = 2048, 320, 2
TOKENS, SCALE, RATE, MAX_NORM = 4096, HIDDEN ** 0.5, 6.0, 0.25


class Trainer:
    def __init__(self, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        self.tensors = models.decoder(0, HIDDEN, 1, 1, HIDDEN, HIDDEN, VOCAB)          # embedding, norm weight, head
        self.master = [torch.randn(t["rows"], t["cols"], generator=g, device="cuda") * 0.02 for t in self.tensors]
        self.master[1].fill_(1.0)
        self.weights = [w.to(torch.bfloat16) for w in self.master]
        self.grads = [torch.zeros_like(w) for w in self.master]
        numels = [w.numel() for w in self.master]
        self.total, self.offsets = sum(numels), R.offset_table(numels)
        self.grad_tab, self.weight_tab, self.master_tab = R.ptr_table(self.grads), R.ptr_table(self.weights), R.ptr_table(self.master)
        self.norm, self.clip_ws = torch.zeros(1, device="cuda"), R.grad_workspace()
        self.lookup_ws = R.embedding_grad_workspace(VOCAB, HIDDEN, TOKENS)
        self.plan = R.shard_plan(self.tensors, TP)
        self.encode_ws = R.workspace(self.plan)
        self.buckets = [R.Bucket(self.plan.bucket_capacity(d), len(self.tensors)) for d in range(TP)]

    def gradients(self, tokens, targets, accumulate):
        """Adds (or sets) the gradients of one micro-batch; returns its loss."""
        _, g, head = self.weights
        x = torch.empty(len(tokens), HIDDEN, dtype=torch.bfloat16, device="cuda")
        R.embedding_lookup(self.weights[0], tokens, x, scale=SCALE)
        y = x.float() * g.float()
        logits = y @ head.float().t()
        loss = torch.nn.functional.cross_entropy(logits, targets)
        d_logits = torch.softmax(logits, 1)
        d_logits[torch.arange(len(tokens), device="cuda"), targets] -= 1
        d_logits /= len(tokens)
        d_y = d_logits @ head.float()
        d_head, d_g = d_logits.t() @ y, (d_y * x.float()).sum(0, keepdim=True)
        for grad, d in ((self.grads[1], d_g), (self.grads[2], d_head)):
            grad.add_(d) if accumulate else grad.copy_(d)
        R.embedding_grad((d_y * g.float()).to(torch.bfloat16), tokens, self.grads[0], self.lookup_ws, scale=SCALE, accumulate=accumulate)
        return loss

    def step(self, micro_batches):
        """One update; the buckets hold what it changed.  Returns loss and norm of the gradients."""
        losses = [self.gradients(tokens, targets, i > 0) for i, (tokens, targets) in enumerate(micro_batches)]
        R.grad_clip_norm(self.grad_tab, self.offsets, self.total, torch.float32, self.grad_tab, MAX_NORM, self.norm, self.clip_ws)
        for w, grad in zip(self.master, self.grads):
            w.sub_(grad, alpha=RATE)
        R.delta_encode_refresh(self.plan, self.weight_tab, self.master_tab, R.FP32_RNE, self.buckets, self.encode_ws)
        return sum(losses).item() / len(losses), self.norm.item()


class Shard:
    """What one receiver holds: its rows of the embedding and of the head."""

    def __init__(self, trainer, d):
        self.plan, self.d = trainer.plan, d
        self.rows = VOCAB // TP
        self.weights = [torch.empty(self.plan.local_numel(t, d), dtype=torch.bfloat16, device="cuda") for t in range(len(trainer.tensors))]
        self.tab = R.ptr_table(self.weights)
        self.head = R.Mx4(self.rows, HIDDEN)
        R.dense_copy(self.plan, d, trainer.weight_tab, R.BF16, self.tab)
        self.round_head()

    def round_head(self):
        R.mx4_quantize(self.weights[2].view(self.rows, HIDDEN), self.head)

    def receive(self, bucket):
        R.delta_apply(self.plan, self.d, bucket, self.tab)
        self.round_head()

    def rows_of(self, tokens):
        out = torch.empty(len(tokens), HIDDEN, dtype=torch.bfloat16, device="cuda")
        R.embedding_lookup(self.weights[0].view(self.rows, HIDDEN), tokens, out, scale=SCALE, first_row=self.d * self.rows)
        return out

    def logits(self, x):
        out = torch.empty(len(x), self.rows, dtype=torch.float32, device="cuda")
        ws = R.mx4_linear_workspace(len(x), self.rows, HIDDEN)
        R.mx4_linear(x * self.weights[1], self.head, out, ws)
        return out


def serve(shards, tokens):
    """Logits for tokens.  (The sum and the concatenation are what ranks would do by all-reduce and all-gather.)"""
    x = sum(s.rows_of(tokens) for s in shards)
    return torch.cat([s.logits(x) for s in shards], 1)


def batch(g, following):
    tokens = torch.randint(0, VOCAB, (TOKENS,), generator=g, device="cuda")
    return tokens, following[tokens]


def main(steps=40, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    following = torch.randperm(VOCAB, generator=g, device="cuda")      # the language: one word follows another
    trainer = Trainer(seed)
    shards = [Shard(trainer, d) for d in range(TP)]
    history = []
    for i in range(steps):
        loss, norm = trainer.step([batch(g, following) for _ in range(2)])
        for s, bucket in zip(shards, trainer.buckets):
            s.receive(bucket)
        entries = sum(R.bucket_check(trainer.plan, b) for b in trainer.buckets)
        history.append((loss, norm, entries))
        if i % 10 == 0 or i == steps - 1:
            print("step %3d  loss %.3f  norm of the gradients %.3f  %5.1f %% of the weights changed"
                  % (i, loss, norm, 100.0 * entries / (trainer.total + HIDDEN)), flush=True)    # (the norm weight goes to both)
    everyone = torch.arange(VOCAB, device="cuda")
    right = (serve(shards, everyone).argmax(1) == following).float().mean().item()
    word = everyone[5:6]
    alone = serve(shards, word)                                        # one token, as a decode step
    print("the receiver names the next word of %.1f %% of the words" % (100 * right), flush=True)
    return history, right, alone, trainer, shards


if __name__ == "__main__":
    main(*(int(v) for v in sys.argv[1:2]))
