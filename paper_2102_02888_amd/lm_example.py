"""A small language model trained with both optimizers of this package:

    python -m paper_2102_02888_amd.lm_example [steps] [heads]

The token table (tied to the output), a bias and the vectors of the layer norms
belong to OnebitAdam, in one flat buffer; the hidden matrices belong to Muon, in
another.  n simulated workers see batches of their own.  A worker's table
gradient is the output product's, to which onebit_embedding_grad adds the
lookup's, both in the worker's row of OnebitAdam's gradients; the matrices'
gradients go to Muon's rows.  The tokens are synthetic: each is followed by one
of four others.  With heads, every layer begins with attention over the batch's
packed sequences; with a teacher, another model's best tokens are learned
instead of the ones that follow.
"""
import sys

import torch
import torch.nn.functional as F

from .attention import attention_workspace, onebit_attention_forward, onebit_attention_grad
from .embedding import embedding_workspace, onebit_embedding_forward, onebit_embedding_grad
from .loss import onebit_distill_grad, onebit_logprobs_forward, onebit_logprobs_grad
from .muon import MUON_SCALE_RMS, Matrices, Muon
from .norm import layer_norm_workspace, onebit_layer_norm_forward, onebit_layer_norm_grad
from .onebit import Plan
from .optimizer import OnebitAdam


def _once(name):
    """A gradient that is to be differentiated again is refused: the operators give none, and
    autograd would leave that part of the second derivative out."""
    if torch.is_grad_enabled():
        raise RuntimeError("%s is not differentiable twice (create_graph)" % name)


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, workspace):
        ctx.save_for_backward(x, weight)
        ctx.workspace = workspace
        y = torch.empty_like(x)
        onebit_layer_norm_forward(x, y, weight, bias)
        return y

    @staticmethod
    def backward(ctx, grad_y):
        _once("layer norm")
        x, weight = ctx.saved_tensors
        grads = [torch.empty_like(t) for t in (x, weight, weight)]
        onebit_layer_norm_grad(grad_y.contiguous(), x, grads[0], ctx.workspace, weight, *grads[1:])
        return (*grads, None)


class _Attention(torch.autograd.Function):
    """Causal attention; q, k and v are parts of a row, as one product gives them."""

    @staticmethod
    def forward(ctx, qkv, starts, heads, workspace):
        tokens, width = qkv.shape[0], qkv.shape[1] // 3
        sides = qkv.bfloat16().view(tokens, 3 * heads, width // heads)
        out = torch.empty_like(sides[:, :heads])
        lse = torch.empty(tokens, heads, device=qkv.device)
        onebit_attention_forward(*sides.split(heads, 1), starts, out, lse)
        ctx.save_for_backward(sides, out, lse, starts)
        ctx.workspace = workspace
        return out.view(tokens, width).to(qkv.dtype)

    @staticmethod
    def backward(ctx, grad_out):
        _once("attention")
        sides, out, lse, starts = ctx.saved_tensors
        heads, grad = out.shape[1], torch.empty_like(sides)
        onebit_attention_grad(grad_out.to(out.dtype).contiguous().view(out.shape),
                              *sides.split(heads, 1), out, lse, starts, *grad.split(heads, 1),
                              ctx.workspace)
        return grad.view(grad.shape[0], -1).to(grad_out.dtype), None, None, None


class Model:
    """Residual two-matrix layers between a tied embedding and its output; with
    heads, each behind a layer norm and an attention layer of its own."""

    def __init__(self, device, vocab=1000, width=128, layers=2, n_workers=4, tokens=512, seed=0,
                 heads=0, teacher=None, alternatives=8):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.vocab, self.width, self.tokens, self.n = vocab, width, tokens, n_workers
        self.heads, self.teacher = heads, teacher
        vectors = [width] * (4 * layers if heads else 0)
        self.plan = Plan([vocab * width, vocab] + vectors, n_workers)
        self.adam = OnebitAdam(self.plan, device, lr=3e-3, warmup_steps=40)
        shapes = ([(width, 3 * width), (width, width)] if heads else []) + \
            [(width, 4 * width), (4 * width, width)]
        self.mats = Matrices(shapes * layers)
        # (a matrix's rows are its inputs here, h @ a: not what the spectral scale is for)
        self.muon = Muon(self.mats, device, lr=0.005, scale=MUON_SCALE_RMS, n_workers=n_workers)
        self.table = self._table(self.adam.x)
        self.table.normal_(0.0, 0.05, generator=gen)
        self.matrices = [self.mats.view(self.muon.x, k) for k in range(len(shapes) * layers)]
        for m in self.matrices:
            m.normal_(0.0, m.shape[0] ** -0.5, generator=gen)
        for w in self._vectors(self.adam.x)[::2]:
            w.fill_(1.0)
        self.workspace = embedding_workspace(tokens, vocab, width, device)
        if heads:
            self.norm_workspace = layer_norm_workspace(tokens, width, device)
            self.attention_workspace = attention_workspace(tokens, heads, device)
            # three sequences of different lengths
            self.starts = torch.tensor([0, tokens // 8, tokens // 2, tokens], dtype=torch.int32,
                                       device=device)
        if teacher:
            self.best = torch.empty(tokens, alternatives, dtype=torch.int32, device=device)
            self.best_logprobs = torch.empty(tokens, alternatives, device=device)
        # the loss is a mean over the batch
        self.weights = torch.full((tokens,), 1.0 / tokens, device=device)
        self.scale = width ** 0.5
        self.next = torch.randint(vocab, (vocab, 4), device=device, generator=gen)
        self.gen = gen

    def _table(self, flat):
        return flat[:self.vocab * self.width].view(self.vocab, self.width)

    def _bias(self, flat):
        at = int(self.plan.tensor_off[1])
        return flat[at:at + self.vocab]

    def _vectors(self, flat):
        """Weight and bias of each layer norm, by turns."""
        return [flat[int(at):int(at) + self.width] for at in self.plan.tensor_off[2:]]

    def batch(self):
        """Tokens and what follows each of them."""
        ids = torch.randint(self.vocab, (self.tokens,), device=self.table.device,
                            generator=self.gen)
        pick = torch.randint(4, (self.tokens, 1), device=ids.device, generator=self.gen)
        return ids, self.next[ids].gather(1, pick)[:, 0]

    def logits(self, hidden, table, bias, mats, vectors):
        """The output for a batch whose embedding is `hidden`."""
        h, mats, vectors = hidden, iter(mats), iter(vectors)
        for qkv in mats:
            if self.heads:
                h = h + _Attention.apply(self._norm(h, vectors) @ qkv, self.starts, self.heads,
                                         self.attention_workspace) @ next(mats)
                h = h + F.relu(self._norm(h, vectors) @ next(mats)) @ next(mats)
            else:
                h = h + F.relu(h @ qkv) @ next(mats)
        h = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6)
        return h @ table.t() + bias

    def _norm(self, h, vectors):
        return _LayerNorm.apply(h, next(vectors), next(vectors), self.norm_workspace)

    def embed(self, ids):
        hidden = torch.empty(self.tokens, self.width, device=ids.device)
        onebit_embedding_forward(self.table, ids, hidden, scale=self.scale)
        return hidden

    def parameters(self):
        """table, bias, matrices, vectors."""
        return (self.table, self._bias(self.adam.x), self.matrices, self._vectors(self.adam.x))

    def loss(self, logits, ids, target):
        """The batch's loss, and the logits' gradient: minus the log-probability of what
        follows, or the divergence from the teacher's best alternatives."""
        value, grad = torch.empty(self.tokens, device=logits.device), torch.empty_like(logits)
        if self.teacher is None:
            onebit_logprobs_grad(logits, target, -self.weights, grad, logprobs=value)
            return -value.mean(), grad
        with torch.no_grad():
            theirs = self.teacher.logits(self.teacher.embed(ids), *self.teacher.parameters())
        onebit_logprobs_forward(theirs, None, None, top_ids=self.best,
                                top_logprobs=self.best_logprobs)
        onebit_distill_grad(logits, self.best, self.best_logprobs, self.weights, grad, loss=value)
        return value.mean(), grad

    def worker(self, i):
        """Worker i's loss on a batch of its own, and its gradients."""
        ids, target = self.batch()
        hidden = self.embed(ids).requires_grad_()
        table, bias, mats, vectors = self.parameters()
        table, bias, *rest = (t.detach().requires_grad_() for t in (table, bias, *mats, *vectors))
        logits = self.logits(hidden, table, bias, rest[:len(mats)], rest[len(mats):])
        loss, d_logits = self.loss(logits.detach(), ids, target)
        d_hidden, d_table, d_bias, *d_rest = torch.autograd.grad(
            logits, [hidden, table, bias, *rest], d_logits)
        row = self.adam.grads[i]
        self._table(row).copy_(d_table)
        onebit_embedding_grad(d_hidden, ids, self._table(row), self.workspace, scale=self.scale,
                              accumulate=True)
        self._bias(row).copy_(d_bias)
        for k, d in enumerate(d_rest[:len(mats)]):
            self.mats.view(self.muon.grads[i], k).copy_(d)
        for v, d in zip(self._vectors(row), d_rest[len(mats):]):
            v.copy_(d)
        return loss

    def step(self):
        """One step of both optimizers; returns the workers' mean loss."""
        loss = torch.stack([self.worker(i) for i in range(self.n)]).mean()
        self.adam.step()
        self.muon.step()
        return loss


def main(steps=200, heads=0):
    model = Model(torch.device("cuda", torch.cuda.current_device()), heads=heads)
    for step in range(1, steps + 1):
        loss = model.step()
        if step == 1 or step % 20 == 0:
            print("step %4d  loss %.4f  (%s)" % (step, float(loss), "warm-up"
                                                 if model.adam.in_warmup else "compressed"))
    return float(loss)


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:3]))
