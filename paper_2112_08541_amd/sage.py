"""A GraphSAGE model over the batches this package prepares, for graphs whose nodes have types: what a training program does
with a batch once its rows are in HBM, with the library's layers (binding.Linear, RowGroups, LayerNorm, ClassLoss, Orthogonalizer).

  input layer    h = gelu(x W_t' + b_t), one weight per node type t (the feature spaces of, say, users and items differ)
  per hop        h_v = gelu(W_n mean(h of v's sampled neighbors) + (W_s h_v + b)): two layers, the second taking the first
                 as its residual before the activation; with norm=True over the layer norm of h
  head           class scores of the seeds; with keep_scores=False their loss alone, for class counts whose scores are not to be kept

Hidden matrices are updated with momentum and orthogonalised updates, biases, norms and the head with plain steps.  The neighbors' mean
and, with scores, the loss are ordinary torch operations.  A Student is taught by such a model: from a node's own features, without its
neighbors, it learns the labels and the model's best classes.

    python -m paper_2112_08541_amd.sage              # a few epochs on the `tiny` configuration, loss and accuracy per epoch
    python -m paper_2112_08541_amd.sage --student    # and a student of the result
"""
from __future__ import annotations

import sys
from typing import List, Sequence

import numpy as np
import torch

from . import binding as B
from .pipeline import NativePipeline


def neighbor_mean(h: torch.Tensor, row_ptr: torch.Tensor, col: torch.Tensor):
    """Mean over each destination's sampled neighbors (zero without any), and what the backward pass needs of it."""
    degree = (row_ptr[1:] - row_ptr[:-1]).long()
    dst = torch.repeat_interleave(torch.arange(degree.numel(), device=h.device), degree, output_size=col.numel())
    share = degree.clamp(min=1).reciprocal().float()[:, None]
    total = torch.zeros((degree.numel(), h.shape[1]), dtype=torch.float32, device=h.device)
    total.index_add_(0, dst, h[col.long()].float())
    return (total * share).to(h.dtype), (dst, share)


def neighbor_mean_backward(d: torch.Tensor, col: torch.Tensor, kept, dh: torch.Tensor) -> None:
    """Adds the mean's gradient to dh (fp32)."""
    dst, share = kept
    dh.index_add_(0, col.long(), (d.float() * share)[dst])


class _Matrix:
    """A weight with its fp32 master, momentum and (hidden matrices) orthogonalised updates."""

    def __init__(self, shape, dtype, scale, generator, orthogonal):
        self.master = torch.randn(shape, generator=generator, device="cuda") * scale
        self.value = self.master.to(dtype)
        self.grad = torch.empty_like(self.value)
        self.momentum = torch.zeros_like(self.master) if orthogonal else None
        if orthogonal:
            lead = (1,) + tuple(shape) if len(shape) == 2 else tuple(shape)
            self.plan = B.Orthogonalizer(*lead)
            self.update = torch.empty(lead, device="cuda")

    def step(self, lr: float, beta: float) -> None:
        if self.momentum is None:
            self.master.add_(self.grad.float(), alpha=-lr)
        else:
            self.momentum.mul_(beta).add_(self.grad.float())
            self.plan.run(torch.add(self.grad.float(), self.momentum, alpha=beta).view(self.update.shape), self.update)
            rows, cols = self.master.shape[-2:]
            self.master.add_(self.update.view(self.master.shape), alpha=-lr * max(1.0, rows / cols) ** 0.5)
        self.value.copy_(self.master)


def _ones(make, width: int) -> _Matrix:
    m = make((width,), 0.0, False)
    m.master.fill_(1.0)
    m.value.copy_(m.master)
    return m


def fused_loss(loss: B.ClassLoss, h: torch.Tensor, weight: _Matrix, bias: _Matrix, labels, teacher=None, label_share: float = 1.0):
    """The rows' losses (label_share of the label's, the rest of the teacher's) and the gradient of their mean: that of h is returned, the
    others go to weight.grad and bias.grad."""
    n = h.shape[0]
    saved, dh = torch.empty((n, loss.saved_width), device="cuda"), torch.empty_like(h)
    by_label = torch.empty(n, device="cuda")
    by_teacher = None if teacher is None else torch.empty(n, device="cuda")
    loss.forward(h, weight.value, bias.value, labels=labels, teacher=teacher, loss=by_label, teacher_loss=by_teacher, saved=saved)
    loss.backward(h, weight.value, saved, bias.value, labels=labels, teacher=teacher, scale=label_share / n, teacher_scale=(1.0 - label_share) / n,
                  dx=dh, dweight=weight.grad, dbias=bias.grad)
    return by_label if teacher is None else label_share * by_label + (1.0 - label_share) * by_teacher, dh


def best_classes(scores: torch.Tensor, top: int):
    """What a Student learns of a model's class scores: each row's best classes (int32) and their scores."""
    best = scores.float().topk(min(top, scores.shape[1]), dim=1)
    return best.indices.int(), best.values.contiguous()


class Student:
    """Classes from a node's own features: layer norm, a hidden layer with gelu, and a head whose scores are not kept; learns labels and a
    teacher's `top` best classes."""

    def __init__(self, max_rows: int, in_dim: int, hidden: int, num_classes: int, top: int, temperature: float = 2.0, label_share: float = 0.5,
                 dtype=torch.float32, lr: float = 0.02, head_lr: float = 0.3, beta: float = 0.9, seed: int = 0):
        self.lr, self.head_lr, self.beta, self.label_share, self.dtype = lr, head_lr, beta, label_share, dtype
        g = torch.Generator(device="cuda").manual_seed(seed)
        make = lambda shape, scale, orthogonal: _Matrix(shape, dtype, scale, g, orthogonal)      # noqa: E731
        self.norm, self.norm_w, self.norm_b = B.LayerNorm(max_rows, in_dim, dtype), _ones(make, in_dim), make((in_dim,), 0.0, False)
        self.layer, self.w, self.b = B.Linear(max_rows, in_dim, hidden, dtype, activation="gelu"), make((hidden, in_dim), in_dim ** -0.5, True), make((hidden,), 0.0, False)
        self.loss = B.ClassLoss(max_rows, hidden, num_classes, dtype, top=top, temperature=temperature)
        self.w_out, self.b_out = make((num_classes, hidden), hidden ** -0.5, False), make((num_classes,), 0.0, False)

    def parameters(self) -> List[_Matrix]:
        return [self.norm_w, self.norm_b, self.w, self.b, self.w_out, self.b_out]

    def forward(self, rows: torch.Tensor) -> torch.Tensor:
        """The rows' last hidden rows."""
        n = rows.shape[0]
        normed, moments = torch.empty((n, rows.shape[1]), dtype=self.dtype, device="cuda"), torch.empty((n, 2), device="cuda")
        self.norm.forward(rows, normed, self.norm_w.value, self.norm_b.value, saved=moments)
        h, z = (torch.empty((n, self.layer.out_dim), dtype=self.dtype, device="cuda") for _ in range(2))
        self.layer.forward(normed, self.w.value, h, self.b.value, saved=z)
        self._kept = rows, normed, moments, z
        return h

    def backward(self, dh: torch.Tensor) -> None:
        """Fills the grads of all but the head from the last hidden rows' gradient."""
        rows, normed, moments, z = self._kept
        d = torch.empty_like(normed)
        self.layer.backward(dh, normed, self.w.value, z, dx=d, dweight=self.w.grad, dbias=self.b.grad)
        self.norm.backward(d, rows, moments, weight=self.norm_w.value, dweight=self.norm_w.grad, dbias=self.norm_b.grad)

    def train_step(self, rows: torch.Tensor, labels: torch.Tensor, teacher) -> torch.Tensor:
        """One step; labels: int32, outside the classes for rows without one.  Returns the mean loss on the device."""
        each, dh = fused_loss(self.loss, self.forward(rows), self.w_out, self.b_out, labels, teacher, self.label_share)
        self.backward(dh)
        for p in self.parameters():
            p.step(self.lr if p.momentum is not None else self.head_lr, self.beta)
        return each.mean()


class TypedSage:
    """max_nodes: bound on a batch's nodes per hop, seeds first (max_nodes[h] for frontier h, as a Sampler's cap_nodes)."""

    SCORES_AT_A_TIME = B.BGL_MAX_DIM     # classes whose scores best_classes() has in memory


    def __init__(self, max_nodes: Sequence[int], in_dim: int, hidden: int, num_classes: int, num_types: int,
                 dtype=torch.float32, lr: float = 0.02, head_lr: float = 0.3, beta: float = 0.9, seed: int = 0,
                 norm: bool = False, keep_scores: bool = True):
        self.num_hops, self.in_dim, self.hidden, self.num_classes, self.dtype = len(max_nodes) - 1, in_dim, hidden, num_classes, dtype
        self.lr, self.head_lr, self.beta = lr, head_lr, beta
        g = torch.Generator(device="cuda").manual_seed(seed)
        make = lambda shape, scale, orthogonal: _Matrix(shape, dtype, scale, g, orthogonal)      # noqa: E731
        self.w_in, self.b_in = make((num_types, hidden, in_dim), in_dim ** -0.5, True), make((num_types, hidden), 0.0, False)
        self.w_self: List[_Matrix] = [make((hidden, hidden), hidden ** -0.5, True) for _ in range(self.num_hops)]
        self.w_near: List[_Matrix] = [make((hidden, hidden), hidden ** -0.5, True) for _ in range(self.num_hops)]
        self.b: List[_Matrix] = [make((hidden,), 0.0, False) for _ in range(self.num_hops)]
        self.w_out, self.b_out = make((num_classes, hidden), hidden ** -0.5, False), make((num_classes,), 0.0, False)
        self.groups = B.RowGroups(max_nodes[-1], num_types)
        self.input = B.Linear(max_nodes[-1], in_dim, hidden, dtype, activation="gelu", num_groups=num_types)
        self.own = [B.Linear(max_nodes[h], hidden, hidden, dtype) for h in range(self.num_hops)]
        self.near = [B.Linear(max_nodes[h], hidden, hidden, dtype, activation="gelu", residual="before") for h in range(self.num_hops)]
        # (a layer has BGL_MAX_DIM columns at most, a loss without kept scores more classes)
        self.head = B.Linear(max_nodes[0], hidden, num_classes, dtype) if keep_scores or num_classes <= B.BGL_MAX_DIM else None
        self.max_seeds = max_nodes[0]
        self.norms = [B.LayerNorm(max_nodes[h + 1], hidden, dtype) for h in range(self.num_hops)] if norm else []
        self.norm_w, self.norm_b = [_ones(make, hidden) for _ in self.norms], [make((hidden,), 0.0, False) for _ in self.norms]
        self.loss = None if keep_scores else B.ClassLoss(max_nodes[0], hidden, num_classes, dtype)

    def parameters(self) -> List[_Matrix]:
        return [self.w_in, self.b_in, *self.w_self, *self.w_near, *self.b, self.w_out, self.b_out, *self.norm_w, *self.norm_b]

    def _empty(self, *shape) -> torch.Tensor:
        return torch.empty(shape, dtype=self.dtype, device="cuda")

    def forward(self, rows: torch.Tensor, types: torch.Tensor, ids: torch.Tensor, blocks) -> torch.Tensor:
        """rows: the batch's feature rows (n x in_dim); types: of every node of the graph (int32); ids: the batch's input nodes;
        blocks: per hop (row_ptr, col_local, destinations, sources).  Returns the seeds' class scores."""
        if self.head is None:
            raise ValueError(f"the scores of {self.num_classes} classes are not kept: best_classes() has the best ones")
        h = self.hidden_rows(rows, types, ids, blocks)
        scores = self._empty(h.shape[0], self.num_classes)
        self.head.forward(h, self.w_out.value, scores, self.b_out.value)
        return scores

    def best_classes(self, rows: torch.Tensor, types: torch.Tensor, ids: torch.Tensor, blocks, top: int):
        """Each seed's best classes (int32) and their scores, as best_classes() of forward()'s; scores are made for some classes at a time, so that memory does not grow with
        their number."""
        h, best = self.hidden_rows(rows, types, ids, blocks), None
        for first in range(0, self.num_classes, self.SCORES_AT_A_TIME):
            some = slice(first, min(first + self.SCORES_AT_A_TIME, self.num_classes))
            scores = self._empty(h.shape[0], some.stop - first)
            head = self.head if scores.shape[1] == self.num_classes else B.Linear(self.max_seeds, self.hidden, scores.shape[1], self.dtype)
            head.forward(h, self.w_out.value[some], scores, self.b_out.value[some])
            classes, values = best_classes(scores, top)
            classes += first
            if best is not None:
                classes, values = torch.cat([best[0], classes], 1), torch.cat([best[1], values], 1)
                at, values = best_classes(values, top)
                classes = classes.gather(1, at.long())
            best = classes, values
        return best

    def hidden_rows(self, rows: torch.Tensor, types: torch.Tensor, ids: torch.Tensor, blocks) -> torch.Tensor:
        """The seeds' last hidden rows, from which forward() makes scores."""
        n = rows.shape[0]
        self.groups.build(types, ids=ids, n=n)
        h, saved = self._empty(n, self.hidden), self._empty(n, self.hidden)
        self.input.forward(rows, self.w_in.value, h, self.b_in.value, saved=saved, groups=self.groups)
        self._kept = [(rows, saved)]
        for hop in reversed(range(self.num_hops)):
            row_ptr, col, nd, ns = blocks[hop]
            raw = moments = None
            if self.norms:
                raw, h, moments = h[:ns], self._empty(ns, self.hidden), torch.empty((ns, 2), device="cuda")
                self.norms[hop].forward(raw, h, self.norm_w[hop].value, self.norm_b[hop].value, saved=moments)
            mean, kept = neighbor_mean(h[:ns], row_ptr, col)
            own, out, saved = self._empty(nd, self.hidden), self._empty(nd, self.hidden), self._empty(nd, self.hidden)
            self.own[hop].forward(h[:nd], self.w_self[hop].value, own, self.b[hop].value)
            self.near[hop].forward(mean, self.w_near[hop].value, out, residual=own, saved=saved)
            self._kept.append((hop, h, mean, kept, saved, col, nd, ns, raw, moments))
            h = out
        self._last = h
        return h

    def backward(self, dscores: torch.Tensor) -> None:
        """Fills every parameter's grad from the scores' gradient (the batch of the last forward call)."""
        dh = self._empty(*self._last.shape)
        self.head.backward(dscores, self._last, self.w_out.value, dx=dh, dweight=self.w_out.grad, dbias=self.b_out.grad)
        self._backward_hidden(dh)

    def _backward_hidden(self, dh: torch.Tensor) -> None:
        for hop, h, mean, kept, saved, col, nd, ns, raw, moments in reversed(self._kept[1:]):
            dmean, down, dself = self._empty(nd, self.hidden), self._empty(nd, self.hidden), self._empty(nd, self.hidden)
            self.near[hop].backward(dh, mean, self.w_near[hop].value, saved, dx=dmean, dweight=self.w_near[hop].grad, dresidual=down)
            self.own[hop].backward(down, h[:nd], self.w_self[hop].value, dx=dself, dweight=self.w_self[hop].grad, dbias=self.b[hop].grad)
            total = torch.zeros((ns, self.hidden), device="cuda")
            total[:nd] = dself
            neighbor_mean_backward(dmean, col, kept, total)
            dh = total.to(self.dtype)
            if self.norms:
                self.norms[hop].backward(dh, raw, moments, weight=self.norm_w[hop].value, dx=dh, dweight=self.norm_w[hop].grad, dbias=self.norm_b[hop].grad)
        rows, saved = self._kept[0]
        self.input.backward(dh, rows, self.w_in.value, saved, dweight=self.w_in.grad, dbias=self.b_in.grad, groups=self.groups)

    def update(self) -> None:
        for p in self.parameters():
            p.step(self.lr if p.momentum is not None else self.head_lr, self.beta)

    def train_step(self, rows, types, ids, blocks, labels) -> torch.Tensor:
        """One step on a batch; labels: of the seeds (int64).  Returns (loss, correct predictions) on the device; without kept scores (loss,
        seeds whose label has more than half of the model's belief)."""
        if self.loss is not None:
            h = self.hidden_rows(rows, types, ids, blocks)
            each, dh = fused_loss(self.loss, h, self.w_out, self.b_out, labels.int())
            self._backward_hidden(dh)
            self.update()
            return torch.stack([each.mean(), (each < 0.6931472).sum().float()])
        scores = self.forward(rows, types, ids, blocks).float()
        logp = torch.log_softmax(scores, 1)
        loss = -logp[torch.arange(len(labels), device="cuda"), labels].mean()
        d = logp.exp()
        d[torch.arange(len(labels), device="cuda"), labels] -= 1.0
        self.backward((d / len(labels)).to(self.dtype))
        self.update()
        return torch.stack([loss, (scores.argmax(1) == labels).sum().float()])


def blocks_of(batch: B.SampledBatch):
    """Per hop (row_ptr, col_local, destinations, sources) of a sampled batch whose sizes are on the host."""
    nodes, edges = (a.tolist() for a in batch.sizes())
    return [(batch.row_ptr(h, nodes[h]), batch.col_local(h, edges[h]), nodes[h], nodes[h + 1]) for h in range(len(edges))]


def _over_batches(pipe, model: TypedSage, seeds, rng_seeds, steps, step_on) -> list:
    """step_on(rows, ids, blocks) on each prepared batch, in stream order; its results."""
    if isinstance(pipe, NativePipeline) and pipe.tier is not None:
        raise ValueError("train() cannot order a NativePipeline with a host tier: use a MinibatchPipeline")
    results = []

    def on_batch(_step, batch, n, p):
        # on the stream that carries the rows; later samplings, which reuse this batch's workspace, come behind it
        with torch.cuda.stream(p.chain):
            p.cache.wait_rows(p.chain)
            blocks = blocks_of(batch)
            rows = p.out_rows[:n].view(model.dtype)[:, : model.in_dim]
            results.append(step_on(rows, batch.input_nodes(n), blocks))
        for stream in (p.work, getattr(p, "samp_stream", None)):
            if stream is not None:
                stream.wait_stream(p.chain)
    torch.cuda.current_stream().synchronize()
    pipe.run(seeds, rng_seeds, steps, on_batch=on_batch)
    return results


def train(pipe, model: TypedSage, seeds: torch.Tensor, rng_seeds, steps: int, types: torch.Tensor, labels: torch.Tensor) -> np.ndarray:
    """Trains on `steps` batches of a MinibatchPipeline, or of a NativePipeline without a host tier (with one its sampling has a stream
    that only the library knows, which could not be kept off the batch in use); labels: of every node.  A batch's sampling workspace is
    read until its step has ended, so the sampling and map updates of later batches wait for that: preparation overlaps the
    fetch, not the training step.  Returns (loss, correct) per batch."""
    step = lambda rows, ids, blocks: model.train_step(rows, types, ids, blocks, labels[ids[: blocks[0][2]].long()])      # noqa: E731
    return torch.stack(_over_batches(pipe, model, seeds, rng_seeds, steps, step)).cpu().numpy()


def train_student(pipe, model: TypedSage, student: Student, seeds: torch.Tensor, rng_seeds, steps: int, types: torch.Tensor, labels: torch.Tensor,
                  top: int) -> np.ndarray:
    """Teaches the student on the seeds of `steps` batches (pipe as in train()): their own rows, their labels (of every node), and the best `top` classes of the
    model's scores.  Returns the loss per batch."""
    def step(rows, ids, blocks):
        n = blocks[0][2]
        return student.train_step(rows[:n], labels[ids[:n].long()].int(), model.best_classes(rows, types, ids, blocks, top))
    return torch.stack(_over_batches(pipe, model, seeds, rng_seeds, steps, step)).cpu().numpy()


def synthetic_task(w, num_types: int, num_classes: int, seed: int = 0):
    """Node types (random) and labels that the features decide, differently for each type."""
    rng = np.random.default_rng(seed)
    n, dim = w.cfg.num_nodes, w.cfg.feat_dim
    types = rng.integers(0, num_types, n).astype(np.int32)
    feats = np.asarray(w.features[:, :dim], dtype=np.float32)
    teachers = rng.standard_normal((num_types, num_classes, dim)).astype(np.float32)
    labels = np.empty(n, dtype=np.int64)
    for t in range(num_types):
        labels[types == t] = (feats[types == t] @ teachers[t].T).argmax(1)
    return torch.from_numpy(types).cuda(), torch.from_numpy(labels).cuda()


def main(epochs: int = 8, hidden: int = 64, num_types: int = 4, num_classes: int = 8, student_epochs: int = 0) -> np.ndarray:
    from . import inputs
    from .pipeline import MinibatchPipeline
    cfg = inputs.CONFIGS["tiny"]
    w = inputs.make_workload(cfg, pinned=True)
    graph = B.Graph(w.row_ptr, w.col)
    cache = B.Cache(cfg.cache_rows, w.features.ctypes.data, num_nodes=cfg.num_nodes, row_bytes=cfg.row_bytes)
    pipe = MinibatchPipeline(graph, cache, cfg.batch, cfg.fanouts, cfg.row_bytes)
    types, labels = synthetic_task(w, num_types, num_classes)
    bounds = [min(cfg.num_nodes, cfg.batch * int(np.prod([1 + f for f in cfg.fanouts[:h]]))) for h in range(len(cfg.fanouts) + 1)]
    model = TypedSage(bounds, cfg.feat_dim, hidden, num_classes, num_types)
    seeds = torch.from_numpy(w.seed_batches).cuda()
    per_epoch = seeds.shape[0]
    history = []
    for epoch in range(epochs):
        r = train(pipe, model, seeds, np.asarray(w.rng_seeds) + epoch, per_epoch, types, labels)
        history.append(r.mean(0))
        print(f"epoch {epoch}: loss {r[:, 0].mean():.4f}, accuracy {r[:, 1].mean() / cfg.batch:.3f}", flush=True)
    if student_epochs:
        student = Student(cfg.batch, cfg.feat_dim, hidden, num_classes, top=4)
        for epoch in range(student_epochs):
            r = train_student(pipe, model, student, seeds, np.asarray(w.rng_seeds) + epoch, per_epoch, types, labels, 4)
            print(f"student, epoch {epoch}: loss {r.mean():.4f}", flush=True)
    return np.stack(history)


if __name__ == "__main__":
    main(student_epochs=8 if "--student" in sys.argv[1:] else 0)
