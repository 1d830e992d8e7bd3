"""A GraphSAGE model over the batches this package prepares, for graphs whose nodes have types: what a training program does
with a batch once its rows are in HBM, with the library's layers (binding.Linear, RowGroups, Orthogonalizer).

  input layer    h = gelu(x W_t' + b_t), one weight per node type t (the feature spaces of, say, users and items differ)
  per hop        h_v = gelu(W_n mean(h of v's sampled neighbors) + (W_s h_v + b)): two layers, the second taking the first
                 as its residual before the activation
  head           class scores of the seeds

Hidden matrices are updated with momentum and orthogonalised updates, biases and the head with plain steps.  The neighbors' mean
and the loss are ordinary torch operations.

    python -m paper_2112_08541_amd.sage              # a few epochs on the `tiny` configuration, loss and accuracy per epoch
"""
from __future__ import annotations

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


class TypedSage:
    """max_nodes: bound on a batch's nodes per hop, seeds first (max_nodes[h] for frontier h, as a Sampler's cap_nodes)."""

    def __init__(self, max_nodes: Sequence[int], in_dim: int, hidden: int, num_classes: int, num_types: int,
                 dtype=torch.float32, lr: float = 0.02, head_lr: float = 0.3, beta: float = 0.9, seed: int = 0):
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
        self.head = B.Linear(max_nodes[0], hidden, num_classes, dtype)

    def parameters(self) -> List[_Matrix]:
        return [self.w_in, self.b_in, *self.w_self, *self.w_near, *self.b, self.w_out, self.b_out]

    def _empty(self, *shape) -> torch.Tensor:
        return torch.empty(shape, dtype=self.dtype, device="cuda")

    def forward(self, rows: torch.Tensor, types: torch.Tensor, ids: torch.Tensor, blocks) -> torch.Tensor:
        """rows: the batch's feature rows (n x in_dim); types: of every node of the graph (int32); ids: the batch's input nodes;
        blocks: per hop (row_ptr, col_local, destinations, sources).  Returns the seeds' class scores."""
        n = rows.shape[0]
        self.groups.build(types, ids=ids, n=n)
        h, saved = self._empty(n, self.hidden), self._empty(n, self.hidden)
        self.input.forward(rows, self.w_in.value, h, self.b_in.value, saved=saved, groups=self.groups)
        self._kept = [(rows, saved)]
        for hop in reversed(range(self.num_hops)):
            row_ptr, col, nd, ns = blocks[hop]
            mean, kept = neighbor_mean(h[:ns], row_ptr, col)
            own, out, saved = self._empty(nd, self.hidden), self._empty(nd, self.hidden), self._empty(nd, self.hidden)
            self.own[hop].forward(h[:nd], self.w_self[hop].value, own, self.b[hop].value)
            self.near[hop].forward(mean, self.w_near[hop].value, out, residual=own, saved=saved)
            self._kept.append((hop, h, mean, kept, saved, col, nd, ns))
            h = out
        scores = self._empty(h.shape[0], self.num_classes)
        self.head.forward(h, self.w_out.value, scores, self.b_out.value)
        self._last = h
        return scores

    def backward(self, dscores: torch.Tensor) -> None:
        """Fills every parameter's grad from the scores' gradient (the batch of the last forward call)."""
        dh = self._empty(*self._last.shape)
        self.head.backward(dscores, self._last, self.w_out.value, dx=dh, dweight=self.w_out.grad, dbias=self.b_out.grad)
        for hop, h, mean, kept, saved, col, nd, ns in reversed(self._kept[1:]):
            dmean, down, dself = self._empty(nd, self.hidden), self._empty(nd, self.hidden), self._empty(nd, self.hidden)
            self.near[hop].backward(dh, mean, self.w_near[hop].value, saved, dx=dmean, dweight=self.w_near[hop].grad, dresidual=down)
            self.own[hop].backward(down, h[:nd], self.w_self[hop].value, dx=dself, dweight=self.w_self[hop].grad, dbias=self.b[hop].grad)
            total = torch.zeros((ns, self.hidden), device="cuda")
            total[:nd] = dself
            neighbor_mean_backward(dmean, col, kept, total)
            dh = total.to(self.dtype)
        rows, saved = self._kept[0]
        self.input.backward(dh, rows, self.w_in.value, saved, dweight=self.w_in.grad, dbias=self.b_in.grad, groups=self.groups)

    def update(self) -> None:
        for p in self.parameters():
            p.step(self.lr if p.momentum is not None else self.head_lr, self.beta)

    def train_step(self, rows, types, ids, blocks, labels) -> torch.Tensor:
        """One step on a batch; labels: of the seeds (int64).  Returns (loss, correct predictions) on the device."""
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


def train(pipe, model: TypedSage, seeds: torch.Tensor, rng_seeds, steps: int, types: torch.Tensor, labels: torch.Tensor) -> np.ndarray:
    """Trains on `steps` batches of a MinibatchPipeline, or of a NativePipeline without a host tier (with one its sampling has a stream
    that only the library knows, which could not be kept off the batch in use); labels: of every node.  A batch's sampling workspace is
    read until its step has ended, so the sampling and map updates of later batches wait for that: preparation overlaps the
    fetch, not the training step.  Returns (loss, correct) per batch."""
    if isinstance(pipe, NativePipeline) and pipe.tier is not None:
        raise ValueError("train() cannot order a NativePipeline with a host tier: use a MinibatchPipeline")
    results = []

    def on_batch(_step, batch, n, p):
        # on the stream that carries the rows; later samplings, which reuse this batch's workspace, come behind it
        with torch.cuda.stream(p.chain):
            p.cache.wait_rows(p.chain)
            blocks = blocks_of(batch)
            ids = batch.input_nodes(n)
            rows = p.out_rows[:n].view(model.dtype)[:, : model.in_dim]
            results.append(model.train_step(rows, types, ids, blocks, labels[ids[: blocks[0][2]].long()]))
        for stream in (p.work, getattr(p, "samp_stream", None)):
            if stream is not None:
                stream.wait_stream(p.chain)
    torch.cuda.current_stream().synchronize()
    pipe.run(seeds, rng_seeds, steps, on_batch=on_batch)
    return torch.stack(results).cpu().numpy()


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


def main(epochs: int = 8, hidden: int = 64, num_types: int = 4, num_classes: int = 8) -> np.ndarray:
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
    return np.stack(history)


if __name__ == "__main__":
    main()
