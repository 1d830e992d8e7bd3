"""The model over prepared batches: its scores and gradients against the same model in 64 bits under torch's own
differentiation, and a short training run through the pipeline."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


def reference(torch, m, rows, types, ids, blocks):
    """Class scores and the parameters they were made from, in 64 bits on the CPU, by loops over the definition."""
    p = {id(q): q.value.double().cpu().requires_grad_(True) for q in m.parameters()}
    v = lambda q: p[id(q)]      # noqa: E731
    gelu = lambda z: 0.5 * z * (1 + torch.erf(z / 2 ** 0.5))      # noqa: E731
    x, t = rows.double().cpu(), types.cpu()[ids.long().cpu()]
    h = torch.zeros(len(t), m.hidden, dtype=torch.float64)
    for k in range(v(m.w_in).shape[0]):
        at = torch.nonzero(t == k).squeeze(1)
        h = h.index_copy(0, at, x[at] @ v(m.w_in)[k].T + v(m.b_in)[k])
    h = gelu(h)
    for hop in reversed(range(m.num_hops)):
        row_ptr, col, nd, ns = (a.cpu().long() if hasattr(a, "cpu") else a for a in blocks[hop])
        near = torch.stack([h[col[row_ptr[i]: row_ptr[i + 1]]].mean(0) if row_ptr[i + 1] > row_ptr[i] else torch.zeros(m.hidden, dtype=torch.float64)
                            for i in range(nd)])
        h = gelu(near @ v(m.w_near[hop]).T + h[:nd] @ v(m.w_self[hop]).T + v(m.b[hop]))
    return h @ v(m.w_out).T + v(m.b_out), [v(q) for q in m.parameters()]


@pytest.mark.parametrize("name,tolerance", [("f32", 1e-5), ("bf16", 0.04)])
def test_scores_and_gradients(torch, name, tolerance):
    """tolerance: of the 2-norms; five layers one after the other, each off by some 2^-22 (fp32) or 2^-7 (bf16: rows, weights and dz
    rounded to 2^-8 each) of what it passes on."""
    from paper_2112_08541_amd import binding as B, sage
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[name]
    rng = np.random.default_rng(3)
    N, dim, types_n, classes, hidden = 3000, 44, 3, 5, 40
    deg = rng.integers(0, 9, N)
    row_ptr = np.concatenate([[0], np.cumsum(deg)]).astype(np.int32)
    graph = B.Graph(row_ptr, rng.integers(0, N, row_ptr[-1]).astype(np.int32))
    sampler = B.Sampler(graph, 60, [4, 3])
    batch = sampler.sample(torch.from_numpy(rng.permutation(N)[:60].astype(np.int32)).cuda(), 7)
    torch.cuda.synchronize()
    blocks = sage.blocks_of(batch)
    n = blocks[-1][3]
    ids = batch.input_nodes(n)
    rows = torch.from_numpy(rng.standard_normal((n, 48)).astype(np.float32)).to(dtype).cuda()[:, :dim]
    types = torch.from_numpy(rng.integers(-1, types_n, N).astype(np.int32)).cuda()
    types[types < 0] = types_n - 1
    m = sage.TypedSage([60, 300, 1200], dim, hidden, classes, types_n, dtype, seed=5)
    scores = m.forward(rows, types, ids, blocks)
    d = torch.from_numpy(rng.standard_normal(tuple(scores.shape)).astype(np.float32)).to(dtype).cuda()
    m.backward(d)
    want, params = reference(torch, m, rows, types, ids, blocks)
    want.backward(d.double().cpu())
    off = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())      # noqa: E731
    assert off(scores, want.detach()) <= tolerance
    for p, q in zip(m.parameters(), params):
        assert off(p.grad, q.grad) <= tolerance


def test_training_through_the_pipeline(torch):
    from paper_2112_08541_amd import sage
    history = sage.main(epochs=5)
    assert np.isfinite(history).all()
    assert history[-1, 0] < 0.8 * history[0, 0] and history[-1, 1] > 1.3 * history[0, 1]


def test_both_loops_without_a_tier_train_alike(torch):
    """The sums of the neighbors' mean come in any order, so the losses of a few steps agree to some places only."""
    from paper_2112_08541_amd import binding as B, inputs, sage
    from paper_2112_08541_amd.pipeline import MinibatchPipeline, NativePipeline
    cfg = inputs.CONFIGS["tiny"]
    w = inputs.make_workload(cfg, pinned=True)
    graph = B.Graph(w.row_ptr, w.col)
    types, labels = sage.synthetic_task(w, 3, 4)
    bounds = [min(cfg.num_nodes, cfg.batch * int(np.prod([1 + f for f in cfg.fanouts[:h]]))) for h in range(len(cfg.fanouts) + 1)]
    seeds, losses = torch.from_numpy(w.seed_batches).cuda(), []
    for loop in (MinibatchPipeline, NativePipeline):
        cache = B.Cache(cfg.cache_rows, w.features.ctypes.data, num_nodes=cfg.num_nodes, row_bytes=cfg.row_bytes)
        pipe = loop(graph, cache, cfg.batch, cfg.fanouts, cfg.row_bytes)
        model = sage.TypedSage(bounds, cfg.feat_dim, 32, 4, 3)
        losses.append(sage.train(pipe, model, seeds, w.rng_seeds, 6, types, labels)[:, 0])
    assert np.isfinite(losses).all() and np.allclose(losses[0], losses[1], rtol=1e-3)
