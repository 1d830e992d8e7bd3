"""Layer norm, the layers and the losses run together, as the models of sage.py use them: their gradients against the same models in 64 bits
under torch's own differentiation, and short runs through the pipeline."""
import numpy as np
import pytest

from test_gpu_sage import torch      # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def gelu(torch, z):
    return 0.5 * z * (1 + torch.erf(z / 2 ** 0.5))


def layer_norm(x, w, b):
    m = x.mean(1, keepdim=True)
    return (x - m) / (((x - m) ** 2).mean(1, keepdim=True) + 1e-5).sqrt() * w + b


def small_batch(torch, dtype, rng):
    from paper_2112_08541_amd import binding as B, sage
    N, dim, types_n = 3000, 44, 3
    deg = rng.integers(0, 9, N)
    row_ptr = np.concatenate([[0], np.cumsum(deg)]).astype(np.int32)
    graph = B.Graph(row_ptr, rng.integers(0, N, row_ptr[-1]).astype(np.int32))
    sampler = B.Sampler(graph, 60, [4, 3])
    batch = sampler.sample(torch.from_numpy(rng.permutation(N)[:60].astype(np.int32)).cuda(), 7)
    torch.cuda.synchronize()
    blocks = sage.blocks_of(batch)
    n = blocks[-1][3]
    rows = torch.from_numpy(rng.standard_normal((n, 48)).astype(np.float32)).to(dtype).cuda()[:, :dim]
    types = torch.from_numpy(rng.integers(0, types_n, N).astype(np.int32)).cuda()
    return (graph, sampler, batch), rows, types, batch.input_nodes(n), blocks, dim, types_n


@pytest.mark.parametrize("name,tolerance", [("f32", 1e-5), ("bf16", 0.05)])
def test_normed_model_without_kept_scores(torch, name, tolerance):      # noqa: F811
    """tolerance: of the 2-norms; six layers one after the other, each off by some 2^-22 (fp32) or 2^-7 (bf16) of what it passes on."""
    from paper_2112_08541_amd import sage
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[name]
    rng = np.random.default_rng(4)
    _keep, rows, types, ids, blocks, dim, types_n = small_batch(torch, dtype, rng)
    m = sage.TypedSage([60, 300, 1200], dim, 40, 700, types_n, dtype, seed=6, norm=True, keep_scores=False)
    labels = torch.from_numpy(rng.integers(0, 700, 60)).cuda()
    h = m.hidden_rows(rows, types, ids, blocks)
    each, dh = sage.fused_loss(m.loss, h, m.w_out, m.b_out, labels.int())
    m._backward_hidden(dh)
    grads = [p.grad.double().cpu() for p in m.parameters()]

    v = {id(q): q.value.double().cpu().requires_grad_(True) for q in m.parameters()}
    p = lambda q: v[id(q)]      # noqa: E731
    x, t = rows.double().cpu(), types.cpu()[ids.long().cpu()]
    g = torch.zeros(len(t), 40, dtype=torch.float64)
    for k in range(types_n):
        at = torch.nonzero(t == k).squeeze(1)
        g = g.index_copy(0, at, x[at] @ p(m.w_in)[k].T + p(m.b_in)[k])
    g = gelu(torch, g)
    for hop in reversed(range(m.num_hops)):
        row_ptr, col, nd, ns = (a.cpu().long() if hasattr(a, "cpu") else a for a in blocks[hop])
        g = layer_norm(g[:ns], p(m.norm_w[hop]), p(m.norm_b[hop]))
        near = torch.stack([g[col[row_ptr[i]: row_ptr[i + 1]]].mean(0) if row_ptr[i + 1] > row_ptr[i] else torch.zeros(40, dtype=torch.float64) for i in range(nd)])
        g = gelu(torch, near @ p(m.w_near[hop]).T + g[:nd] @ p(m.w_self[hop]).T + p(m.b[hop]))
    z = g @ p(m.w_out).T + p(m.b_out)
    want = torch.logsumexp(z, 1) - z[torch.arange(60), labels.cpu()]
    want.mean().backward()
    off = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())      # noqa: E731
    assert off(each, want.detach()) <= tolerance
    for got, q in zip(grads, m.parameters()):
        assert off(got, p(q).grad) <= tolerance


@pytest.mark.parametrize("name,tolerance", [("f32", 1e-5), ("bf16", 0.04)])
def test_a_students_gradients(torch, name, tolerance):      # noqa: F811
    from paper_2112_08541_amd import sage
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[name]
    g = torch.Generator(device="cuda").manual_seed(3)
    n, dim, hidden, classes, top = 150, 44, 72, 330, 6
    s = sage.Student(200, dim, hidden, classes, top, temperature=2.0, label_share=0.3, dtype=dtype, seed=2)
    rows = (torch.randn((n, dim), generator=g, device="cuda") * 3 + 1).to(dtype)
    labels = torch.randint(-1, classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    teacher = sage.best_classes(torch.randn((n, classes), generator=g, device="cuda") * 3, top)
    each, dh = sage.fused_loss(s.loss, s.forward(rows), s.w_out, s.b_out, labels, teacher, 0.3)
    s.backward(dh)
    v = [p.value.double().cpu().requires_grad_(True) for p in s.parameters()]
    h = gelu(torch, layer_norm(rows.double().cpu(), v[0], v[1]) @ v[2].T + v[3])
    z = h @ v[4].T + v[5]
    lab = labels.cpu().long()
    by_label = torch.where(lab >= 0, torch.logsumexp(z, 1) - z[torch.arange(n), lab.clamp(min=0)], torch.zeros(1, dtype=torch.float64))
    p, logq = torch.softmax(teacher[1].double().cpu() / 2, 1), torch.log_softmax(z / 2, 1).gather(1, teacher[0].long().cpu())
    want = 0.3 * by_label + 0.7 * 4 * (p * (p.log() - logq)).sum(1)
    want.mean().backward()
    off = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())      # noqa: E731
    assert off(each, want.detach()) <= tolerance
    for q, w in zip(s.parameters(), v):
        assert off(q.grad, w.grad) <= tolerance


def test_a_model_and_its_student_through_the_pipeline(torch):      # noqa: F811
    from paper_2112_08541_amd import binding as B, inputs, sage
    from paper_2112_08541_amd.pipeline import MinibatchPipeline
    cfg = inputs.CONFIGS["tiny"]
    w = inputs.make_workload(cfg, pinned=True)
    graph = B.Graph(w.row_ptr, w.col)
    types, labels = sage.synthetic_task(w, 3, 4)
    bounds = [min(cfg.num_nodes, cfg.batch * int(np.prod([1 + f for f in cfg.fanouts[:h]]))) for h in range(len(cfg.fanouts) + 1)]
    seeds = torch.from_numpy(w.seed_batches).cuda()
    cache = B.Cache(cfg.cache_rows, w.features.ctypes.data, num_nodes=cfg.num_nodes, row_bytes=cfg.row_bytes)
    pipe = MinibatchPipeline(graph, cache, cfg.batch, cfg.fanouts, cfg.row_bytes)
    model = sage.TypedSage(bounds, cfg.feat_dim, 32, 4, 3, norm=True, keep_scores=False)
    history = sage.train(pipe, model, seeds, w.rng_seeds, 6, types, labels)
    assert history.shape == (6, 2) and np.isfinite(history).all()
    student = sage.Student(cfg.batch, cfg.feat_dim, 32, 4, top=3)
    losses = sage.train_student(pipe, model, student, seeds, w.rng_seeds, 4, types, labels, 3)
    assert losses.shape == (4,) and np.isfinite(losses).all()
