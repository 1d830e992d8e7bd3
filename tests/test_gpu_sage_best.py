"""The classes that a model teaches a student, without all scores in memory."""
import numpy as np
import pytest

from test_gpu_sage import torch      # noqa: F401  (the fixture)
from test_gpu_sage_losses import small_batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,tolerance", [("f32", 1e-5), ("bf16", 2.0 ** -7)])
@pytest.mark.parametrize("classes,top", [(700, 5), (16_384, 3), (16_385, 4), (70_001, 32)])
def test_best_classes_of_a_model(torch, name, tolerance, classes, top):      # noqa: F811
    """The best of all of them: fp32 sums of 40 terms, or a bf16's rounding (two kinds of it for classes as good as each other)."""
    from paper_2112_08541_amd import sage
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[name]
    _keep, rows, types, ids, blocks, dim, types_n = small_batch(torch, dtype, np.random.default_rng(5))
    m = sage.TypedSage([60, 300, 1200], dim, 40, classes, types_n, dtype, seed=7, norm=True, keep_scores=False)
    m.b_out.value.copy_(torch.randn(classes, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda"))
    scores = m.hidden_rows(rows, types, ids, blocks).double() @ m.w_out.value.double().t() + m.b_out.value.double()
    want = scores.topk(top, 1).values
    if classes <= m.SCORES_AT_A_TIME:
        assert (m.forward(rows, types, ids, blocks).double() - scores).abs().max() <= tolerance * scores.abs().max()
    else:
        with pytest.raises(ValueError, match="not kept"):
            m.forward(rows, types, ids, blocks)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    best, values = m.best_classes(rows, types, ids, blocks, top)
    if classes > 4 * m.SCORES_AT_A_TIME:
        hidden = 3 * 1_500 * (40 * 4 + 8) * 4      # rows of the hops, what they keep, means and their indices
        assert torch.cuda.max_memory_allocated() - before < 60 * classes * 4 + hidden
    assert best.shape == values.shape == (60, top) and best.dtype is torch.int32
    size = scores.abs().max()
    assert (values - want).abs().max() <= tolerance * size
    assert (scores.gather(1, best.long()) - values).abs().max() <= tolerance * size
    assert all(len(set(r)) == top for r in best.tolist())


def test_training_with_more_classes_than_a_layer_has_columns(torch):      # noqa: F811
    """A class for every item, and a student of them: losses are numbers, and every gradient is written."""
    from paper_2112_08541_amd import sage
    classes = 20_003
    rng = np.random.default_rng(6)
    _keep, rows, types, ids, blocks, dim, types_n = small_batch(torch, torch.float32, rng)
    m = sage.TypedSage([60, 300, 1200], dim, 40, classes, types_n, torch.float32, seed=7, norm=True, keep_scores=False)
    labels = torch.from_numpy(rng.integers(0, classes, 60)).cuda()
    for p in m.parameters():
        p.grad.fill_(float("nan"))
    loss = m.train_step(rows, types, ids, blocks, labels)[0]
    assert loss.isfinite() and all(p.grad.isfinite().all() for p in m.parameters())
    student = sage.Student(60, dim, 24, classes, 8)
    for p in student.parameters():
        p.grad.fill_(float("nan"))
    loss = student.train_step(rows[:60].contiguous(), labels.int(), m.best_classes(rows, types, ids, blocks, 8))
    assert loss.isfinite() and all(p.grad.isfinite().all() for p in student.parameters())
