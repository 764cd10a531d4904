"""The vocabulary loss's gradients under a gradient of the loss that is not finite (a loss scale that overflowed): rows without
a label get zeros whatever it is, and without any labelled row so does dweight."""

import pytest

from gpu_common import say
from test_gpu_training_use import Loss

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def tr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_23087_amd import training
    return training


def operands(rows, hidden, vocab, dtype):
    gen = torch.Generator().manual_seed(rows)
    return torch.randn(rows, hidden, generator=gen).to(dtype).cuda(), torch.randn(vocab, hidden, generator=gen).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("scale", [float("inf"), float("-inf"), float("nan")])
def test_rows_without_a_label_get_zeros(tr, scale, dtype):
    say(f"case gradient of the loss {scale} {dtype}")
    x, w = operands(300, 72, 500, dtype)
    labels = torch.where(torch.arange(300) % 3 == 0, torch.arange(300) % 500, -100).int().cuda()
    t = Loss(tr, x, w, labels).forward()
    t.dloss.fill_(scale)
    t.backward()
    has = labels >= 0
    assert bool((t.dx[~has] == 0).all())
    assert not bool(torch.isfinite(t.dx[has]).any()) and not bool(torch.isfinite(t.dw).any())


@pytest.mark.parametrize("scale", [float("inf"), float("nan")])
def test_no_labelled_row(tr, scale):
    say(f"case gradient of the loss {scale}, no labelled row")
    x, w = operands(70, 72, 500, torch.bfloat16)
    t = Loss(tr, x, w, torch.full((70,), -1, dtype=torch.int32, device="cuda"), f32=True).forward()
    t.dloss.fill_(scale)
    t.backward()
    assert float(t.loss) == 0 and bool((t.dx == 0).all()) and bool((t.dw == 0).all())
    t.dw.fill_(3.0)
    tr.vocab_loss_backward(t.x, t.w, t.labels, t.lse, t.dloss, None, t.dw, t.space, accumulate=True)
    assert bool((t.dw == 3).all())
    half = torch.full_like(w, 3.0)
    tr.vocab_loss_backward(t.x, t.w, t.labels, t.lse, t.dloss, None, half, t.space, reduction="sum")
    assert bool((half == 0).all())
