"""The gradient of the vocabulary loss at a row's own label: minus the probability of all other classes, which has to keep its
relative accuracy where the label is nearly certain, and enters dx and dweight unrounded. The logits here are exact, so the
errors are those of exponentials and sums (training_ref.py: a probability's exponent loses 4 u (|z| + |lse| + 16))."""

import numpy as np
import pytest

from gpu_common import say
import training_ref as ref
from test_gpu_training_use import Loss

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

FLUSHED = 2.0 ** -126             # an exponential below it is 0


@pytest.fixture(scope="module")
def tr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_23087_amd import training
    return training


def certain(logit, vocab, label, rows, dtype):
    """x and weight of rows whose label has this logit and all other classes 0; column 1 of the weight is 1 for the others."""
    w = torch.zeros(vocab, 8)
    w[:, 1] = 1.0
    w[label, 0], w[label, 1] = logit, 0.0
    x = torch.zeros(rows, 8)
    x[:, 0] = 1.0
    return x.to(dtype).cuda(), w.to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,vocab", [(1, 152064), (3, 1000), (300, 1000), (700, 70001)])
@pytest.mark.parametrize("logit", [10.0, 27.75, 45.25, 250.0])
def test_gradient_of_a_nearly_certain_label(tr, logit, rows, vocab, dtype):
    say(f"case label's logit {logit}, {rows} rows, {vocab} classes, {dtype}")
    label = vocab * 2 // 3
    x, w = certain(logit, vocab, label, rows, dtype)
    t = Loss(tr, x, w, torch.full((rows,), label, dtype=torch.int32, device="cuda"), f32=True)
    t.forward()
    t.dloss.fill_(float(rows))                     # each row's own gradient, whatever the number of rows
    t.backward()
    loss = np.log1p((vocab - 1) * np.exp(-logit))
    want, lse = float(np.expm1(-loss)), logit + loss
    share = np.expm1(4 * ref.U * (logit + lse + 16)) + ref.slack(vocab) + 16 * ref.U
    error = share * abs(want) + FLUSHED
    for column, value in ((0, want * logit), (1, -want)):
        # the others' gradients, in column 1, are rounded to 16 bits (f16: in steps of 2^-36) before their product
        e = error * logit if column == 0 else error + ref.HALF_ULP[dtype] * abs(want) + (2.0 ** -37 * vocab if dtype == torch.float16 else 0)
        bound = e + ref.HALF_ULP[dtype] * (abs(value) + e) + ref.TINY[dtype]
        assert float((t.dx[:, column].double() - value).abs().max()) <= bound, (column, value, t.dx[:3, column])
    got = float(t.dw[label, 0])
    assert abs(got - want * rows) <= error * rows + (ref.slack(rows) + 4 * ref.U) * abs(want) * rows, (got, want * rows)
    assert got <= 0


def test_gradient_of_nearly_certain_labels_over_pieces(tr):
    """A gradient of the logits of several pieces, labels in all of them, of one row and of many: for most of a step's time a
    row's other classes are not all known."""
    rows, vocab, logit = 3000, 200003, 27.75
    say(f"case labels' logits {logit}, {rows} rows, {vocab} classes")
    labels = torch.tensor([0, 17, 99999, 100200, 200002])[torch.arange(rows) % 5]
    labels[::7] = 150000
    x, w = torch.zeros(rows, 8), torch.zeros(vocab, 8)
    for c, v in enumerate(labels.unique().tolist()):
        w[v, c] = logit
        x[labels == v, c] = 1.0
    t = Loss(tr, x.bfloat16().cuda(), w.bfloat16().cuda(), labels.int().cuda(), f32=True).forward()
    t.dloss.fill_(float(rows))
    t.backward()
    loss = np.log1p((vocab - 1) * np.exp(-logit))
    want = np.expm1(-loss)
    share = np.expm1(4 * ref.U * (2 * logit + 16)) + ref.slack(vocab) + 16 * ref.U
    dx, dw = t.dx.cpu().double(), t.dw.cpu().double()
    for c, v in enumerate(labels.unique().tolist()):
        mine = labels == v
        value = want * logit
        assert float((dx[mine, c] - value).abs().max()) <= (share + ref.HALF_ULP[torch.bfloat16] * (1 + share)) * abs(value)
        m = int(mine.sum())
        assert abs(float(dw[v, c]) - want * m) <= (share + ref.slack(m)) * abs(want) * m, (v, float(dw[v, c]), want * m)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_weight_gradient_at_the_label_is_not_rounded(tr, dtype):
    """With weights of 0 and 3 classes the label's gradient is 1 / 3 - 1, which no 16-bit type has: a class's row of dweight is
    that times the row that has it as its label, to f32's accuracy (64 roundings allowed), in f32 and rounded once to 16 bits."""
    x = torch.linspace(-3, 3, 2 * 264).reshape(2, 264).to(dtype)
    w = torch.zeros(3, 264, dtype=dtype)
    want = -2 / 3 * x[0].double()
    t = Loss(tr, x[:1].cuda(), w.cuda(), torch.tensor([1], dtype=torch.int32, device="cuda"), f32=True).forward().backward()
    over = (t.dw[1].cpu().double() - want).abs() - (64 * ref.U * want.abs() + ref.TINY[torch.float32])
    assert float(over.max()) <= 0, float(over.max())
    # in 16 bits what values this close to it are rounded to, and nothing else
    t = Loss(tr, x[:1].cuda(), w.cuda(), torch.tensor([1], dtype=torch.int32, device="cuda")).forward().backward()
    ends = [(want * (1 + s * 64 * ref.U)).float().to(dtype) for s in (-1, 1)]
    got = t.dw[1].cpu()
    assert bool(((got == ends[0]) | (got == ends[1])).all()), float((got.double() - want).abs().max())
    # two rows with the same label, and a row without one between them
    x = torch.stack([x[0], torch.full_like(x[0], float("nan")), x[1]])
    t = Loss(tr, x.cuda(), w.cuda(), torch.tensor([2, -1, 2], dtype=torch.int32, device="cuda"), f32=True).forward().backward()
    want = -1 / 3 * (x[0].double() + x[2].double())
    over = (t.dw[2].cpu().double() - want).abs() - 64 * ref.U * (x[0].double().abs() + x[2].double().abs())
    assert float(over.max()) <= 0, float(over.max())


@pytest.mark.parametrize("rows,vocab", [(600, 1), (600, 3), (3000, 700), (65, 100000), (5000, 40000), (1400, 1), (5000, 1), (9000, 2),
                                        (6000, 30)])
def test_rows_of_one_class_are_added_in_order(tr, rows, vocab):
    """Labels that many rows share, few share and none share: dweight against 64 bits, and the same bits every time."""
    from test_gpu_training import loss_case, run_loss
    say(f"case shared labels {rows} x 72 x {vocab}")
    gen = np.random.default_rng([rows, vocab])
    x, w, lab = loss_case(gen, rows, 72, vocab, torch.bfloat16, "some")
    lab[lab >= 0] = torch.from_numpy((vocab * gen.random(int((lab >= 0).sum())) ** 3).astype(np.int32))
    gx, gw, gl, space, loss, lse, count, dx, dw, d, red = run_loss(tr, x, w, lab, torch.bfloat16, 0, True, 0.75, True)
    f = ref.vocab_loss(x, w, lab)
    assert int(count) == len(f["rows"])
    (want_x, want_w), (e_x, e_w) = ref.vocab_gradients(x, w, lab, lse.cpu(), 0.75)
    ref.check(dx, want_x, ref.rounded(want_x, dx.dtype, e_x), "dx")
    ref.check(dw, want_w, e_w, "dweight")
    again = torch.zeros_like(dw)
    tr.vocab_loss_backward(gx, gw, gl, lse, d, None, again, space, reduction=red)
    assert torch.equal(again, dw)
    tr.vocab_loss_backward(gx, gw, gl, lse, d, None, again, space, reduction=red, accumulate=True)
    assert torch.equal(again, 2 * dw)
