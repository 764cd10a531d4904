"""What the binding of the training operators keeps a caller from: calls whose tensors or stream belong to another device than
the current one, where the kernel would be launched."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def tr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_23087_amd import training
    return training


class Operators:
    """One call of each, and all that they write."""

    def __init__(self, tr):
        rows, hidden, vocab, n = 40, 64, 100, 700
        f32 = lambda *shape: torch.full(shape, 5.0, device="cuda")  # noqa: E731
        half = lambda *shape: torch.full(shape, 5.0, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        x, w, labels = torch.randn_like(half(rows, hidden)), half(vocab, hidden), torch.zeros(rows, dtype=torch.int32, device="cuda")
        mean, rstd, y, dw, db = f32(rows), f32(rows), half(rows, hidden), f32(hidden), f32(hidden)
        loss, lse, dx, dweight = f32(1), f32(rows), half(rows, hidden), half(vocab, hidden)
        space = torch.empty(max(tr.norm_workspace(rows, hidden), tr.vocab_loss_workspace(rows, hidden, vocab)), dtype=torch.uint8,
                            device="cuda")
        p, g, m, v, out = (f32(n) for _ in range(5))
        codes, scales = torch.zeros(n, dtype=torch.uint8, device="cuda"), f32(3)
        self.tensors = tr.adamw_tensors([p], [g], [m], [v])
        self.scale = f32(1)
        self.calls = {
            "norm_forward": lambda **kw: tr.norm_forward(x, None, None, y, mean, rstd, **kw),
            "norm_backward": lambda **kw: tr.norm_backward(x, x, None, mean, rstd, dx, dw, db, space, **kw),
            "vocab_loss_forward": lambda **kw: tr.vocab_loss_forward(x, w, labels, loss, lse, None, space, **kw),
            "vocab_loss_backward": lambda **kw: tr.vocab_loss_backward(x, w, labels, lse, None, dx, dweight, space, **kw),
            "adamw_step": lambda **kw: tr.adamw_step(self.tensors, 1, 1e-3, grad_scale=self.scale, **kw),
            "adamw_state_values": lambda **kw: tr.adamw_state_values(codes, scales, out, 1, **kw),
        }
        self.written = [y, mean, rstd, dx, dw, db, loss, lse, dweight, p, m, v, out]


NAMES = ["norm_forward", "norm_backward", "vocab_loss_forward", "vocab_loss_backward", "adamw_step", "adamw_state_values"]


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_device(tr, name, monkeypatch):
    o = Operators(tr)
    before = [t.clone() for t in o.written]
    with monkeypatch.context() as mp:
        mp.setattr(torch._C, "_cuda_getDevice", lambda: 1)      # as on a machine with two, with the other one current
        with pytest.raises(ValueError, match="current device"):
            o.calls[name](stream=0)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(o.written, before))
    o.calls[name]()
    torch.cuda.synchronize()
    assert not all(torch.equal(a, b) for a, b in zip(o.written, before))


@pytest.mark.parametrize("name", NAMES)
def test_stream_of_another_device(tr, name, monkeypatch):
    o = Operators(tr)
    before = [t.clone() for t in o.written]

    class Elsewhere(torch.cuda.Stream):
        device = torch.device("cuda", 1)

    stream = Elsewhere()
    with pytest.raises(ValueError, match="stream"):
        o.calls[name](stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(o.written, before))


def test_grad_scale_of_another_device(tr):
    o = Operators(tr)

    class Elsewhere:
        is_cuda, device, dtype = True, torch.device("cuda", 1), torch.float32
        numel, is_contiguous, data_ptr = (lambda s: 1), (lambda s: True), (lambda s: 0)

    with pytest.raises(ValueError, match="grad_scale"):
        tr.adamw_step(o.tensors, 1, 1e-3, grad_scale=Elsewhere())


def test_list_of_tensors_dropped_behind_a_queued_step(tr):
    """A step queued on another stream reads its table and its tensors by address: once the list of them is dropped, nothing may
    be given their memory before the step has run."""
    n = 300000
    for raw in (False, True):
        side = torch.cuda.Stream()
        p, g, m, v = (torch.full((n,), 1.0, device="cuda") for _ in range(4))
        tensors = tr.adamw_tensors([p], [g], [m], [v])
        want = p.clone(), g.clone(), m.clone(), v.clone()
        tr.adamw_step(tr.adamw_tensors(*[[t] for t in want]), 1, 1e-3)
        size, taken = tensors.table.nbytes, {tensors.table.data_ptr(), g.data_ptr(), v.data_ptr()}
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(2_000_000_000)
        tr.adamw_step(tensors, 1, 1e-3, stream=side.cuda_stream if raw else side)
        del tensors, g, v
        after = [torch.zeros(size, dtype=torch.uint8, device="cuda"), *(torch.zeros(n, device="cuda") for _ in range(6))]
        queued = not side.query()
        assert taken.isdisjoint(t.data_ptr() for t in after)
        torch.cuda.synchronize()
        assert queued, "the step was over before memory was asked for: the test shows nothing"
        assert torch.equal(p, want[0]) and torch.equal(m, want[2]) and all(bool((t == 0).all()) for t in after)
