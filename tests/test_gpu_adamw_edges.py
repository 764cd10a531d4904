"""AdamW's states at the ends of f32's range: runs of 8-bit states whose largest value is tiny, roots below the normal numbers,
gradients that are not finite."""

import numpy as np
import pytest

from gpu_common import say
import training_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LEAST = 2.0 ** -149               # f32's smallest value: a result below 2^-126 is off by half of it


@pytest.fixture(scope="module")
def tr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_23087_amd import training
    return training


class State:
    """One tensor with its state, before its first step."""

    def __init__(self, tr, grad, bits, start=0.0):
        self.tr, self.g, n = tr, grad, grad.numel()
        self.p = torch.full((n,), start, device="cuda")
        state = torch.uint8 if bits == 8 else torch.float32
        self.m, self.v = (torch.zeros(n, dtype=state, device="cuda") for _ in range(2))
        self.scales = torch.zeros(2, -(-n // 256), device="cuda") if bits == 8 else None
        self.tensors = tr.adamw_tensors([self.p], [self.g], [self.m], [self.v], scales=None if bits == 32 else [self.scales])

    def step(self, number, **kw):
        self.tr.adamw_step(self.tensors, number, **kw)

    def values(self, moment):
        if self.scales is None:
            return (self.m, self.v)[moment - 1].cpu().double().numpy()
        out = torch.full((self.p.numel(),), float("nan"), device="cuda")
        self.tr.adamw_state_values((self.m, self.v)[moment - 1], self.scales[moment - 1], out, moment)
        return out.cpu().double().numpy()


@pytest.mark.parametrize("size", [1e-9, 1e-11, 3e-12, 1e-13, 1e-14, 1e-16, 1e-18, 1e-20, 1e-25, 1e-37])
def test_codes_of_tiny_runs(tr, size):
    """Whatever a run's largest value is, it has the top level, and each code is the level whose thresholds the value lies
    between. Values whose root is held with n bits below f32's smallest normal one carry that rounding, and no more."""
    say(f"case adamw gradients of {size}")
    gen = np.random.default_rng(3)
    n, beta1, beta2 = 1000, 0.9, 0.95
    g = (gen.normal(size=n) * 10.0 ** gen.uniform(-2, 0, n) * size).astype(np.float32)
    for offset in (0, 1):                          # whole vectors, and element by element
        buf = torch.zeros(n + 1, device="cuda")
        buf[offset:offset + n] = torch.from_numpy(g).cuda()
        t = State(tr, buf[offset:offset + n], 8)
        t.step(1, lr=1e-3, beta1=beta1, beta2=beta2, eps=1e-8)
        g64 = g.astype(np.float64)
        for k, (exact, levels, power) in enumerate([((1 - beta1) * g64, 127, 2), ((1 - beta2) * g64 * g64, 255, 4)]):
            e = 8 * ref.U * np.abs(exact) + 2 * LEAST      # 1 - beta, the products and the sum
            scale = t.scales[k].cpu().double().numpy()
            top = ref.runs(np.abs(exact)).max(1)
            assert np.all(np.abs(scale - top) <= ref.runs(e).max(1)), (k, scale, top)
            code = (t.m, t.v)[k].cpu().numpy().astype(np.int64)
            level = code & 127 if k == 0 else code
            s = np.repeat(scale, 256)[:n]
            assert np.all(ref.runs(level).max(1)[scale > 0] == levels), (k, ref.runs(level).max(1))
            low, high = s * (np.maximum(level - 0.5, 0) / levels) ** power, s * ((level + 0.5) / levels) ** power
            slip = e + 8 * ref.U * np.abs(exact)
            assert np.all((np.abs(exact) <= high + slip) | (level == levels)), f"moment {k + 1}: level too low"
            assert np.all((np.abs(exact) >= low - slip) | ((level == 1) & (k == 1))), f"moment {k + 1}: level too high"
            held = ref.values(code.astype(np.uint8), scale, k + 1)
            got = t.values(k + 1)
            assert np.all(np.abs(got - held) <= 4 * ref.U * np.abs(held) + LEAST), (k, got[:4], held[:4])


@pytest.mark.parametrize("size,eps", [(size, eps) for size in (1e-3, 1e-12, 1e-13, 1e-15) for eps in (1e-12, 1e-15, 0.0)
                                      if eps <= size * 1e-2])
def test_tiny_gradients_move_as_large_ones(tr, size, eps):
    """Steps with gradients of one value: with any eps far below it an element moves by lr a step, in 8 bits as in 32."""
    say(f"case adamw 60 steps of {size}, eps {eps}")
    for bits in (32, 8):
        t = State(tr, torch.full((512,), size, device="cuda"), bits)
        for k in range(60):
            t.step(k + 1, lr=1e-3, beta1=0.9, beta2=0.95, eps=eps)
        # the codes of a constant run are exact (the top level): what is left are some 10 roundings a step and eps' share
        assert float((t.p + 0.06).abs().max()) <= 0.06 * (1000 * ref.U + 1.1 * eps / size), (bits, t.p[:4])


@pytest.mark.parametrize("bits", [32, 8])
def test_root_of_a_state_below_the_normal_numbers(tr, bits):
    """v of 5e-44 is 36 times the smallest f32, so its root is known to 1 / 72: the step is finite and lr to that accuracy."""
    say(f"case adamw v below 2^-126, {bits} bits")
    t = State(tr, torch.full((300,), 1e-21, device="cuda"), bits)
    t.step(1, lr=1e-3, beta1=0.9, beta2=0.95, eps=0.0)
    assert float((t.p + 1e-3).abs().max()) <= 1e-3 * 0.02, t.p[:4]


@pytest.mark.parametrize("eps", [1e-38, 1e-40, 1e-60])
def test_eps_below_the_normal_numbers(tr, eps):
    """Above 0 it keeps elements without a gradient where they are."""
    say(f"case adamw eps {eps}")
    for bits in (32, 8):
        t = State(tr, torch.zeros(300, device="cuda"), bits, 0.5)
        t.step(1, lr=1e-3, eps=eps)
        assert bool((t.p == 0.5).all()), (bits, t.p[:4])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("offset", [0, 1])
def test_gradient_that_is_not_finite(tr, bad, offset):
    """It reaches its element's parameter and state, in 8 bits its run's scales, and with them the run's next step; nothing
    else."""
    say(f"case adamw gradient {bad} offset {offset}")
    n, at = 5000, 1300
    run = slice(1280, 1536)
    for bits in (32, 8):
        buf = torch.linspace(-1, 1, n + 1, device="cuda")
        t = State(tr, buf[offset:offset + n], bits, 0.5)
        good = State(tr, t.g.clone(), bits, 0.5)
        t.g[at] = bad
        for s in (t, good):
            s.step(1, lr=1e-3)
        others = torch.arange(n, device="cuda") != at
        assert bool(torch.isnan(t.p[at])) and torch.equal(t.p[others], good.p[others])
        if bits == 32:
            want = [bad, abs(bad)]
            for state, clean, w in ((t.m, good.m, want[0]), (t.v, good.v, want[1])):
                assert np.isnan(w) and bool(torch.isnan(state[at])) or float(state[at]) == w
                assert torch.equal(state[others], clean[others])
            continue
        runs = torch.arange(t.scales.shape[1], device="cuda") != at // 256
        for k in (0, 1):
            top = float(t.scales[k, at // 256])
            assert np.isnan(top) if np.isnan(bad) else top == float("inf"), top
            assert torch.equal(t.scales[k][runs], good.scales[k][runs])
        assert bool((t.m[run] % 128 == 0).all()) and bool((t.v[run] <= 1).all())       # v above 0 has no level 0
        outside = torch.ones(n, dtype=torch.bool, device="cuda")
        outside[run] = False
        assert torch.equal(t.m[outside], good.m[outside]) and torch.equal(t.v[outside], good.v[outside])
        t.g[at] = 0.0
        good.g[at] = 0.0
        for s in (t, good):
            s.step(2, lr=1e-3)
        assert bool(torch.isnan(t.p[run]).all()) and torch.equal(t.p[outside], good.p[outside])
