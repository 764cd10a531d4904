"""Trains an adapter, a norm and a vocabulary head on packed microbatches.

A step goes all the way: samples in the pool are planned into microbatches, each is packed into consecutive rows, the rows
pass the user's own layer (here one square matrix added to its input, where a program has its backbone), the layer norm and
the vocabulary loss; the gradients come back through both, summed in f32 over the microbatches, and one AdamW step per group
of tensors updates f32 parameters and the bf16 copies that the products read. The head's states are held in 8 bits.

    python examples/train_head.py [--steps 30] [--config tiny]
"""

from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_23087_amd import training as tr  # noqa: E402
from paper_2606_23087_amd.harness import GpuWorkload  # noqa: E402
from paper_2606_23087_amd.workloads import CONFIGS, SampleSpec, gen_samples  # noqa: E402

NO_LABEL = -100


def with_chained_text(specs, vocab: int, period: int, seed: int):
    """The samples with texts in which each id decides the next (there is no real text here, and random ids teach nothing)."""
    gen = np.random.default_rng(seed)
    chain = gen.permutation(vocab)[:period].astype(np.int32)
    return [SampleSpec(chain[(gen.integers(period) + np.arange(s.n_text)) % period], s.img_pos, s.img_ntok) for s in specs]


def next_ids(spec: SampleSpec) -> np.ndarray:
    """For each of a sample's rows the text id in the row behind it; none where that is an image's row or there is none."""
    rows = np.insert(spec.text_ids, np.repeat(spec.img_pos, spec.img_ntok), NO_LABEL) if spec.n_vis else spec.text_ids
    return np.append(rows[1:], NO_LABEL).astype(np.int32)


def clip_factor(grads, clip: float):
    """The factor that brings the gradients' norm down to `clip`, f32 [1]. Where the norm is not finite neither is the factor,
    and adamw_step changes nothing (clip over an infinite norm would be 0, a step like any other)."""
    norm = torch.sqrt(sum(g.square().sum() for g in grads))
    return torch.where(torch.isfinite(norm), torch.clamp(clip / norm, max=1.0), norm).reshape(1)


class Model:
    """f32 parameters, their bf16 copies, f32 gradients and AdamW's states."""

    def __init__(self, hidden: int, vocab: int, seed: int):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
        self.params = {"adapter": normal(hidden, hidden) * 0.1 / hidden ** 0.5, "weight": torch.ones(hidden, device="cuda"),
                       "bias": torch.zeros(hidden, device="cuda"), "head": normal(vocab, hidden) / hidden ** 0.5}
        self.bf16 = {k: p.bfloat16() for k, p in self.params.items()}
        self.grads = {k: torch.zeros_like(p) for k, p in self.params.items()}
        inner = ("adapter", "weight", "bias")
        pick = lambda d: [d[k] for k in inner]  # noqa: E731
        zeros = [[torch.zeros_like(self.params[k]) for k in inner] for _ in range(2)]
        self.inner = tr.adamw_tensors(pick(self.params), pick(self.grads), *zeros, copies=pick(self.bf16),
                                      weight_decay=[0.01, 0.0, 0.0])
        n = vocab * hidden
        codes = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
        scales = torch.zeros(2, -(-n // tr.FP_ADAMW_BLOCK), device="cuda")
        flat = lambda d: [d["head"].view(-1)]  # noqa: E731
        self.states = [*zeros[0], *zeros[1], *codes, scales]
        self.head = tr.adamw_tensors(flat(self.params), flat(self.grads), codes[:1], codes[1:], scales=[scales],
                                     copies=flat(self.bf16), weight_decay=0.01)


class Trainer:
    def __init__(self, config: str = "tiny", seed: int = 0, period: int = 64):
        cfg = CONFIGS[config]
        self.cfg, self.specs = cfg, with_chained_text(gen_samples(cfg, seed), cfg.vocab, period, seed)
        self.work = GpuWorkload(cfg, seed, specs=self.specs)
        self.model = Model(cfg.hidden, cfg.vocab, seed)
        rows, hidden = cfg.capacity, cfg.hidden
        half = lambda: torch.empty(rows, hidden, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.packed, self.cu, self.pos = self.work.alloc_outputs()
        self.y, self.dy, self.dz = half(), half(), half()
        self.mean, self.rstd, self.lse = (torch.empty(rows, device="cuda") for _ in range(3))
        self.loss = torch.empty(1, device="cuda")
        space = max(tr.norm_workspace(rows, hidden), tr.vocab_loss_workspace(rows, hidden, cfg.vocab))
        self.space = torch.empty(space, dtype=torch.uint8, device="cuda")
        self.labels_of = {i: next_ids(s) for i, s in zip(self.work.ids, self.specs)}
        self.steps = 0

    def step(self, lr: float = 3e-3, clip: float = 1.0) -> float:
        """One step over the plan's microbatches; the mean loss of their labelled rows before the step."""
        m, plan = self.model, self.work.plan()
        batches = [ids for ids in self.work.microbatches(plan) if ids]
        labels = [np.concatenate([self.labels_of[i] for i in ids]) for ids in batches]
        n_labelled = max(sum(int((lab >= 0).sum()) for lab in labels), 1)
        share = torch.full((1,), 1.0 / n_labelled, device="cuda")
        for g in m.grads.values():
            g.zero_()
        total = torch.zeros(1, device="cuda")
        for ids, lab in zip(batches, labels):
            n, _ = self.work.pack(ids, self.packed, self.cu, self.pos)
            lab = torch.from_numpy(lab).cuda()
            x = self.packed[:n].view(torch.bfloat16)
            z = x + x @ m.bf16["adapter"]                                # the user's own layer
            y, dy, dz, mean, rstd, lse = (t[:n] for t in (self.y, self.dy, self.dz, self.mean, self.rstd, self.lse))
            tr.norm_forward(z, m.bf16["weight"], m.bf16["bias"], y, mean, rstd)
            tr.vocab_loss_forward(y, m.bf16["head"], lab, self.loss, lse, None, self.space, reduction="sum")
            total += self.loss
            tr.vocab_loss_backward(y, m.bf16["head"], lab, lse, share, dy, m.grads["head"], self.space, reduction="sum",
                                   accumulate=True)
            tr.norm_backward(dy, z, m.bf16["weight"], mean, rstd, dz, m.grads["weight"], m.grads["bias"], self.space,
                             accumulate=True)
            m.grads["adapter"] += x.t() @ dz
        self.update(lr, clip)
        return float(total) / n_labelled

    def update(self, lr: float, clip: float) -> None:
        """One AdamW step of the model's gradients."""
        scale = clip_factor(self.model.grads.values(), clip)
        self.steps += 1
        for group in (self.model.inner, self.model.head):
            tr.adamw_step(group, self.steps, lr, 0.9, 0.95, grad_scale=scale)

    def close(self):
        self.work.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--config", default="tiny", choices=list(CONFIGS))
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    t = Trainer(a.config, a.seed)
    for i in range(a.steps):
        print(f"step {i + 1}: loss {t.step():.4f}", flush=True)
    t.close()


if __name__ == "__main__":
    main()
