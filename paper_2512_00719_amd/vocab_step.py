"""A decoding step and a training step over one tied [V, D] matrix, with the operators of ``vocab`` and a sampling call of ``binding``.

    python -m paper_2512_00719_amd.vocab_step [--vocab V] [--width D] [--tokens T] [--steps N]

The model between the embedding and the final norm is a stand-in, one matrix on the residual stream; what stands at the
vocabulary is as a program has it.  Decoding: ``embed`` the last ids, the model, ``rms_norm_int8`` with the residual's addition, ``linear_int8``
against the table's codes, ``Sampler.sample``.  Training: the same up to ``rms_norm``, ``linear_xent`` and the gradients back to
the table, to which the head's and the embedding's are added up in float32, and a step of gradient descent.
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import binding, synth, vocab


class TiedModel:
    """Table, model matrix and norm weight in bfloat16, with float32 masters for training."""

    def __init__(self, V: int, D: int, seed: int = 0, device: str = "cuda:0"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.V, self.D = V, D
        self.table32 = torch.randn(V, D, generator=g, device=device) * 0.02
        self.mix32 = torch.randn(D, D, generator=g, device=device) * D ** -0.5
        self.norm32 = torch.ones(D, device=device)
        self.scale = D ** 0.5  # of the embedding
        self.refresh()

    def refresh(self) -> None:
        """The working copies from the masters; the head's codes are laid out here, once for all decoding steps that follow."""
        self.table, self.mix, self.norm = self.table32.bfloat16(), self.mix32.bfloat16(), self.norm32.bfloat16()
        self.codes, self.scales = vocab.quantize_rows(self.table)

    def stream(self, ids):
        """The residual stream's two last terms for tokens `ids`."""
        x = vocab.embed(ids, self.table, scale=self.scale)
        return x, torch.mm(x, self.mix)

    def logits(self, ids):
        x, update = self.stream(ids)
        codes, scales, _ = vocab.rms_norm_int8(update, self.norm, residual=x)
        return vocab.linear_int8(codes, scales, self.codes, self.scales)

    def train_step(self, ids, targets, rate: float) -> torch.Tensor:
        """One step on next-token pairs (a target outside the vocabulary is masked).  Returns the mean loss before it, on the device."""
        x, update = self.stream(ids)
        y, h, rstd = vocab.rms_norm(update, self.norm, residual=x, need_rstd=True)
        loss, lse = vocab.linear_xent(y, self.table, targets)
        live = (targets >= 0) & (targets < self.V)
        dloss = live.float() / live.sum().clamp(min=1)
        dtable = torch.empty_like(self.table32)
        dy, _ = vocab.linear_xent_grad(dloss, y, self.table, targets, lse, dweight=dtable)
        dh, dnorm = vocab.rms_norm_grad(dy, h, self.norm, rstd)
        dx = dh + torch.mm(dh, self.mix.t())
        dmix = torch.mm(x.t(), dh)
        vocab.embed_grad(ids, dx, self.V, scale=self.scale, dtable=dtable, accumulate=True)  # tied: onto the head's gradient
        self.table32.add_(dtable, alpha=-rate)
        self.mix32.add_(dmix, alpha=-rate)
        self.norm32.add_(dnorm, alpha=-rate)
        self.refresh()
        return (loss * dloss).sum()


def decode(model: TiedModel, first_ids: torch.Tensor, steps: int, seed: int = 1) -> torch.Tensor:
    """`steps` further ids of each sequence, [sequences, steps]."""
    n = first_ids.numel()
    sampler = binding.Sampler(model.V, 0)
    params = torch.from_numpy(synth.make_params(n, temperature=0.8, top_k=50, top_p=0.95).view(np.uint8).reshape(n, 32)).to(first_ids.device)
    ids, out = first_ids, []
    for step in range(steps):
        ids = sampler.sample(model.logits(ids), params, seed=seed, step=step)
        out.append(ids)
    result = torch.stack(out, 1)
    torch.cuda.synchronize()  # the context is freed behind the calls that use it
    sampler.close()
    return result


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    model = TiedModel(a.vocab, a.width)
    ids = torch.arange(a.tokens, device="cuda:0", dtype=torch.int32) % a.vocab
    targets = (ids + 1) % a.vocab  # something that can be learnt: to count
    for step in range(a.steps):
        loss = model.train_step(ids, targets, rate=1.0)
        print(f"step {step}: loss {float(loss):.4f}", flush=True)
    print("drawn from the trained model:", decode(model, ids[:: max(1, a.tokens // 4)], 5).tolist(), flush=True)


if __name__ == "__main__":
    main()
