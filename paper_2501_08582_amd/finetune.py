"""Preference fine-tuning of a small sparse model, with every operator in its place.

The model is a stack of gateless feed-forward blocks over single tokens (no
attention, so it learns which token follows which): embedding, then in each block
residual + dropout(branch) and its norm, a sparse up projection with adapters,
SiLU and a sparse down projection, at last a norm and a sparse head.  All
projections are ``ops.lors_linear``; embedding, norms, dropout and the loss are
those of ``train``.  The weights are pruned and frozen; adapters, norm weights and
the embedding train.

The loss prefers continuations that follow a rule over random ones.  Its
reference is the model before training: the adapters start at B = 0, so it is the
sparse model alone, and its log-probabilities are taken once.

``python -m paper_2501_08582_amd.finetune --steps 30``
"""
from __future__ import annotations

import argparse
import dataclasses
from typing import Dict, List, Optional, Tuple

import torch

from . import ops, train


@dataclasses.dataclass(frozen=True)
class Config:
    vocab: int = 2048
    width: int = 512
    hidden: int = 1536
    layers: int = 2
    rank: int = 16
    scale: float = 2.0
    mask: str = ops.TWO_FOUR
    kind: str = train.RMS
    dropout: float = 0.05
    beta: float = 0.1
    pairs: int = 16
    length: int = 64
    prompt: int = 16
    lr: float = 3e-4
    seed: int = 0


class Projection:
    """A frozen pruned weight, its packed mask and its adapters."""

    def __init__(self, R: int, C: int, cfg: Config, g: torch.Generator):
        W = torch.randn((R, C), generator=g, device="cuda") / C**0.5
        if cfg.mask == ops.TWO_FOUR:
            top = W.abs().view(R, C // 4, 4).topk(2, dim=2).indices
            keep = torch.zeros((R, C // 4, 4), dtype=torch.bool, device="cuda").scatter_(2, top, True).view(R, C)
        else:
            keep = W.abs() >= W.abs().median(dim=1, keepdim=True).values
        self.W = (W * keep).bfloat16()
        self.M = ops.mask_pack(keep, cfg.mask)
        self.A = (torch.randn((cfg.rank, C), generator=g, device="cuda") / cfg.rank).bfloat16().requires_grad_(True)
        self.B = torch.zeros((R, cfg.rank), dtype=torch.bfloat16, device="cuda", requires_grad=True)
        self.cfg = cfg

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        return ops.lors_linear(x, self.W, self.M, self.B, self.A, self.cfg.scale, self.cfg.mask)

    def serve(self, x: torch.Tensor) -> torch.Tensor:
        return ops.forward(x, self.W, self.M, self.B.detach(), self.A.detach(), self.cfg.scale, self.cfg.mask)


class Model:
    def __init__(self, cfg: Config):
        self.cfg = cfg
        g = torch.Generator(device="cuda").manual_seed(cfg.seed)
        self.table = (0.02 * torch.randn((cfg.vocab, cfg.width), generator=g, device="cuda")).bfloat16().requires_grad_(True)
        self.blocks = [(Projection(cfg.hidden, cfg.width, cfg, g), Projection(cfg.width, cfg.hidden, cfg, g))
                       for _ in range(cfg.layers)]
        self.head = Projection(cfg.vocab, cfg.width, cfg, g)
        self.norms = [torch.ones(cfg.width, dtype=torch.bfloat16, device="cuda", requires_grad=True)
                      for _ in range(cfg.layers + 1)]

    def parameters(self) -> Dict[str, torch.Tensor]:
        out = {"table": self.table, "head.A": self.head.A, "head.B": self.head.B}
        for i, (up, down) in enumerate(self.blocks):
            out.update({f"{i}.up.A": up.A, f"{i}.up.B": up.B, f"{i}.down.A": down.A, f"{i}.down.B": down.B})
        out.update({f"norm.{i}": w for i, w in enumerate(self.norms)})
        return out

    def logits(self, ids: torch.Tensor, p: float = 0.0, offset: int = 0) -> torch.Tensor:
        """Logits of the token after each of ``ids``.  Every dropout of a pass takes an
        offset of its own."""
        cfg = self.cfg
        table_scale = cfg.width**0.5
        branch, stream = train.embedding(ids, self.table, table_scale), None
        for i, (up, down) in enumerate(self.blocks):
            x, stream = train.norm(branch, self.norms[i], kind=cfg.kind, residual=stream, p=p, seed=cfg.seed,
                                   offset=offset * (cfg.layers + 1) + i)
            branch = down(torch.nn.functional.silu(up(x)))
        x, _ = train.norm(branch, self.norms[-1], kind=cfg.kind, residual=stream, p=p, seed=cfg.seed,
                          offset=offset * (cfg.layers + 1) + cfg.layers)
        return self.head(x)

    @torch.no_grad()
    def generate(self, ids: torch.Tensor, tokens: int) -> torch.Tensor:
        """Greedy continuation of the last token of each sequence, one token a pass:
        the forms without gradients and statistics."""
        cfg, out = self.cfg, [ids]
        for _ in range(tokens):
            branch, stream = train.embedding_forward(out[-1][:, -1:].contiguous(), self.table, cfg.width**0.5), None
            for i, (up, down) in enumerate(self.blocks):
                x, stream, _, _ = train.norm_forward(branch, self.norms[i], kind=cfg.kind, residual=stream, need_stats=False)
                branch = down.serve(torch.nn.functional.silu(up.serve(x)))
            x, _, _, _ = train.norm_forward(branch, self.norms[-1], kind=cfg.kind, residual=stream, need_stats=False)
            out.append(self.head.serve(x).argmax(dim=-1))
        return torch.cat(out, dim=1)


def rule(ids: torch.Tensor, vocab: int) -> torch.Tensor:
    """The token that the preferred continuations put after each of ``ids``."""
    return (5 * ids + 7) % vocab


def batch(cfg: Config, seed: int) -> Tuple[torch.Tensor, torch.Tensor]:
    """(ids, targets) of 2 P sequences: preferred ones that follow the rule after a random
    prompt, then rejected ones of the same prompts that go on at random.  Prompts and
    padding behind sequences of unequal lengths have the target -100."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    P, S = cfg.pairs, cfg.length

    def randint(*shape):
        return torch.randint(0, cfg.vocab, shape, generator=g, device="cuda")

    start: List[torch.Tensor] = [randint(P, 1)]
    for _ in range(S):
        start.append(rule(start[-1], cfg.vocab))
    good, bad = torch.cat(start, dim=1), randint(P, S + 1)
    head = randint(P, cfg.prompt)
    good[:, :cfg.prompt], bad[:, :cfg.prompt] = head, head
    both = torch.cat([good, bad])
    ends = torch.randint(S // 2, S + 1, (P, 1), generator=g, device="cuda").repeat(2, 1)
    at = torch.arange(S, device="cuda").unsqueeze(0)
    counted = (at >= cfg.prompt) & (at < ends)
    ids = torch.where(at < ends, both[:, :-1], torch.full_like(both[:, :-1], -1))  # padding is no token
    return ids.contiguous(), torch.where(counted, both[:, 1:], torch.full_like(ids, -100)).contiguous()


class Trainer:
    """Descent with momentum on fp32 copies of the trained parameters, every array's step
    of the same root mean square."""

    def __init__(self, cfg: Optional[Config] = None):
        self.cfg = cfg = cfg or Config()
        self.model = Model(cfg)
        self.params = self.model.parameters()
        self.master = {k: p.detach().float() for k, p in self.params.items()}
        self.speed = {k: torch.zeros_like(m) for k, m in self.master.items()}
        self.count = 0

    @torch.no_grad()
    def reference(self, ids: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """Log-probabilities of the targets under the present model, without dropout."""
        return train.logprob_forward(self.model.logits(ids), targets)[0]

    def step(self, ids: torch.Tensor, targets: torch.Tensor, ref: torch.Tensor):
        """One update; (loss, rewards) before it."""
        cfg = self.cfg
        logits = self.model.logits(ids, cfg.dropout, self.count)
        loss, reward, _ = train.preference_loss(logits, targets, ref, cfg.beta)
        grads = torch.autograd.grad(loss, list(self.params.values()))
        with torch.no_grad():
            for (k, p), grad in zip(self.params.items(), grads):
                self.speed[k].mul_(0.9).add_(grad.float(), alpha=0.1)
                rms = self.speed[k].square().mean().sqrt() + 1e-12
                self.master[k].sub_(self.speed[k] / rms, alpha=cfg.lr)
                p.copy_(self.master[k])
        self.count += 1
        return loss.detach(), reward


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--kind", choices=(train.LAYER, train.RMS), default=train.RMS)
    ap.add_argument("--mask", choices=(ops.BITMAP, ops.TWO_FOUR), default=ops.TWO_FOUR)
    a = ap.parse_args(argv)
    trainer = Trainer(Config(kind=a.kind, mask=a.mask))
    cfg = trainer.cfg
    batches = [batch(cfg, 100 + i) for i in range(4)]
    refs = [trainer.reference(*b) for b in batches]
    for i in range(a.steps):
        k = i % len(batches)
        loss, reward = trainer.step(*batches[k], refs[k])
        P = cfg.pairs
        margin = (reward[:P] - reward[P:]).mean()
        print(f"step {i}: loss {float(loss):.4f}, preferred over rejected by {float(margin):.4f}", flush=True)
    start = torch.arange(8, device="cuda").unsqueeze(1)
    told = trainer.model.generate(start, 4)
    hits = (told[:, 1:] == rule(told[:, :-1], cfg.vocab)).float().mean()
    print(f"greedy continuations that follow the rule: {float(hits):.2f}", flush=True)


if __name__ == "__main__":
    main()
