"""Preference fine-tuning of a small sparse model, with every operator in its place.

The model is a stack of feed-forward blocks over single tokens (no attention, so
it learns which token follows which): embedding, then in each block
residual + dropout(branch) and its norm, a sparse up projection with adapters,
SiLU and a sparse down projection, at last a norm and a sparse head.  With
``gated`` a second projection of the same input, through SiLU, multiplies the up
projection instead (``ops.lors_gated``).  The other projections are
``ops.lors_linear``; embedding, norms, dropout and the loss are those of
``train``.  The weights are pruned and frozen; adapters, norm weights and the
embedding train: by descent with momentum, or the adapters along orthogonalised
momenta (``update="orthogonal"``, ``train.OrthogonalUpdate``).

The loss prefers continuations that follow a rule over random ones.  Its
reference is the model before training: the adapters start at B = 0, so it is the
sparse model alone, and its log-probabilities are taken once.

After training the model continues prompts greedily, or by ``train.sample`` at a
temperature.

``python -m paper_2501_08582_amd.finetune --steps 30 --gated --update orthogonal``
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
    gated: bool = False
    update: str = "momentum"  # or "orthogonal": the adapters' rule, whose matrix_lr is of another kind
    matrix_lr: float = 0.02


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

    def parts(self):
        """(W, M, B, A), as the gated block takes a projection."""
        return self.W, self.M, self.B, self.A

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
        self.gates = [Projection(cfg.hidden, cfg.width, cfg, g) for _ in range(cfg.layers if cfg.gated else 0)]

    def parameters(self) -> Dict[str, torch.Tensor]:
        out = {"table": self.table, "head.A": self.head.A, "head.B": self.head.B}
        for i, (up, down) in enumerate(self.blocks):
            out.update({f"{i}.up.A": up.A, f"{i}.up.B": up.B, f"{i}.down.A": down.A, f"{i}.down.B": down.B})
        for i, gate in enumerate(self.gates):
            out.update({f"{i}.gate.A": gate.A, f"{i}.gate.B": gate.B})
        out.update({f"norm.{i}": w for i, w in enumerate(self.norms)})
        return out

    def inner(self, i: int, x: torch.Tensor) -> torch.Tensor:
        """What block i's down projection takes."""
        up, _ = self.blocks[i]
        if self.cfg.gated:
            return ops.lors_gated(x, self.gates[i].parts(), up.parts(), self.cfg.scale, self.cfg.mask)
        return torch.nn.functional.silu(up(x))

    def inner_serve(self, i: int, x: torch.Tensor) -> torch.Tensor:
        up, _ = self.blocks[i]
        if self.cfg.gated:
            return ops.gated_forward(x, self.gates[i].parts(), up.parts(), self.cfg.scale, self.cfg.mask, save=False)[0]
        return torch.nn.functional.silu(up.serve(x))

    def logits(self, ids: torch.Tensor, p: float = 0.0, offset: int = 0) -> torch.Tensor:
        """Logits of the token after each of ``ids``.  Every dropout of a pass takes an
        offset of its own."""
        cfg = self.cfg
        table_scale = cfg.width**0.5
        branch, stream = train.embedding(ids, self.table, table_scale), None
        for i, (_, down) in enumerate(self.blocks):
            x, stream = train.norm(branch, self.norms[i], kind=cfg.kind, residual=stream, p=p, seed=cfg.seed,
                                   offset=offset * (cfg.layers + 1) + i)
            branch = down(self.inner(i, x))
        x, _ = train.norm(branch, self.norms[-1], kind=cfg.kind, residual=stream, p=p, seed=cfg.seed,
                          offset=offset * (cfg.layers + 1) + cfg.layers)
        return self.head(x)

    @torch.no_grad()
    def generate(self, ids: torch.Tensor, tokens: int, temperature: float = 0.0, top_k: int = 0, top_p: float = 1.0,
                 generator: Optional[torch.Generator] = None) -> torch.Tensor:
        """Continuation of the last token of each sequence, one token a pass: greedy, or sampled
        at a temperature with ``generator``'s numbers.  The forms without gradients and
        statistics."""
        cfg, out = self.cfg, [ids]
        for _ in range(tokens):
            branch, stream = train.embedding_forward(out[-1][:, -1:].contiguous(), self.table, cfg.width**0.5), None
            for i, (_, down) in enumerate(self.blocks):
                x, stream, _, _ = train.norm_forward(branch, self.norms[i], kind=cfg.kind, residual=stream, need_stats=False)
                branch = down.serve(self.inner_serve(i, x))
            x, _, _, _ = train.norm_forward(branch, self.norms[-1], kind=cfg.kind, residual=stream, need_stats=False)
            logits = self.head.serve(x)
            if temperature == 0.0:
                out.append(logits.argmax(dim=-1))
                continue
            u = torch.rand(logits.shape[:-1], generator=generator, device="cuda")
            out.append(train.sample(logits, u, temperature, top_k, top_p)[0])
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
    of the same root mean square; with ``update="orthogonal"`` all adapters take one
    ``train.OrthogonalUpdate`` instead."""

    def __init__(self, cfg: Optional[Config] = None):
        self.cfg = cfg = cfg or Config()
        self.model = Model(cfg)
        self.params = self.model.parameters()
        self.master = {k: p.detach().float() for k, p in self.params.items()}
        self.speed = {k: torch.zeros_like(m) for k, m in self.master.items()}
        self.matrices: List[str] = []
        if cfg.update == "orthogonal":
            self.matrices = [k for k in self.params if k.endswith((".A", ".B"))]
            kept = [[of[k] for k in self.matrices] for of in (self.master, self.params, self.speed)]
            self.rule = train.OrthogonalUpdate(kept[0], [p.detach() for p in kept[1]], kept[2])
        elif cfg.update != "momentum":
            raise ValueError(f"unknown update {cfg.update!r} (momentum, orthogonal)")
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
            if self.matrices:
                by_name = dict(zip(self.params, grads))
                self.rule.step([by_name[k] for k in self.matrices], cfg.matrix_lr)
            for (k, p), grad in zip(self.params.items(), grads):
                if k in self.matrices:
                    continue
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
    ap.add_argument("--gated", action="store_true", help="gated blocks")
    ap.add_argument("--update", choices=("momentum", "orthogonal"), default="momentum", help="the adapters' rule")
    ap.add_argument("--temperature", type=float, default=0.0, help="also sample continuations at it")
    a = ap.parse_args(argv)
    trainer = Trainer(Config(kind=a.kind, mask=a.mask, gated=a.gated, update=a.update))
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
    if a.temperature > 0.0:
        told = trainer.model.generate(start, 4, a.temperature, top_p=0.95, generator=torch.Generator(device="cuda").manual_seed(1))
        hits = (told[:, 1:] == rule(told[:, :-1], cfg.vocab)).float().mean()
        print(f"sampled ones: {float(hits):.2f}", flush=True)


if __name__ == "__main__":
    main()
