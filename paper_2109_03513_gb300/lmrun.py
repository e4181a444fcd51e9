"""A small language model on ESB codes: the coded feed-forward stack and output
head of a decoder, as it answers (4-bit weights with group scales, 8-bit
activations) and as it is trained (fake-quantised weights and activations,
straight-through gradients).

The model that is trained has no attention: a layer is norm -> up -> relu ->
down with a residual stream, a token's answer depends on that token alone.  It
runs the library's language-model operators together, in the order in which a
decoding or training step calls them; PyTorch adds the embedding lookup, the
rectifier and, in training, the dense products of the fake-quantised values.

Decoder answers with attention as well: before each such layer the heads'
norms and rotation, the 4-bit cache and attention over it, with 4-bit
projections around them.  It takes prompts and single tokens alike.

    python -m paper_2109_03513_gb300.lmrun        # trains on a fixed next-token rule, then answers
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import torch

from . import esb

W_FMT, X_FMT, GROUP = esb.Fmt(4, 2), esb.Fmt(8, 6), 64


@dataclass
class Config:
    vocab: int = 1000
    width: int = 256
    hidden: int = 512
    layers: int = 2
    eps: float = 1e-6


class Model:
    """fp32 master weights; serving() lays them out as codes once."""

    def __init__(self, cfg: Config, seed: int = 0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def normal(*shape, std):
            return torch.randn(*shape, generator=g, device=device) * std

        self.cfg = cfg
        self.p = {"embed": normal(cfg.vocab, cfg.width, std=1.0), "norm": torch.ones(cfg.width, device=device),
                  "head": normal(cfg.vocab, cfg.width, std=cfg.width ** -0.5)}
        for i in range(cfg.layers):
            self.p[f"norm{i}"] = torch.ones(cfg.width, device=device)
            self.p[f"up{i}"] = normal(cfg.hidden, cfg.width, std=(2.0 / cfg.width) ** 0.5)
            self.p[f"down{i}"] = normal(cfg.width, cfg.hidden, std=cfg.hidden ** -0.5)

    def matrices(self):
        return [n for n in self.p if n.startswith(("up", "down", "head"))]

    # ------------------------------------------------------------ serving
    def serving(self) -> "Serving":
        return Serving(self)

    # ----------------------------------------------------------- training
    def step(self, tokens: torch.Tensor, targets: torch.Tensor, lr: float, entropy_weight: float = 0.0) -> torch.Tensor:
        """One step of gradient descent on -mean log p(target) - entropy_weight * mean H; returns the loss (a
        tensor).  Negative targets are positions without one."""
        c, p, n = self.cfg, self.p, tokens.numel()
        # forward: the values that the codes stand for, as serving multiplies them
        wq = {m: esb.esb_project_groups(p[m], W_FMT, GROUP, want_xq=True)[1] for m in self.matrices()}
        stream, out, tape = p["embed"][tokens], None, []
        for i in range(c.layers):
            o = self._norm(stream, p[f"norm{i}"], out)
            u = torch.relu(o.yq @ wq[f"up{i}"].t())
            uq = esb.esb_project_groups(u, X_FMT, 0, want_xq=True)[1]
            tape.append((o, u, uq))
            stream, out = o.h, uq @ wq[f"down{i}"].t()
        o = self._norm(stream, p["norm"], out)
        logits = o.yq @ wq["head"].t()
        lp = esb.esb_logprobs(logits, targets)
        has = (targets >= 0).sum().clamp_min(1)
        loss = -(lp.logp.sum() / has + entropy_weight * lp.entropy.mean())
        # backward: the projections pass gradients unchanged
        g = {}
        d = esb.esb_logprobs_backward(logits, targets, lp.lse, lp.entropy, (-1.0 / has).expand(n).contiguous(),
                                      torch.full((n,), -entropy_weight / n, device=logits.device))
        g["head"] = d.t() @ o.yq
        dh, g["norm"] = esb.esb_rmsnorm_backward(d @ wq["head"], o.h, p["norm"], o.rstd)
        for i in reversed(range(c.layers)):
            o, u, uq = tape[i]
            g[f"down{i}"] = dh.t() @ uq
            du = (dh @ wq[f"down{i}"]) * (u > 0)
            g[f"up{i}"] = du.t() @ o.yq
            dh, g[f"norm{i}"] = esb.esb_rmsnorm_backward(du @ wq[f"up{i}"], o.h, p[f"norm{i}"], o.rstd, dh=dh)
        g["embed"] = torch.zeros_like(p["embed"]).index_add_(0, tokens, dh)
        for name, grad in g.items():
            p[name].sub_(grad, alpha=lr)
        return loss

    def _norm(self, x, weight, residual):
        if residual is None:
            residual = torch.zeros_like(x)
        return esb.esb_rmsnorm(x, weight, self.cfg.eps, residual=residual, fmt=X_FMT, yq=torch.empty_like(x), want_rstd=True)


class Serving:
    """The model laid out for answering: 4-bit codes with a scale for every GROUP weights."""

    def __init__(self, m: Model):
        self.cfg = m.cfg
        self.w = {n: esb.esb_project_groups(m.p[n], W_FMT, GROUP)[0] for n in m.matrices()}
        self.embed = m.p["embed"].to(torch.bfloat16)
        self.norms = {n: v.clone() for n, v in m.p.items() if n.startswith("norm")}

    def answer(self, tokens: torch.Tensor, targets: Optional[torch.Tensor] = None, top: int = 1) -> esb.LogProbs:
        """Log probabilities of `targets`, entropy and the `top` likeliest next tokens for each token."""
        c, w = self.cfg, self.w
        stream, out = self.embed[tokens], None
        for i in range(c.layers):
            o = esb.esb_rmsnorm(stream, self.norms[f"norm{i}"], c.eps, residual=out, fmt=X_FMT, want_y=False)
            u = torch.relu_(esb.esb_matvec_groups(o.coded, w[f"up{i}"]))
            uq, _ = esb.esb_project_groups(u, X_FMT, 0)
            stream, out = (o.h if out is not None else stream), esb.esb_matvec_groups(uq, w[f"down{i}"])
        o = esb.esb_rmsnorm(stream, self.norms["norm"], c.eps, residual=out, fmt=X_FMT)
        logits = esb.esb_matvec_groups(o.coded, w["head"], y_dtype=torch.float32)
        return esb.esb_logprobs(logits, targets, top=top)


class Decoder:
    """Serving of layers with attention (random weights): norm -> q, k, v -> norms of heads and rotation -> append ->
    attention -> output projection, then the feed-forward layer.  Sequences grow in pages of a shared cache; step()
    takes some new tokens of each, a prompt's or one."""

    def __init__(self, cfg: Config, heads: int = 4, kv_heads: int = 2, head_dim: int = 64, pages: int = 64, page_size: int = 16,
                 most: int = 4096, k_fmt: esb.Fmt = esb.Fmt(4, 2), v_fmt: esb.Fmt = esb.Fmt(4, 2), seed: int = 0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.ffn = Model(cfg, seed, device).serving()
        self.cfg, self.heads, self.kv_heads, self.head_dim, self.page_size = cfg, heads, kv_heads, head_dim, page_size
        self.rotation = esb.rotation(head_dim, most, device=device)
        self.caches = [esb.kv_cache(pages, kv_heads, page_size, head_dim, k_fmt, v_fmt, device) for _ in range(cfg.layers)]
        rows = (heads + 2 * kv_heads) * head_dim

        def coded(n, k):
            return esb.esb_project_groups(torch.randn(n, k, generator=g, device=device) * k ** -0.5, W_FMT, GROUP)[0]

        self.qkv = [coded(rows, cfg.width) for _ in range(cfg.layers)]
        self.out = [coded(cfg.width, heads * head_dim) for _ in range(cfg.layers)]
        self.norms = [[1 + 0.1 * torch.randn(n, generator=g, device=device) for n in (cfg.width, head_dim, head_dim)] for _ in range(cfg.layers)]

    def step(self, tokens: torch.Tensor, starts: torch.Tensor, lens: torch.Tensor, pages: torch.Tensor) -> torch.Tensor:
        """Logits (n, vocab) of new tokens (n,): sequence i's are rows starts[i] .. starts[i + 1] - 1, lens[i] its places
        with them, pages[i] the cache's pages it has (int32 each)."""
        c, f, d = self.cfg, self.ffn, self.head_dim
        n = tokens.numel()
        seq = torch.bucketize(torch.arange(n, device=tokens.device), starts[1:], right=True)
        positions = lens[seq].long() - starts[seq + 1] + torch.arange(n, device=tokens.device)
        slots = pages[seq, positions // self.page_size].long() * self.page_size + positions % self.page_size
        stream, out, nq, nk = f.embed[tokens], None, self.heads * d, self.kv_heads * d
        for i in range(c.layers):
            wx, wq, wk = self.norms[i]
            o = esb.esb_rmsnorm(stream, wx, c.eps, residual=out, fmt=X_FMT, want_y=False)
            stream = o.h if out is not None else stream
            qkv = esb.esb_matvec_groups(o.coded, self.qkv[i])
            hn = esb.esb_headnorm(qkv[:, :nq], qkv[:, nq:nq + nk], d, wq, wk, c.eps, rotation=self.rotation, positions=positions)
            esb.esb_cache_append(self.caches[i], hn.k, qkv[:, nq + nk:], slots)
            a, _ = esb.esb_cache_attention(hn.q, self.caches[i], lens, pages, starts=starts)
            out = esb.esb_matvec_groups(esb.esb_project_groups(a, X_FMT, 0)[0], self.out[i])
            o = esb.esb_rmsnorm(stream, f.norms[f"norm{i}"], c.eps, residual=out, fmt=X_FMT, want_y=False)
            u = torch.relu_(esb.esb_matvec_groups(o.coded, f.w[f"up{i}"]))
            stream, out = o.h, esb.esb_matvec_groups(esb.esb_project_groups(u, X_FMT, 0)[0], f.w[f"down{i}"])
        o = esb.esb_rmsnorm(stream, f.norms["norm"], c.eps, residual=out, fmt=X_FMT)
        return esb.esb_matvec_groups(o.coded, f.w["head"], y_dtype=torch.float32)


def main(steps: int = 200, seed: int = 0) -> float:
    cfg = Config()
    m = Model(cfg, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    rule = torch.randperm(cfg.vocab, generator=g, device="cuda")          # the next token of each token
    for i in range(steps):
        t = torch.randint(0, cfg.vocab, (512,), generator=g, device="cuda")
        loss = m.step(t, rule[t], lr=1.0)
        if i % 50 == 0 or i == steps - 1:
            print(f"step {i}: loss {float(loss):.3f}")
    t = torch.randint(0, cfg.vocab, (16,), generator=g, device="cuda")
    a = m.serving().answer(t, rule[t], top=3)
    right = float((a.top_ids[:, 0] == rule[t]).float().mean())
    print(f"answers: {right:.0%} right, mean log p {float(a.logp.mean()):.3f}, entropy {float(a.entropy.mean()):.3f}")
    return right


if __name__ == "__main__":
    main()
