"""A small recurrent language model trained by P simulated workers with compressed gradients.

Each worker runs the model on its own batch.  Everything but the matrix products and the loss
is a call of the library: dropout of the embeddings, the gated linear recurrence, and at each
layer's boundary dropout + residual add + RMS norm, forward and backward.  The gradients are
views into the worker's flat fp32 vector, which ``gs_train_step`` sketches, merges and turns
into a sparse update of the shared weights.  Generation carries the recurrence's state from
token to token with ``gs_recurrence_step``.

    python examples/train_recurrent.py --steps 200
"""

from __future__ import annotations

import argparse
import dataclasses
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2108_06004_gb300 as gs  # noqa: E402


@dataclasses.dataclass(frozen=True)
class Config:
    vocab: int = 64
    hidden: int = 128
    layers: int = 2
    batch: int = 16
    length: int = 64
    workers: int = 4
    dropout: float = 0.1
    rho: float = 0.9
    lr: float = 2.0
    rows: int = 5
    cols: int = 1 << 15
    keep: int = 4000
    seed: int = 1

    def shapes(self):
        d = self.hidden
        out = {"embed": (self.vocab, d)}
        for n in range(self.layers):
            out.update({f"in{n}": (d, d), f"gates{n}": (d, 2 * d), f"decay{n}": (d,), f"out{n}": (d, d), f"norm{n}": (d,)})
        return out


def views(flat, cfg: Config):
    """The parameters (or their gradients) as views of one flat vector."""
    out, at = {}, 0
    for name, shape in cfg.shapes().items():
        n = math.prod(shape)
        out[name] = flat[at:at + n].view(shape)
        at += n
    return out


def size(cfg: Config) -> int:
    return sum(math.prod(s) for s in cfg.shapes().values())


def init(cfg: Config, device="cuda"):
    gen = torch.Generator(device=device).manual_seed(cfg.seed)
    flat = torch.empty(size(cfg), device=device)
    for name, v in views(flat, cfg).items():
        if name.startswith("norm"):
            v.fill_(1.0)
        elif name.startswith("decay"):   # at an open gate the state decays by 0.9 ... 0.999 a token
            u = torch.empty_like(v).uniform_(0.9, 0.999, generator=gen)
            v.copy_(torch.log(torch.expm1(-torch.log(u) / 8.0)))
        else:
            v.normal_(0.0, 0.3 if name == "embed" else v.shape[0] ** -0.5, generator=gen)
    return flat


class Worker:
    """One worker's buffers: activations that the backward pass needs, and the library's
    workspaces, all kept from step to step."""

    def __init__(self, cfg: Config, number: int, dtype=torch.bfloat16, device="cuda"):
        self.cfg, self.number, self.dtype = cfg, number, dtype
        B, T, D = cfg.batch, cfg.length, cfg.hidden

        def act(*shape):
            return torch.empty(shape, dtype=dtype, device=device)

        self.stream = [act(B, T, D) for _ in range(cfg.layers + 1)]    # the residual stream between layers
        self.z = [None] + [act(B, T, D) for _ in range(cfg.layers)]    # its norm; a layer's input
        self.h = [act(B, T, D) for _ in range(cfg.layers)]
        self.rstd = [torch.empty(B, T, device=device) for _ in range(cfg.layers)]
        self.states = [torch.empty(gs.gs_recurrence_states_size(B, T, D), dtype=torch.uint8, device=device)
                       for _ in range(cfg.layers)]
        need = max(gs.gs_recurrence_workspace_size(B, T, D), gs.gs_dropout_add_norm_workspace_size(B * T, D))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)
        self.grad = torch.zeros(size(cfg), device=device)

    def offset(self, step: int, site: int) -> int:
        """Another mask for every worker, step and place in the model."""
        return (step * (self.cfg.layers + 1) + site) * self.cfg.workers + self.number

    def forward_backward(self, flat, tokens, step: int, p=None):
        """The mean loss on tokens [B][T + 1]; fills self.grad."""
        cfg, p = self.cfg, self.cfg.dropout if p is None else p
        w, g = views(flat, cfg), views(self.grad, cfg)
        low = {k: v.to(self.dtype) for k, v in w.items()}
        B, T, D = cfg.batch, cfg.length, cfg.hidden
        seen, target = tokens[:, :-1], tokens[:, 1:]
        gs.gs_dropout(low["embed"][seen], self.stream[0], p, cfg.seed, self.offset(step, 0))
        self.z[0] = self.stream[0]
        x, gates = [], []
        for n in range(cfg.layers):
            x.append(self.z[n] @ low[f"in{n}"])
            gates.append(self.z[n] @ low[f"gates{n}"])
            r, i = gates[n][..., :D], gates[n][..., D:]
            gs.gs_recurrence_forward(x[n], r, i, w[f"decay{n}"], self.h[n], states=self.states[n])
            gs.gs_dropout_add_norm(self.h[n] @ low[f"out{n}"], self.stream[n], w[f"norm{n}"], self.stream[n + 1],
                                   self.z[n + 1], self.rstd[n], p, cfg.seed, self.offset(step, n + 1))
        top = self.z[cfg.layers]
        logp = torch.log_softmax((top @ low["embed"].t()).float() * D ** -0.5, dim=-1)
        loss = -logp.gather(-1, target.unsqueeze(-1)).mean()
        dlogits = logp.exp()
        dlogits.scatter_add_(-1, target.unsqueeze(-1), torch.full_like(dlogits[..., :1], -1.0))
        dlogits = (dlogits * (D ** -0.5 / (B * T))).to(self.dtype)

        def weight_grad(name, inputs, outputs):
            g[name].copy_(inputs.reshape(-1, inputs.shape[-1]).t() @ outputs.reshape(-1, outputs.shape[-1]))

        weight_grad("embed", dlogits, top)
        dz, ds = dlogits @ low["embed"], None
        for n in reversed(range(cfg.layers)):
            do, dres, dh = (torch.empty_like(self.h[n]) for _ in range(3))
            gs.gs_dropout_add_norm_backward(dz, ds, self.stream[n + 1], w[f"norm{n}"], self.rstd[n], do, dres, g[f"norm{n}"],
                                            p, cfg.seed, self.offset(step, n + 1), self.workspace)
            weight_grad(f"out{n}", self.h[n], do)
            torch.matmul(do, low[f"out{n}"].t(), out=dh)
            r, i = gates[n][..., :D], gates[n][..., D:]
            dx, dgates = torch.empty_like(x[n]), torch.empty_like(gates[n])
            gs.gs_recurrence_backward(dh, x[n], r, i, w[f"decay{n}"], self.states[n], dx, dgates[..., :D], dgates[..., D:],
                                      g[f"decay{n}"], self.workspace)
            weight_grad(f"in{n}", self.z[n], dx)
            weight_grad(f"gates{n}", self.z[n], dgates)
            dz = dx @ low[f"in{n}"].t() + dgates @ low[f"gates{n}"].t()
            ds = dres
        de = torch.empty_like(ds)
        gs.gs_dropout_backward(ds + dz, de, p, cfg.seed, self.offset(step, 0))
        g["embed"].index_add_(0, seen.reshape(-1), de.reshape(-1, D).float())
        return loss


def make_tokens(cfg: Config, step: int, worker: int, device="cuda"):
    """Sequences that count up by three from a random start: the next token follows from the last."""
    gen = torch.Generator(device=device).manual_seed(cfg.seed * 1_000_003 + step * 101 + worker)
    start = torch.randint(0, cfg.vocab, (cfg.batch, 1), generator=gen, device=device)
    return (start + 3 * torch.arange(cfg.length + 1, device=device)) % cfg.vocab


def train(cfg: Config, steps: int, report=None):
    """Trains and returns (weights, losses)."""
    P, d = cfg.workers, size(cfg)
    flat = init(cfg)
    workers = [Worker(cfg, p) for p in range(P)]
    us, es = ([torch.zeros(d, device="cuda") for _ in range(P)] for _ in range(2))
    idx, vals = torch.empty(cfg.keep, dtype=torch.int64, device="cuda"), torch.empty(cfg.keep, device="cuda")
    ws = torch.empty(gs.gs_step_workspace_size(d, cfg.keep), dtype=torch.uint8, device="cuda")
    sketch = gs.gs_sketch_create(cfg.rows, cfg.cols, cfg.seed, P)
    losses = []
    try:
        for t in range(steps):
            loss = [w.forward_backward(flat, make_tokens(cfg, t, p), t) for p, w in enumerate(workers)]
            gs.gs_train_step(sketch, flat, cfg.lr / P, us, es, [w.grad for w in workers], d, cfg.rho, cfg.keep, idx, vals,
                             None, ws)
            losses.append(torch.stack(loss).mean().item())
            if report:
                report(t, losses[-1])
    finally:
        gs.gs_sketch_destroy(sketch)
    return flat, losses


def generate(flat, cfg: Config, prompt, count: int, dtype=torch.bfloat16):
    """Continues each row of prompt [B][T] by `count` tokens, the likeliest each time."""
    w = views(flat, cfg)
    low = {k: v.to(dtype) for k, v in w.items()}
    B, T, D = prompt.shape[0], prompt.shape[1], cfg.hidden
    state = [torch.zeros(B, D, device="cuda") for _ in range(cfg.layers)]

    def run(tokens):
        s = z = low["embed"][tokens]
        for n in range(cfg.layers):
            x, gates = z @ low[f"in{n}"], z @ low[f"gates{n}"]
            h, y, z = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
            r, i = gates[..., :D], gates[..., D:]
            if tokens.dim() == 2:
                gs.gs_recurrence_forward(x, r, i, w[f"decay{n}"], h, h_last=state[n])
            else:
                gs.gs_recurrence_step(x, r, i, w[f"decay{n}"], state[n], h)
            gs.gs_dropout_add_norm(h @ low[f"out{n}"], s, w[f"norm{n}"], y, z, torch.empty(x.shape[:-1], device="cuda"),
                                   0.0, 0, 0)
            s = y
        return z @ low["embed"].t()

    out = [run(prompt)[:, -1].argmax(dim=-1)]
    for _ in range(count - 1):
        out.append(run(out[-1]).argmax(dim=-1))
    return torch.stack(out, dim=1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    a = ap.parse_args()
    cfg = Config()
    flat, losses = train(cfg, a.steps, lambda t, v: print(f"step {t:3d}  loss {v:.4f}") if t % 10 == 0 else None)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} ({size(cfg)} parameters, {cfg.keep} updated a step)")
    tokens = make_tokens(cfg, 10_000, 0)
    got = generate(flat, cfg, tokens[:, :20], 10)
    print(f"continued correctly: {(got == tokens[:, 20:30]).float().mean().item():.2f} of tokens")


if __name__ == "__main__":
    main()
