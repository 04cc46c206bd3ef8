"""The recurrent model of examples/train_recurrent.py: its gradient against one by automatic
differentiation in fp64, training with compressed gradients, and generation token by token."""

import os
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import train_recurrent
    finally:
        sys.path.pop(0)
    torch.cuda.set_device(0)
    return train_recurrent


def plain_loss(ex, cfg, flat, tokens, keep, seed, offset):
    """The model in elementary operations, in the type of `flat`."""
    from oracle import layer

    def drop(v, site):
        kept = torch.from_numpy(layer.dropout_kept(v.numel(), keep, seed, offset(0, site))).to(v.device).view(v.shape)
        t = layer.dropout_threshold(keep)
        return torch.where(kept, v * (65536 / (65536 - t)), torch.zeros_like(v))

    w, D = ex.views(flat, cfg), cfg.hidden
    seen, target = tokens[:, :-1], tokens[:, 1:]
    s = z = drop(w["embed"][seen], 0)
    for n in range(cfg.layers):
        x, gates = z @ w[f"in{n}"], z @ w[f"gates{n}"]
        la = -8 * torch.nn.functional.softplus(w[f"decay{n}"]) * torch.sigmoid(gates[..., :D])
        a, b = torch.exp(la), torch.sqrt(-torch.expm1(2 * la)) * torch.sigmoid(gates[..., D:]) * x
        h, out = torch.zeros_like(x[:, 0]), []
        for t in range(x.shape[1]):
            h = a[:, t] * h + b[:, t]
            out.append(h)
        s = s + drop(torch.stack(out, dim=1) @ w[f"out{n}"], n + 1)
        z = s * torch.rsqrt(s.square().mean(dim=-1, keepdim=True) + 1e-6) * w[f"norm{n}"]
    return torch.nn.functional.cross_entropy((z @ w["embed"].t()).flatten(0, 1) * D ** -0.5, target.flatten())


def test_gradient(example):
    ex = example
    cfg = ex.Config(vocab=17, hidden=40, batch=3, length=21, workers=1)
    flat = ex.init(cfg)
    worker = ex.Worker(cfg, 0, dtype=torch.float32)
    tokens = torch.randint(0, cfg.vocab, (cfg.batch, cfg.length + 1), device="cuda",
                           generator=torch.Generator(device="cuda").manual_seed(3))
    before = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        loss = worker.forward_backward(flat, tokens, 0)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = before
    exact = flat.double().requires_grad_()
    want = plain_loss(ex, cfg, exact, tokens, cfg.dropout, cfg.seed, worker.offset)
    (grad,) = torch.autograd.grad(want, exact)
    # fp32 through two layers of products of length 40 and 80 and a state of 21 tokens: a few
    # hundred roundings of 6e-8 at the most
    assert abs(loss.item() - want.item()) < 1e-4 * want.item()
    for name, v in ex.views(worker.grad.double(), cfg).items():
        e = ex.views(grad, cfg)[name]
        assert (v - e).norm() < 1e-4 * e.norm(), name


def test_training_and_generation(example):
    ex = example
    cfg = ex.Config()
    flat, losses = ex.train(cfg, 200)
    assert losses[-1] < 0.25 * losses[0], losses[::10]
    tokens = ex.make_tokens(cfg, 10_000, 0)
    got = ex.generate(flat, cfg, tokens[:, :20], 10)
    assert (got == tokens[:, 20:30]).float().mean().item() > 0.9
    again, losses2 = ex.train(cfg, 3)
    assert losses2 == losses[:3] or max(abs(a - b) for a, b in zip(losses2, losses)) < 1e-2
