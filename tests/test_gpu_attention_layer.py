"""A linear attention layer made of the library's operators: rotary positions of queries and keys, linear attention with
a decay for each head, the heads' norm with its gate, an output projection, and the layer's boundary (norm, gate,
residual scale, next norm).  Forward and backward against the same layer in fp64 with PyTorch's gradients, captured and
replayed, on several streams at once, and from a prompt to single tokens."""

import math

import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_attention import gs  # noqa: E402, F401

pytestmark = pytest.mark.gpu

B, T, H, K, D = 3, 200, 4, 2, 64
HIDDEN = 96
EPS, SCALE, RES = 1e-5, D ** -0.5, 0.5
DECAY = [-0.7, -0.1, -0.02, -0.003]


def weights(dtype):
    gen = torch.Generator(device="cuda").manual_seed(1)

    def draw(*shape):
        return torch.randn(shape, generator=gen, device="cuda") / math.sqrt(shape[0])

    w = {"qkv": draw(HIDDEN, (H + 2 * K) * D), "gate": draw(HIDDEN, H * D), "out": draw(H * D, HIDDEN), "gate2": draw(HIDDEN, HIDDEN)}
    w = {k: v.to(dtype) for k, v in w.items()}
    for name, n in (("norm", H * D), ("norm1", HIDDEN), ("norm2", HIDDEN)):
        w[name] = 1 + 0.1 * torch.randn(n, generator=gen, device="cuda")
    return w


class Layer:
    """The layer's buffers for B x T tokens; every call is on the current stream."""

    def __init__(self, gs, w, dtype, B=B, T=T, first=0):
        self.gs, self.w, self.dtype, self.sizes, self.first = gs, w, dtype, (B, T), first
        f32 = torch.float32

        def act(*shape, t=dtype):
            return torch.empty(shape, dtype=t, device="cuda")

        self.qkv, self.gate, self.o, self.n = act(B, T, H + 2 * K, D), act(B, T, H * D), act(B, T, H, D), act(B, T, H * D)
        self.rstd, self.branch, self.gate2 = act(B, T, H, t=f32), act(B, T, HIDDEN), act(B, T, HIDDEN)
        self.y, self.z, self.r1, self.r2 = act(B, T, HIDDEN), act(B, T, HIDDEN), act(B, T, 1, t=f32), act(B, T, t=f32)
        self.g, self.freq = torch.tensor(DECAY, device="cuda"), gs.gs_rotary_frequencies(D).cuda()
        self.state = act(B, H, D, D, t=f32)
        need = max(gs.gs_linear_attention_workspace_size(B, T, H, K, D, D, dtype, backward=back) for back in (False, True))
        need = max(need, gs.gs_gated_norm_workspace_size(B * T, H * D, H), gs.gs_gated_norm_workspace_size(B * T, HIDDEN))
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def turn(self, x, inverse=False):
        self.gs.gs_rotary(x[:, :, :H + K], x[:, :, :H + K], self.freq, first=self.first, inverse=inverse)

    def forward(self, x, lengths=None, step=False):
        gs, w, (B, T) = self.gs, self.w, self.sizes
        torch.matmul(x, w["qkv"], out=self.qkv.view(B, T, -1))
        torch.matmul(x, w["gate"], out=self.gate)
        self.turn(self.qkv)
        q, k, v = self.qkv[:, :, :H], self.qkv[:, :, H:H + K], self.qkv[:, :, H + K:]
        if step:
            gs.gs_linear_attention_step(q[:, 0], k[:, 0], v[:, 0], self.g, self.state, self.o[:, 0], scale=SCALE)
        else:
            gs.gs_linear_attention_forward(q, k, v, self.g, self.o, self.ws, lengths=lengths, s_last=self.state, scale=SCALE)
        gs.gs_gated_norm(self.o.view(B, T, H * D), w["norm"], self.n, self.rstd, gate=self.gate, groups=H, eps=EPS)
        torch.matmul(self.n, w["out"], out=self.branch)
        torch.matmul(x, w["gate2"], out=self.gate2)
        gs.gs_gated_norm(self.branch, w["norm1"], self.y, self.r1, gate=self.gate2, residual=x, next_weight=w["norm2"], z=self.z,
                         next_rstd=self.r2, activation="sigmoid", scale=RES, eps=EPS)
        return self.y, self.z

    def backward(self, x, dy, dz, lengths=None):
        gs, w, (B, T) = self.gs, self.w, self.sizes
        new = torch.empty_like
        out = {n: torch.empty(w[n].shape, device="cuda") for n in ("norm", "norm1", "norm2")}
        dbranch, dgate2, dx = new(self.branch), new(self.gate2), new(x)
        gs.gs_gated_norm_backward(dy, self.branch, w["norm1"], self.r1, dbranch, out["norm1"], self.ws, gate=self.gate2, dgate=dgate2, dz=dz,
                                  y=self.y, next_weight=w["norm2"], next_rstd=self.r2, dresidual=dx, dnext_weight=out["norm2"],
                                  activation="sigmoid", scale=RES)
        dn, do, dgate = dbranch @ w["out"].t(), new(self.o), new(self.gate)
        gs.gs_gated_norm_backward(dn, self.o.view(B, T, -1), w["norm"], self.rstd, do.view(B, T, -1), out["norm"], self.ws, gate=self.gate,
                                  dgate=dgate, groups=H)
        dqkv = new(self.qkv)
        part = [self.qkv[:, :, :H], self.qkv[:, :, H:H + K], self.qkv[:, :, H + K:]]
        gs.gs_linear_attention_backward(do, *part, self.g, dqkv[:, :, :H], dqkv[:, :, H:H + K], dqkv[:, :, H + K:], self.ws, lengths=lengths,
                                        scale=SCALE)
        self.turn(dqkv, inverse=True)
        flat = lambda t: t.reshape(-1, t.shape[-1])   # noqa: E731
        for name, a, b in (("qkv", x, dqkv.view(B, T, -1)), ("gate", x, dgate), ("out", self.n, dbranch), ("gate2", x, dgate2)):
            out[name] = flat(a).t() @ flat(b)
        out["x"] = dx + dqkv.view(B, T, -1) @ w["qkv"].t() + dgate @ w["gate"].t() + dgate2 @ w["gate2"].t()
        return out


def reference(w, x, lengths=None, first=0):
    """y, z in fp64."""
    B, T = x.shape[:2]
    qkv = (x @ w["qkv"]).view(B, T, H + 2 * K, D)
    f = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    a = (first + torch.arange(T, device="cuda", dtype=torch.float64))[:, None] * f
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    p, q = qkv[..., :H + K, :D // 2], qkv[..., :H + K, D // 2:]
    turned = torch.cat((p * c - q * s, p * s + q * c), dim=-1)
    q, k, v = turned[:, :, :H], turned[:, :, H:].repeat_interleave(H // K, 2), qkv[:, :, H + K:].repeat_interleave(H // K, 2)
    t = torch.arange(T, device="cuda")
    d = t[:, None] - t[None, :]
    g = torch.tensor(DECAY, device="cuda").double()
    m = torch.where(d >= 0, torch.exp(g[:, None, None] * d.clamp(min=0)), 0.0)
    o = SCALE * torch.einsum("bihd,bjhd,hij,bjhe->bihe", q, k, m, v)
    if lengths is not None:
        o = o * (t[None, :] < torch.tensor(lengths, device="cuda")[:, None])[..., None, None]
    n = (o * torch.rsqrt(o.square().mean(-1, keepdim=True) + EPS)).reshape(B, T, H * D) * w["norm"] * torch.nn.functional.silu(x @ w["gate"])
    b = n @ w["out"]
    y = x + RES * torch.sigmoid(x @ w["gate2"]) * (b * torch.rsqrt(b.square().mean(-1, keepdim=True) + EPS)) * w["norm1"]
    return y, y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * w["norm2"]


def near(got, want, rel, what):
    off = float((got.detach().double() - want.detach()).norm() / want.detach().norm())
    assert off < rel, (what, off)


# What one rounding to the type leaves, relative to a tensor's norm, is at most eps / 2; a value passes through up to a
# dozen stored tensors (x, products, o, n, the branch, their gradients and back), each of which the layer's norms and gates may
# magnify by a few: 32 roundings are allowed, added up.
REL = {torch.float32: 32 * 2.0 ** -24 * 8, torch.bfloat16: 32 * 2.0 ** -9, torch.float16: 32 * 2.0 ** -12}


@pytest.mark.parametrize("lengths", [None, [200, 61, 128]])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_layer(gs, dtype, lengths):
    w = weights(dtype)
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, dy, dz = (torch.randn(B, T, HIDDEN, generator=gen, device="cuda").to(dtype) for _ in range(3))
    whole = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    layer = Layer(gs, w, dtype, first=1000)
    torch.backends.cuda.matmul.allow_tf32 = False
    y, z = layer.forward(x, whole)
    got = layer.backward(x, dy, dz, whole)
    leaves = {k: v.double().requires_grad_() for k, v in w.items()}
    xs = x.double().requires_grad_()
    ry, rz = reference(leaves, xs, lengths, 1000)
    near(y, ry, REL[dtype], "y")
    near(z, rz, REL[dtype], "z")
    names = list(leaves)
    grads = torch.autograd.grad((ry * dy.double()).sum() + (rz * dz.double()).sum(), [xs] + [leaves[n] for n in names])
    for n, want in zip(["x"] + names, grads):
        near(got[n], want, 2 * REL[dtype], n)


def test_captured_and_replayed(gs):
    """A whole training pass in a graph, replayed on new inputs, next to eager passes with buffers of their own."""
    dtype = torch.bfloat16
    w = weights(dtype)
    layer, eager = Layer(gs, w, dtype), Layer(gs, w, dtype)
    x, dy, dz = (torch.randn(B, T, HIDDEN, device="cuda").to(dtype) for _ in range(3))

    def run(it):
        y, z = it.forward(x)
        return [y, z] + list(it.backward(x, dy, dz).values())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(layer)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run(layer)
    for seed in range(3):
        for t in (x, dy, dz):
            t.copy_(torch.randn(t.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        for a, b in zip(captured, run(eager)):
            assert torch.equal(a, b)


def test_streams_at_once(gs):
    """Layers with buffers of their own on four streams give what each gives alone."""
    dtype = torch.bfloat16
    w = weights(dtype)
    xs = [torch.randn(B, T, HIDDEN, device="cuda").to(dtype) for _ in range(4)]
    layers, streams = [Layer(gs, w, dtype) for _ in xs], [torch.cuda.Stream() for _ in xs]
    want = []
    for it, x in zip(layers, xs):
        want.append([t.clone() for t in it.forward(x)] + list(it.backward(x, x, x).values()))
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for it, x, s in zip(layers, xs, streams):
            with torch.cuda.stream(s):
                y, z = it.forward(x)
                got.append([y, z] + list(it.backward(x, x, x).values()))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_prompt_then_tokens(gs):
    """Reading a prompt and then single tokens gives what one pass over all of them gives, to the type's rounding."""
    dtype = torch.bfloat16
    w = weights(dtype)
    x = torch.randn(B, T, HIDDEN, device="cuda").to(dtype)
    y, z = (t.clone() for t in Layer(gs, w, dtype).forward(x))
    n = T - 6
    layer = Layer(gs, w, dtype, T=n)
    near(layer.forward(x[:, :n].contiguous())[1], z[:, :n].double(), 2.0 ** -7, "prompt")
    step = Layer(gs, w, dtype, T=1)
    step.state.copy_(layer.state)
    for t in range(n, T):
        step.first = t
        near(step.forward(x[:, t:t + 1].contiguous(), step=True)[1], z[:, t:t + 1].double(), 2.0 ** -6, t)


def test_results_do_not_depend_on_what_was_there(gs):
    """Outputs and workspaces of NaN and of zeros give the same bits."""
    dtype = torch.bfloat16
    w = weights(dtype)
    x = torch.randn(B, T, HIDDEN, device="cuda").to(dtype)
    seen = []
    for fill in (float("nan"), 0.0):
        layer = Layer(gs, w, dtype)
        for t in vars(layer).values():
            if torch.is_tensor(t) and t.is_floating_point() and t is not layer.g and t is not layer.freq:
                t.fill_(fill)
        layer.ws.fill_(255 if fill != 0 else 0)
        out = [t.clone() for t in layer.forward(x)]
        layer.ws.fill_(255 if fill != 0 else 0)
        seen.append(out + list(layer.backward(x, x, x).values()))
    assert all(torch.equal(a, b) for a, b in zip(*seen))
