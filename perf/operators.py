"""Measured cases of the recurrent layer's operators: the gated linear recurrence, dropout, and
dropout with residual add and RMS norm.

Each case runs either as the plain form, elementary torch operations in fp32, or (``own``)
as calls of the library.  Formulas, with s() the logistic function:

recurrence   log a = -c softplus(lam) s(r),  h_t = a_t h_{t-1} + sqrt(1 - a_t^2) s(i_t) x_t,  y = h;
             at a reset a = 0; from a row's length on y = 0 and the state stays.
dropout      element e uses 16 bits of Philox4x32-10 (Salmon et al., SC 2011): key = seed,
             counter = (e // 8, offset), half-word e % 8; dropped when below t = round(65536 p),
             otherwise scaled by 65536 / (65536 - t); plus the residual, when there is one.
add + norm   y = residual + dropout(x),  rstd = 1 / sqrt(mean(y^2) + eps),  z = y rstd w;
             the backward pass takes y as it is stored.
"""

import math

import torch

own = False

DECAY_SCALE = 8.0
EPS = 1e-6
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ITEM = {"f32": 4, "f16": 2, "bf16": 2}
MOST_REC = 1 << 26      # elements of the largest recurrence
MOST_ROWS = 1 << 27     # elements of the largest rowwise case


# ---- the cases --------------------------------------------------------------------------------

def _rec(name, op, B, T, D, dtype, reset=False, ragged=False):
    return {"name": name, "op": op, "B": B, "T": T, "D": D, "dtype": dtype, "reset": reset, "ragged": ragged}


def _rows(name, op, rows, cols, dtype, p, residual=False, pad=0):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "dtype": dtype, "p": p, "residual": residual, "pad": pad}


def listed():
    return [
        # one token of one stream at hidden size 1024: generation, latency alone
        _rec("step 1x1024 bf16", "rec_step", 1, 1, 1024, "bf16"),
        # one token of each of 256 streams served together, some slots idle
        _rec("step 256x4096 bf16", "rec_step", 256, 1, 4096, "bf16", ragged=True),
        # reading one prompt of an odd length before generation: no gradient, state kept
        _rec("prompt 1x8191x1024 bf16", "rec_fwd", 1, 8191, 1024, "bf16"),
        # a small fp32 training batch of padded rows, one empty, an odd width
        _rec("train 5x777x1001 f32 ragged", "rec_train", 5, 777, 1001, "f32", ragged=True),
        # a training batch with documents packed into each row
        _rec("train 8x2048x2048 bf16 packed", "rec_train", 8, 2048, 2048, "bf16", reset=True),
        # one very long sequence: too few columns to fill the device without splitting time
        _rec("train 1x65536x1024 bf16", "rec_train", 1, 65536, 1024, "bf16"),
        # a few rows at hidden size 1024
        _rows("dropout 64x1024 bf16", "dropout", 64, 1024, "bf16", 0.1, residual=True),
        # an odd number of fp32 values
        _rows("dropout 1x1000003 f32", "dropout", 1, 1000003, "f32", 0.2),
        # the feed-forward activations of a large batch, forward and backward
        _rows("dropout train 16384x4096 bf16", "dropout_train", 16384, 4096, "bf16", 0.1),
        # the layer boundary of 8 sequences of 512 tokens at hidden size 1024
        _rows("norm 4096x1024 bf16", "norm_fwd", 4096, 1024, "bf16", 0.1),
        # an odd width in half precision, its backward pass
        _rows("norm back 333x1001 f16", "norm_bwd", 333, 1001, "f16", 0.1),
        # the layer boundary of a large batch, backward
        _rows("norm back 32768x4096 bf16", "norm_bwd", 32768, 4096, "bf16", 0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width of a model (1, 5/4 or 7/4 times a power of two), or for one in three any that is
    no multiple of 4."""
    d = _log(rng, lo, hi)
    if rng.random() < 0.35:
        return min(hi, d // 4 * 4 + 4) - rng.choice([1, 2, 3])
    k = 1 << (d.bit_length() - 1)
    return rng.choice([w for w in (k, k + k // 4, k + k // 4 * 3) if w <= hi])


def draw(rng):
    op = rng.choice(["rec_step", "rec_fwd", "rec_train", "rec_train", "dropout", "dropout_train", "norm_fwd", "norm_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "rec_step":
        c = _rec("", op, _log(rng, 1, 512), 1, _width(rng, 256, 8192), dtype, ragged=rng.random() < 0.5)
    elif op.startswith("rec"):
        D = _width(rng, 128, 4096)
        T = _log(rng, 2, 65536)
        most = MOST_REC // (2 if dtype == "f32" else 1)
        T = max(1, min(T, most // D))
        B = _log(rng, 1, max(1, min(64, most // (D * T))))
        c = _rec("", op, B, T, D, dtype, reset=rng.random() < 0.4, ragged=rng.random() < 0.4)
    else:
        most = MOST_ROWS // (2 if dtype == "f32" else 1)
        cols = _width(rng, 64, 16384)
        rows = _log(rng, 1, most // cols)
        c = _rows("", op, rows, cols, dtype, rng.choice([0.0, 0.05, 0.1, 0.1, 0.2, 0.5]),
                  residual=op == "dropout" and rng.random() < 0.5, pad=rng.choice([0, 0, 0, 8, 24, 5]))
    del c["name"]
    return c


# ---- what one pass cannot do without ----------------------------------------------------------

def work(case):
    e, op = ITEM[case["dtype"]], case["op"]
    if op == "rec_step":          # x, r, i, y, the state in and out; one slot in ten is idle in a ragged batch
        n = case["B"] * case["D"]
        live = n * (0.9 if case["ragged"] else 1.0)
        return {"bytes": (3 * e + 8) * live + e * n + 4 * case["D"], "flops": 20 * live}
    if op.startswith("rec"):
        n, bd = case["B"] * case["T"] * case["D"], case["B"] * case["D"]
        # a ragged batch: the first row is full, the last one empty, the others half full on average
        live = n / 2 if case["ragged"] and case["B"] > 1 else n
        flags = case["B"] * case["T"] if case["reset"] else 0
        if op == "rec_fwd":       # x, r, i in, y out
            return {"bytes": e * (3 * live + n) + 8 * bd + flags, "flops": 20 * live}
        # x, r, i, dy in, y, dx, dr, di out; two calls, the second of which has to read x, r and i
        # again where they are larger than a cache, which is not counted here
        return {"bytes": e * (4 * live + 4 * n) + 16 * bd + 8 * case["D"] + flags, "flops": 70 * live}
    n = case["rows"] * case["cols"]
    if op == "dropout":
        return {"bytes": (3 if case["residual"] else 2) * e * n, "flops": 12 * n}
    if op == "dropout_train":
        return {"bytes": 4 * e * n, "flops": 24 * n}
    if op == "norm_fwd":
        return {"bytes": 4 * e * n + 4 * case["rows"] + 4 * case["cols"], "flops": 18 * n}
    return {"bytes": 5 * e * n + 4 * case["rows"] + 8 * case["cols"], "flops": 26 * n}


# ---- inputs -----------------------------------------------------------------------------------

def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(seed * 7919 + 17)
    dt = TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        out = torch.empty(shape, dtype=dtype, device=dev)
        return out.normal_(0.0, scale, generator=g)

    def empty(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device=dev)

    f32 = torch.float32
    s = {"case": case}
    if case["op"].startswith("rec"):
        B, T, D = case["B"], case["T"], case["D"]
        # gate pre-activations come out of one product as halves of a row; the decay at an open
        # gate lies between 0.9 and 0.999
        u = torch.empty(D, dtype=f32, device=dev).uniform_(0.9, 0.999, generator=g)
        s["lam"] = torch.log(torch.expm1(-torch.log(u) / DECAY_SCALE))
        if case["op"] == "rec_step":
            gates = normal(B, 2 * D)
            s.update(x=normal(B, D), r=gates[:, :D], i=gates[:, D:], y=empty(B, D), slots=None)
            n = B + B // 4 + 1
            s["state"] = normal(n, D, dtype=f32)
            # each stream's state lives in a slot of a larger cache
            s["slots"] = torch.randperm(n, generator=g, device=dev)[:B].to(torch.int32)
            if case["ragged"]:
                s["slots"][torch.rand(B, generator=g, device=dev) < 0.1] = -1
            return s
        gates = normal(B, T, 2 * D)
        s.update(x=normal(B, T, D), r=gates[..., :D], i=gates[..., D:], h0=normal(B, D, dtype=f32), y=empty(B, T, D),
                 h_last=empty(B, D, dtype=f32), reset=None, lengths=None)
        if case["reset"]:
            s["reset"] = (torch.rand(B, T, generator=g, device=dev) < 4.0 / max(T, 8)).to(torch.uint8)
        if case["ragged"]:
            s["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device=dev, dtype=torch.int32)
            s["lengths"][0] = T
            if B > 1:
                s["lengths"][B - 1] = 0
        if case["op"] == "rec_train":
            s.update(dy=normal(B, T, D), dh_last=normal(B, D, dtype=f32), dx=empty(B, T, D), dr=empty(B, T, D),
                     di=empty(B, T, D), dlam=empty(D, dtype=f32), dh0=empty(B, D, dtype=f32))
        return s
    rows, cols, pad = case["rows"], case["cols"], case["pad"]
    s["seed"] = (seed * 0x9E3779B97F4A7C15 + 0x1234567) % (1 << 64)
    s["offset"] = (seed * 1000003 + 5) % (1 << 40)

    def wide(scale=1.0):     # a column slice of a wider buffer where the case has padding
        return normal(rows, cols + pad, scale=scale)[:, :cols]

    s["x"] = wide()
    s["residual"] = wide() if case["residual"] or case["op"] == "norm_fwd" else None
    s["out"] = empty(rows, cols)
    if case["op"] == "dropout_train":
        s.update(dout=wide(), dx=empty(rows, cols))
    if case["op"].startswith("norm"):
        s["weight"] = 1.0 + normal(cols, scale=0.1, dtype=f32)
    if case["op"] == "norm_fwd":
        s.update(z=empty(rows, cols), rstd=empty(rows, dtype=f32))
    if case["op"] == "norm_bwd":
        s["y"] = s.pop("x")
        s["rstd"] = torch.rsqrt(torch.linalg.vector_norm(s["y"], dim=1, dtype=f32) ** 2 / cols + EPS)
        s.update(dz=wide(), dy=wide(), dx=s.pop("out"), dresidual=empty(rows, cols), dweight=empty(cols, dtype=f32))
    return s


# ---- one pass ---------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _workspace(s, size):
    """The workspace that a program keeps beside its buffers."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(size, 1), dtype=torch.uint8, device=_device())
    return s["workspace"]


def _run_own(s):
    import paper_2108_06004_gb300 as gs

    c = s["case"]
    op = c["op"]
    if op == "rec_step":
        gs.gs_recurrence_step(s["x"], s["r"], s["i"], s["lam"], s["state"], s["y"], slots=s["slots"], c=DECAY_SCALE)
        return {"y": s["y"], "state": s["state"]}
    if op == "rec_fwd":
        gs.gs_recurrence_forward(s["x"], s["r"], s["i"], s["lam"], s["y"], h0=s["h0"], reset=s["reset"],
                                 lengths=s["lengths"], h_last=s["h_last"], c=DECAY_SCALE)
        return {"y": s["y"], "h_last": s["h_last"]}
    if op == "rec_train":
        B, T, D = c["B"], c["T"], c["D"]
        if "states" not in s:
            s["states"] = torch.empty(gs.gs_recurrence_states_size(B, T, D), dtype=torch.uint8, device=_device())
        ws = _workspace(s, gs.gs_recurrence_workspace_size(B, T, D))
        gs.gs_recurrence_forward(s["x"], s["r"], s["i"], s["lam"], s["y"], h0=s["h0"], reset=s["reset"],
                                 lengths=s["lengths"], h_last=s["h_last"], states=s["states"], c=DECAY_SCALE)
        gs.gs_recurrence_backward(s["dy"], s["x"], s["r"], s["i"], s["lam"], s["states"], s["dx"], s["dr"], s["di"],
                                  s["dlam"], ws, dh_last=s["dh_last"], reset=s["reset"], lengths=s["lengths"],
                                  dh0=s["dh0"], c=DECAY_SCALE)
        return {k: s[k] for k in ("y", "h_last", "dx", "dr", "di", "dlam", "dh0")}
    p, seed, offset = c["p"], s["seed"], s["offset"]
    if op in ("dropout", "dropout_train"):
        gs.gs_dropout(s["x"], s["out"], p, seed, offset, residual=s["residual"])
        if op == "dropout":
            return {"out": s["out"]}
        gs.gs_dropout_backward(s["dout"], s["dx"], p, seed, offset)
        return {"out": s["out"], "dx": s["dx"]}
    if op == "norm_fwd":
        gs.gs_dropout_add_norm(s["x"], s["residual"], s["weight"], s["out"], s["z"], s["rstd"], p, seed, offset, eps=EPS)
        return {"y": s["out"], "z": s["z"], "rstd": s["rstd"]}
    ws = _workspace(s, gs.gs_dropout_add_norm_workspace_size(c["rows"], c["cols"]))
    gs.gs_dropout_add_norm_backward(s["dz"], s["dy"], s["y"], s["weight"], s["rstd"], s["dx"], s["dresidual"],
                                    s["dweight"], p, seed, offset, ws)
    return {"dx": s["dx"], "dresidual": s["dresidual"], "dweight": s["dweight"]}


M32 = 0xFFFFFFFF


def _keep(n, p, seed, offset, dev):
    """(kept, scale) of n elements: the generator in 64-bit integers."""
    t = int(math.floor(p * 65536.0 + 0.5))
    blocks = torch.arange((n + 7) // 8, dtype=torch.int64, device=dev)
    x0, x1 = blocks & M32, blocks >> 32
    x2, x3 = torch.full_like(blocks, offset & M32), torch.full_like(blocks, (offset >> 32) & M32)
    k0, k1 = seed & M32, (seed >> 32) & M32
    for _ in range(10):
        m0, m1 = x0 * 0xD2511F53, x2 * 0xCD9E8D57
        x0, x1, x2, x3 = ((m1 >> 32) & M32) ^ x1 ^ k0, m1 & M32, ((m0 >> 32) & M32) ^ x3 ^ k1, m0 & M32
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    words = torch.stack((x0, x1, x2, x3), dim=1)
    halves = torch.stack((words & 0xFFFF, words >> 16), dim=2).reshape(-1)[:n]
    return halves >= t, (65536.0 / (65536 - t) if t < 65536 else 0.0)


def _drop(x, kept, scale):
    return torch.where(kept.view(x.shape), x.float() * scale, torch.zeros((), device=x.device))


def _gates(s, valid):
    """sigmoids of both gates, log a, a, the input's gain and the gated input, in fp32; a token
    past the end of its row leaves the state as it is."""
    sr, si = torch.sigmoid(s["r"].float()), torch.sigmoid(s["i"].float())
    la = -DECAY_SCALE * torch.nn.functional.softplus(s["lam"]) * sr
    a = torch.exp(la)
    gain = torch.sqrt(-torch.expm1(2 * la))
    if s.get("reset") is not None:
        at = s["reset"].bool().unsqueeze(-1)
        a, gain = a.masked_fill(at, 0.0), gain.masked_fill(at, 1.0)
    x = s["x"].float()
    if valid is not None:
        a, gain = a.masked_fill(~valid, 1.0), gain.masked_fill(~valid, 0.0)
        x = x.masked_fill(~valid, 0.0)
    return sr, si, la, a, gain, x


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t over dimension 1 from h = 0, doubling the distance each time;
    also the products of a from the start."""
    a, b, step = a.clone(), b.clone(), 1
    while step < a.shape[1]:
        b[:, step:] += a[:, step:] * b[:, :-step].clone()
        a[:, step:] *= a[:, :-step].clone()
        step *= 2
    return a, b


def _run_plain(s):
    c = s["case"]
    op, dt, dev = c["op"], TYPES[c["dtype"]], s["weight" if c["op"].startswith("norm") else "x"].device
    if op == "rec_step":
        _, si, _, a, gain, x = _gates(s, None)
        live = (s["slots"] >= 0).unsqueeze(-1)
        at = torch.where(s["slots"] >= 0, s["slots"], torch.zeros_like(s["slots"])).long()
        h = a * s["state"][at] + gain * si * x
        s["y"].copy_(torch.where(live, h, torch.zeros_like(h)))
        s["state"][at[live[:, 0]]] = h[live[:, 0]]
        return {"y": s["y"], "state": s["state"]}
    if op in ("rec_fwd", "rec_train"):
        T = c["T"]
        valid = None
        if s["lengths"] is not None:
            valid = (torch.arange(T, device=dev) < s["lengths"].unsqueeze(-1)).unsqueeze(-1)
        sr, si, la, a, gain, x = _gates(s, valid)
        products, h = _scan(a, gain * si * x)
        h += products * s["h0"].unsqueeze(1)
        y = h if valid is None else h.masked_fill(~valid, 0.0)
        out = {"y": y.to(dt), "h_last": h[:, -1].clone()}
        if op == "rec_fwd":
            return out
        before = torch.cat((s["h0"].unsqueeze(1), h[:, :-1]), dim=1)
        dy = s["dy"].float()
        if valid is not None:
            dy = dy.masked_fill(~valid, 0.0)
        dy = torch.cat((dy, s["dh_last"].unsqueeze(1)), dim=1).flip(1)
        g = _scan(torch.cat((torch.ones_like(a[:, :1]), torch.ones_like(a[:, :1]), a.flip(1)[:, :-1]), dim=1), dy)[1]
        g = g.flip(1)[:, :-1]       # the last token's own entry, and what comes from past the end
        dla = g * (a * before - si * x * a * a / gain)
        fixed = torch.zeros_like(a, dtype=torch.bool)
        if s["reset"] is not None:
            fixed |= s["reset"].bool().unsqueeze(-1)
        if valid is not None:
            fixed |= ~valid
        dla = dla.masked_fill(fixed, 0.0)
        out["dx"] = (g * gain * si).to(dt)
        out["dr"] = (dla * la * (1 - sr)).to(dt)
        out["di"] = (g * gain * x * si * (1 - si)).to(dt)
        out["dlam"] = (dla * sr).sum(dim=(0, 1)) * (-DECAY_SCALE) * torch.sigmoid(s["lam"])
        out["dh0"] = a[:, 0] * g[:, 0]
        return out
    n = c["rows"] * c["cols"]
    kept, scale = _keep(n, c["p"], s["seed"], s["offset"], dev)
    if op in ("dropout", "dropout_train"):
        t = _drop(s["x"], kept, scale)
        if s["residual"] is not None:
            t = t + s["residual"].float()
        out = {"out": t.to(dt)}
        if op == "dropout_train":
            out["dx"] = _drop(s["dout"], kept, scale).to(dt)
        return out
    if op == "norm_fwd":
        t = s["residual"].float() + _drop(s["x"], kept, scale)
        rstd = torch.rsqrt(t.square().mean(dim=1) + EPS)
        return {"y": t.to(dt), "z": (t * rstd.unsqueeze(1) * s["weight"]).to(dt), "rstd": rstd}
    normed, u = s["y"].float() * s["rstd"].unsqueeze(1), s["dz"].float() * s["weight"]
    dt_ = s["rstd"].unsqueeze(1) * (u - normed * (u * normed).mean(dim=1, keepdim=True)) + s["dy"].float()
    return {"dx": _drop(dt_, kept, scale).to(dt), "dresidual": dt_.to(dt), "dweight": (s["dz"].float() * normed).sum(dim=0)}


# ---- the definition in 64 bits ----------------------------------------------------------------

def _exact_mask(n, p, seed, offset):
    import numpy as np

    t = math.floor(p * 65536.0 + 0.5)
    low = np.uint64(M32)
    c = [np.arange((n + 7) // 8, dtype=np.uint64)]
    c = [c[0] & low, c[0] >> np.uint64(32), np.uint64(offset & M32), np.uint64(offset >> 32)]
    key = [seed & M32, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(key[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(key[1]), a & low]
        key = [(key[0] + 0x9E3779B9) & M32, (key[1] + 0xBB67AE85) & M32]
    u = np.empty((c[0].size, 8), dtype=np.uint16)
    for j in range(4):
        u[:, 2 * j] = (c[j] & np.uint64(0xFFFF)).astype(np.uint16)
        u[:, 2 * j + 1] = (c[j] >> np.uint64(16)).astype(np.uint16)
    factor = np.where(u.reshape(-1)[:n] >= t, 65536.0 / max(65536 - t, 1), 0.0)
    return torch.from_numpy(factor).to(_device())


def exact(case, seed):
    s, f64 = prepare(case, seed), torch.float64
    op = case["op"]
    if op.startswith("rec"):
        step = op == "rec_step"
        add = (lambda t: t.unsqueeze(1)) if step else (lambda t: t)
        leaves = [t.detach().to(f64).requires_grad_() for t in (add(s["x"]), add(s["r"]), add(s["i"]), s["lam"])]
        x, r, i, lam = leaves
        la = DECAY_SCALE * torch.nn.functional.logsigmoid(-lam) / (1 + torch.exp(-r))
        a = torch.exp(la)
        b = torch.sqrt((1 - a) * (1 + a)) * x / (1 + torch.exp(-i))
        B, T, D = x.shape
        live = torch.ones(B, T, 1, dtype=torch.bool, device=x.device)
        if not step:
            if s["reset"] is not None:
                at = s["reset"].bool().unsqueeze(-1)
                a, b = torch.where(at, torch.zeros_like(a), a), torch.where(at, x / (1 + torch.exp(-i)), b)
            if s["lengths"] is not None:
                live = (torch.arange(T, device=x.device)[None, :] < s["lengths"][:, None]).unsqueeze(-1)
                a, b = torch.where(live, a, torch.ones_like(a)), torch.where(live, b, torch.zeros_like(b))
        with torch.no_grad():
            if step:
                slots = s["slots"].tolist()
                state, y = s["state"].to(f64), torch.zeros(B, D, dtype=f64, device=x.device)
                rows = [k for k in range(B) if slots[k] >= 0]
                where = [slots[k] for k in rows]
                state[where] = a[rows, 0] * state[where] + b[rows, 0]
                y[rows] = state[where]
                return {"y": y, "state": state}
            at_, bt_ = a.transpose(0, 1).contiguous(), b.transpose(0, 1).contiguous()
            h = torch.empty(T + 1, B, D, dtype=f64, device=x.device)
            h[0] = s["h0"]
            for t in range(T):
                torch.addcmul(bt_[t], at_[t], h[t], out=h[t + 1])
            out = {"y": h[1:].transpose(0, 1) * live, "h_last": h[T].clone()}
            if op == "rec_fwd":
                return out
            g = (s["dy"].to(f64) * live).transpose(0, 1).contiguous()
            g[T - 1] += s["dh_last"]
            for t in range(T - 2, -1, -1):
                g[t].addcmul_(at_[t + 1], g[t + 1])
            out["dh0"] = at_[0] * g[0]
            ga, gb = (g * h[:-1]).transpose(0, 1), g.transpose(0, 1)
        out["dx"], out["dr"], out["di"], out["dlam"] = torch.autograd.grad((a, b), leaves, (ga, gb))
        return out
    rows, cols = case["rows"], case["cols"]
    factor = _exact_mask(rows * cols, case["p"], s["seed"], s["offset"]).view(rows, cols)
    if op in ("dropout", "dropout_train"):
        out = {"out": torch.where(factor > 0, s["x"].to(f64) * factor, 0.0)}
        if s["residual"] is not None:
            out["out"] += s["residual"]
        if op == "dropout_train":
            out["dx"] = torch.where(factor > 0, s["dout"].to(f64) * factor, 0.0)
        return out
    if op == "norm_fwd":
        t = s["residual"].to(f64) + s["x"].to(f64) * factor
        rstd = 1 / torch.sqrt((t * t).sum(dim=1) / cols + EPS)
        return {"y": t, "z": s["weight"].to(f64) * t * rstd[:, None], "rstd": rstd}
    y, dz, k = s["y"].to(f64), s["dz"].to(f64), s["rstd"].to(f64)[:, None]
    dw = (dz * y * k).sum(dim=0)
    dz = dz * s["weight"].to(f64)
    dt = k * dz - y * k ** 3 * (dz * y).sum(dim=1, keepdim=True) / cols + s["dy"].to(f64)
    return {"dx": dt * factor, "dresidual": dt, "dweight": dw}
