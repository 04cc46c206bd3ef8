"""Measured cases of a linear attention layer's operators: rotary positions, linear attention with a
decay for each head, and the norms around a block with its gate and residual scale.

Each case runs either as the plain form, elementary torch operations in fp32 (fp64 for angles), or
(``own``) as calls of the library.  Formulas, per sequence and head:

attention    S_t = e^g S_{t-1} + k_t v_t',  o_t = scale S_t' q_t,  S_{-1} = s0; g <= 0 is the head's log
             decay; several heads may share one k and v.  With the gradients dS_t of the states,
             dS_t = e^g dS_{t+1} + scale q_t do_t',  dq_t = scale S_t do_t,  dk_t = dS_t v_t,  dv_t = dS_t' k_t.
             A step is one token of each of many streams, whose states lie in slots of a cache.
rotary       pair j of a head turns by position * frequency_j; a pair is two adjacent elements (interleaved)
             or one of each half of the rotated part; the rest of the head stays.
gated norm   rstd = 1 / sqrt(mean(x^2) + eps) for each group of a row's columns,
             y = residual + scale act(gate) x rstd w,  and where there is a next norm, over whole rows,
             z = y rstd_next w_next.  The backward pass takes y as it is stored.
"""

import math

import torch

own = False

EPS = 1e-6
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ITEM = {"f32": 4, "f16": 2, "bf16": 2}
MOST_HEADS = 1 << 27    # elements of the queries of the largest attention
MOST_STATE = 1 << 26    # elements of the states of the largest step
MOST_ROWS = 1 << 27     # elements of the largest rotary or norm case
BASE, FACTOR, ORIGINAL = 10000.0, 8.0, 4096    # of the rotary frequencies


# ---- the cases --------------------------------------------------------------------------------

def _att(name, op, B, T, H, K, dk, dv, dtype, mask="none"):
    return {"name": name, "op": op, "B": B, "T": T, "H": H, "K": K, "dk": dk, "dv": dv, "dtype": dtype, "mask": mask}


def _rot(name, B, T, H, D, R, dtype, interleaved=False, inplace=True, inverse=False, pad=0):
    return {"name": name, "op": "rotary", "B": B, "T": T, "H": H, "D": D, "R": R, "dtype": dtype, "interleaved": interleaved,
            "inplace": inplace, "inverse": inverse, "pad": pad}


def _norm(name, op, rows, cols, groups, dtype, gate="silu", residual=True, follow=True, pad=0):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "groups": groups, "dtype": dtype, "gate": gate,
            "residual": residual, "follow": follow, "pad": pad}


def listed():
    return [
        # one token of one stream, a small layer: generation, latency alone
        _att("step 1x16x64 bf16", "att_step", 1, 1, 16, 16, 64, 64, "bf16"),
        # one token of each of 200 streams served together, some slots idle
        _att("step 200x16x128 bf16", "att_step", 200, 1, 16, 16, 128, 128, "bf16", "ragged"),
        # reading one prompt of an odd length before generation: few heads, state kept
        _att("prompt 1x8191x16x64 bf16", "att_fwd", 1, 8191, 16, 16, 64, 64, "bf16"),
        # a batch of padded prompts, one empty; groups of four heads share a key and value
        _att("prompt 8x2048x32/8x128 f16", "att_fwd", 8, 2048, 32, 8, 128, 128, "f16", "ragged"),
        # a small fp32 training batch of padded rows, odd head sizes
        _att("train 5x333x3x40/72 f32", "att_train", 5, 333, 3, 3, 40, 72, "f32", "ragged"),
        # documents of many lengths packed into one row
        _att("train 24 in 32768x16x64 bf16", "att_train", 24, 32768, 16, 16, 64, 64, "bf16", "packed"),
        # a large training batch
        _att("train 16x4096x16x128 bf16", "att_train", 16, 4096, 16, 16, 128, 128, "bf16"),
        # queries and keys of one new token of each of 32 streams far into their texts
        _rot("rotary 32x1x40x128 bf16", 32, 1, 40, 128, 128, "bf16"),
        # queries and keys of a training batch, part of each head turned, adjacent pairs
        _rot("rotary 8x4096x40x128/64 bf16", 8, 4096, 40, 128, 64, "bf16", interleaved=True, inplace=False),
        # the layer boundary of 8 sequences of 512 tokens at hidden size 1024
        _norm("norm 4096x1024 bf16", "norm_fwd", 4096, 1024, 1, "bf16"),
        # the norm of each head with its gate, before the output projection, in half precision
        _norm("norm back 8192x16x128 f16", "norm_bwd", 8192, 2048, 16, "f16", residual=False, follow=False),
        # the layer boundary of a large batch, backward
        _norm("norm back 32768x4096 bf16", "norm_bwd", 32768, 4096, 1, "bf16"),
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


def _head(rng):
    return rng.choice([32, 64, 64, 64, 80, 96, 128, 128, 128, 128, 160, 256, 47])


def draw(rng):
    op = rng.choice(["att_step", "att_fwd", "att_fwd", "att_train", "att_train", "rotary", "rotary", "norm_fwd", "norm_bwd"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])
    if op.startswith("att"):
        dk = _head(rng)
        dv = dk if rng.random() < 0.7 else _head(rng)
        K = rng.choice([1, 2, 4, 5, 8, 12, 16, 16, 32])
        H = K * (rng.choice([2, 4]) if K <= 16 and rng.random() < 0.3 else 1)
        mask = rng.choice(["none", "none", "ragged", "packed"])
        if op == "att_step":
            B = _log(rng, 1, max(1, min(512, MOST_STATE // (H * dk * dv))))
            c = _att("", op, B, 1, H, K, dk, dv, dtype, "ragged" if mask == "ragged" else "none")
        else:
            # the plain form keeps a state for each 128 tokens
            most = MOST_HEADS // (2 if dtype == "f32" else 1) // (H * max(dk, dv) * (2 if max(dk, dv) > 128 else 1))
            T = max(1, min(_log(rng, 2, 65536), most))
            B = _log(rng, 1, max(1, min(64, most // T, MOST_STATE // (4 * H * dk * dv))))
            if mask == "packed":
                T = max(1, min(T * max(1, B // 2), most // 2))
            c = _att("", op, B, T, H, K, dk, dv, dtype, mask)
    elif op == "rotary":
        D = _head(rng)
        R = D // 2 * 2 if rng.random() < 0.6 else max(2, D // rng.choice([2, 4]) // 2 * 2)
        H = rng.choice([1, 2, 8, 12, 16, 40, 48])
        most = MOST_ROWS // (2 if dtype == "f32" else 1) // (H * D)
        B = _log(rng, 1, 64)
        T = _log(rng, 1, max(1, most // B))
        c = _rot("", B, T, H, D, R, dtype, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.3, rng.choice([0, 0, 8, 3]))
    else:
        heads = rng.random() < 0.35
        most = MOST_ROWS // (2 if dtype == "f32" else 1)
        groups, cols = 1, _width(rng, 64, 16384)
        if heads:
            groups = rng.choice([2, 4, 8, 12, 16, 32])
            cols = groups * _head(rng)
        rows = _log(rng, 1, most // cols)
        gate = rng.choice(["silu", "silu", "sigmoid", "none"])
        c = _norm("", op, rows, cols, groups, dtype, gate, not heads, not heads and rng.random() < 0.8, rng.choice([0, 0, 0, 8, 24, 5]))
    del c["name"]
    return c


# ---- what one pass cannot do without ----------------------------------------------------------

def work(case):
    e, op = ITEM[case["dtype"]], case["op"]
    if op.startswith("att"):
        B, T, H, K, dk, dv = (case[k] for k in ("B", "T", "H", "K", "dk", "dv"))
        rows = 1 if case["mask"] == "packed" else B
        state = H * dk * dv
        if op == "att_step":      # the state in and out; one slot in ten is idle in a ragged batch
            live = B * (0.9 if case["mask"] == "ragged" else 1.0)
            return {"bytes": live * (8 * state + e * (H * dk + K * (dk + dv))) + e * B * H * dv, "flops": live * 5 * state}
        n = rows * T
        # a ragged batch: the first row is full, the last one empty, the others half full on average
        live = n / 2 if case["mask"] == "ragged" and B > 1 else n
        q, kv, o = H * dk, K * (dk + dv), H * dv
        if op == "att_fwd":       # q, k, v in, o out; the first and last states
            return {"bytes": e * (live * (q + kv) + n * o) + 8 * B * state, "flops": 4 * live * state}
        # q, k, v, do in, o, dq, dk, dv out; the first and last states and their gradients; the second
        # call has to read q, k and v again where they are larger than a cache, which is not counted here
        return {"bytes": e * (live * (q + kv + o) + n * (o + q + kv)) + 16 * B * state, "flops": 14 * live * state}
    if op == "rotary":
        tokens = case["B"] * case["T"]
        moved = case["R"] if case["inplace"] else case["D"]
        return {"bytes": tokens * (2 * e * case["H"] * moved + 4), "flops": tokens * case["H"] * case["R"] * 3}
    n, rows = case["rows"] * case["cols"], case["rows"]
    gate, res, follow = case["gate"] != "none", case["residual"], case["follow"]
    if op == "norm_fwd":          # x, gate, residual in; y, z out
        return {"bytes": e * n * (2 + gate + res + follow) + 4 * rows * (case["groups"] + follow) + 4 * case["cols"] * (1 + follow),
                "flops": n * (6 + 8 * gate + 4 * follow)}
    # dy, x, gate, dz and y in; dx, dgate, dresidual out
    return {"bytes": e * n * (3 + 2 * gate + 2 * follow + (res and follow)) + 4 * rows * (case["groups"] + follow)
            + 8 * case["cols"] * (1 + follow), "flops": n * (10 + 12 * gate + 8 * follow)}


# ---- inputs -----------------------------------------------------------------------------------

def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _frequencies(R, dev):
    """Frequencies for contexts FACTOR times as long as the ORIGINAL ones: turns that the original length
    saw fewer than once are slowed down by the factor, those that it saw over 32 times stay."""
    f = BASE ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    stay = ((ORIGINAL * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
    return (f * (stay + (1 - stay) / FACTOR)).to(dev)


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(seed * 7919 + 17)
    dt, f32 = TYPES[case["dtype"]], torch.float32

    def normal(*shape, scale=1.0, dtype=dt):
        out = torch.empty(shape, dtype=dtype, device=dev)
        return out.normal_(0.0, scale, generator=g)

    def empty(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device=dev)

    s = {"case": case}
    if case["op"].startswith("att"):
        B, T, H, K, dk, dv = (case[k] for k in ("B", "T", "H", "K", "dk", "dv"))
        rows = 1 if case["mask"] == "packed" else B
        # queries, keys and values come out of one product, as parts of a row
        x = normal(rows, T, H * dk + K * dk + K * dv)
        s["q"] = x[..., :H * dk].unflatten(-1, (H, dk))
        s["k"] = x[..., H * dk:(H + K) * dk].unflatten(-1, (K, dk))
        s["v"] = x[..., (H + K) * dk:].unflatten(-1, (K, dv))
        s["scale"] = dk ** -0.5
        # heads forget within 2 to 1000 tokens
        s["g"] = -torch.exp(torch.empty(H, dtype=f32, device=dev).uniform_(-7.0, -0.5, generator=g))
        s["o"] = empty(rows, T, H, dv)
        if case["op"] == "att_step":
            for k in ("q", "k", "v", "o"):
                s[k] = s[k][:, 0]
            n = B + B // 4 + 1
            s["state"] = normal(n, H, dk, dv, dtype=f32)
            # each stream's state lives in a slot of a larger cache
            s["slots"] = torch.randperm(n, generator=g, device=dev)[:B].to(torch.int32)
            if case["mask"] == "ragged":
                s["slots"][torch.rand(B, generator=g, device=dev) < 0.1] = -1
            return s
        s.update(s0=normal(B, H, dk, dv, dtype=f32), s_last=empty(B, H, dk, dv, dtype=f32), lengths=None, offsets=None)
        if case["mask"] == "ragged":
            s["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device=dev, dtype=torch.int32)
            s["lengths"][0] = T
            if B > 1:
                s["lengths"][B - 1] = 0
        if case["mask"] == "packed":
            # lengths of documents between a third of the mean and five thirds of it
            part = torch.empty(B, dtype=torch.float64, device=dev).uniform_(1 / 3, 5 / 3, generator=g)
            ends = (part.cumsum(0) / part.sum() * T).round().to(torch.int32)
            s["offsets"] = torch.cat((torch.zeros_like(ends[:1]), ends))
        if case["op"] == "att_train":
            s.update(do=normal(rows, T, H, dv), ds_last=normal(B, H, dk, dv, dtype=f32), dq=empty(rows, T, H, dk),
                     dk=empty(rows, T, K, dk), dv=empty(rows, T, K, dv), ds0=empty(B, H, dk, dv, dtype=f32))
        return s
    if case["op"] == "rotary":
        B, T, H, D, R = (case[k] for k in ("B", "T", "H", "D", "R"))
        s["x"] = normal(B, T, H, D + case["pad"])[..., :D]
        s["out"] = s["x"] if case["inplace"] else empty(B, T, H, D)
        s["freq"] = _frequencies(R, dev)
        # a call starts anywhere in a text, each stream at a place of its own
        first = torch.randint(0, int(FACTOR * ORIGINAL), (B, 1), generator=g, device=dev, dtype=torch.int32)
        s["positions"] = first + torch.arange(T, device=dev, dtype=torch.int32)
        return s
    rows, cols, groups, pad = (case[k] for k in ("rows", "cols", "groups", "pad"))

    def wide(scale=1.0):     # a column slice of a wider buffer where the case has padding
        return normal(rows, cols + pad, scale=scale)[:, :cols]

    s["x"], s["y"] = wide(), empty(rows, cols)
    s["gate"] = wide() if case["gate"] != "none" else None
    s["residual"] = wide() if case["residual"] else None
    s["scale"] = 0.5
    s["weight"] = 1.0 + normal(cols, scale=0.1, dtype=f32)
    s["follow"] = 1.0 + normal(cols, scale=0.1, dtype=f32) if case["follow"] else None
    s["rstd"] = empty(rows, groups, dtype=f32)
    s["z"], s["rstd2"] = (empty(rows, cols), empty(rows, dtype=f32)) if case["follow"] else (None, None)
    if case["op"] == "norm_bwd":
        norms = torch.linalg.vector_norm(s["x"].unflatten(-1, (groups, -1)), dim=-1, dtype=f32)
        s["rstd"] = torch.rsqrt(norms ** 2 * (groups / cols) + EPS)
        s["dy"], s["dz"] = wide(), None
        if case["follow"]:
            s["y"], s["dz"] = wide(), wide()
            s["rstd2"] = torch.rsqrt(torch.linalg.vector_norm(s["y"], dim=1, dtype=f32) ** 2 / cols + EPS)
        s.update(dx=empty(rows, cols), dgate=empty(rows, cols) if s["gate"] is not None else None,
                 dresidual=empty(rows, cols) if s["residual"] is not None and case["follow"] else None,
                 dweight=empty(cols, dtype=f32), dfollow=empty(cols, dtype=f32) if case["follow"] else None)
    return s


# ---- one pass ---------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _workspace(s, name, size):
    """The workspace that a program keeps beside its buffers."""
    if name not in s:
        s[name] = torch.empty(max(size(), 1), dtype=torch.uint8, device=_device())
    return s[name]


def _run_own(s):
    import paper_2108_06004_gb300 as gs

    c = s["case"]
    op = c["op"]
    if op == "att_step":
        gs.gs_linear_attention_step(s["q"], s["k"], s["v"], s["g"], s["state"], s["o"], slots=s["slots"], scale=s["scale"])
        return {"o": s["o"], "state": s["state"]}
    if op.startswith("att"):
        sizes = (c["B"], c["T"], c["H"], c["K"], c["dk"], c["dv"])
        more = {"lengths": s["lengths"], "offsets": s["offsets"], "scale": s["scale"]}
        ws = _workspace(s, "ws", lambda: gs.gs_linear_attention_workspace_size(*sizes, s["q"].dtype, packed=s["offsets"] is not None))
        gs.gs_linear_attention_forward(s["q"], s["k"], s["v"], s["g"], s["o"], ws, s0=s["s0"], s_last=s["s_last"], **more)
        if op == "att_fwd":
            return {"o": s["o"], "s_last": s["s_last"]}
        ws = _workspace(s, "ws_back", lambda: gs.gs_linear_attention_workspace_size(*sizes, s["q"].dtype, backward=True,
                                                                                    packed=s["offsets"] is not None))
        gs.gs_linear_attention_backward(s["do"], s["q"], s["k"], s["v"], s["g"], s["dq"], s["dk"], s["dv"], ws, s0=s["s0"],
                                        ds_last=s["ds_last"], ds0=s["ds0"], **more)
        return {k: s[k] for k in ("o", "s_last", "dq", "dk", "dv", "ds0")}
    if op == "rotary":
        gs.gs_rotary(s["x"], s["out"], s["freq"], positions=s["positions"], interleaved=c["interleaved"], inverse=c["inverse"])
        return {"out": s["out"]}
    if op == "norm_fwd":
        gs.gs_gated_norm(s["x"], s["weight"], s["y"], s["rstd"], gate=s["gate"], residual=s["residual"], next_weight=s["follow"],
                         z=s["z"], next_rstd=s["rstd2"], groups=c["groups"], activation=c["gate"], scale=s["scale"], eps=EPS)
        return {k: s[k] for k in ("y", "z", "rstd", "rstd2") if s[k] is not None}
    ws = _workspace(s, "ws", lambda: gs.gs_gated_norm_workspace_size(c["rows"], c["cols"], c["groups"]))
    gs.gs_gated_norm_backward(s["dy"], s["x"], s["weight"], s["rstd"], s["dx"], s["dweight"], ws, gate=s["gate"],
                              dgate=s["dgate"], dz=s["dz"], y=s["y"] if c["follow"] else None, next_weight=s["follow"],
                              next_rstd=s["rstd2"], dresidual=s["dresidual"], dnext_weight=s["dfollow"], groups=c["groups"],
                              activation=c["gate"], scale=s["scale"])
    return {k: s[k] for k in ("dx", "dgate", "dresidual", "dweight", "dfollow") if s[k] is not None}


CHUNK = 128


def _tokens(s):
    """(start, length) of each sequence in the flat list of tokens."""
    c, dev = s["case"], s["q"].device
    if s["offsets"] is not None:
        return s["offsets"][:-1].long(), (s["offsets"][1:] - s["offsets"][:-1]).long()
    start = torch.arange(c["B"], device=dev) * c["T"]
    return start, torch.full_like(start, c["T"]) if s["lengths"] is None else s["lengths"].long()


def _order(s, back):
    """Token numbers [B][n * CHUNK] of the sequences, each at the end of its row, forwards or backwards,
    and whether there is one."""
    start, length = _tokens(s)
    c = s["case"]
    longest = c["T"] if c["mask"] != "packed" else min(c["T"], 6 * c["T"] // c["B"] + 2)
    n = -(-longest // CHUNK) * CHUNK
    at = torch.arange(n, device=start.device) - (n - length.unsqueeze(1))
    live = at >= 0
    at = length.unsqueeze(1) - 1 - at if back else at
    return torch.where(live, start.unsqueeze(1) + at, torch.zeros_like(at)), live, length


def _pick(x, at, live, heads):
    """[B][heads][chunks][CHUNK][D] of a [rows][T][heads or fewer][D] tensor, zero where there is no token."""
    x = x.reshape(-1, x.shape[-2], x.shape[-1])[at].float()
    x = x.masked_fill(~live[..., None, None], 0.0).unflatten(1, (-1, CHUNK)).permute(0, 3, 1, 2, 4)
    return x.repeat_interleave(heads // x.shape[1], dim=1)


def _attend(s, q, k, v, first, back, scale):
    """Walking the tokens in turn from the state `first`: S = e^g S + k_t v_t', o_t = scale S' q_t, and the
    last state.  Backwards, from a sequence's end, for gradients: S = S + scale k_t v_t', o_t = S' q_t, S = e^g S."""
    at, live, length = _order(s, back)
    H, g = s["case"]["H"], s["g"].double()
    q, k, v = (_pick(x, at, live, H) for x in (q, k, v))
    i = torch.arange(CHUNK, device=q.device)
    n = q.shape[2]
    power = lambda e: torch.exp(g.view(H, *[1] * e.dim()) * e).float()   # noqa: E731
    near = power((i[:, None] - i[None, :]).clamp(min=0)).masked_fill(i[:, None] < i[None, :], 0.0)
    out = ((q @ k.transpose(-1, -2)) * near.unsqueeze(1)) @ v
    # each chunk's own sum at its end, then the sums before each chunk
    sums = ((k * power(CHUNK - 1 - i)[:, None, :, None]).transpose(-1, -2) @ v)
    a = torch.arange(n + 1, device=q.device)[:, None] - 1 - torch.arange(n, device=q.device)[None, :]
    far = power(a.clamp(min=0) * CHUNK).masked_fill(a < 0, 0.0)
    before = (far @ sums.flatten(-2)).unflatten(-1, sums.shape[-2:])
    out += (q * power(i + 1)[:, None, :, None]) @ before[:, :, :-1]
    # what was there before the first token
    step = 0 if back else 1
    place = (torch.arange(n * CHUNK, device=q.device) - (n * CHUNK - length.unsqueeze(1)) + step).clamp(min=0)
    w = torch.exp(g.view(1, H, 1) * place.unsqueeze(1)).float().view(*q.shape[:-1], 1)
    out = out * scale + (q * w) @ first.unsqueeze(2) * (1.0 if back else scale)
    last = before[:, :, -1] * (torch.exp(g * (1 - step)).float()[:, None, None])
    last = last * scale if back else last
    last += torch.exp(g * length.unsqueeze(1)).float()[..., None, None] * first
    return out.flatten(2, 3).transpose(1, 2), last, at, live


def _place(s, o, at, live, heads, dt):
    """The tokens' rows back in their places, summed over the heads that share one."""
    c = s["case"]
    o = o.unflatten(2, (heads, -1)).sum(3)
    rows = 1 if c["mask"] == "packed" else c["B"]
    out = torch.zeros(rows * c["T"], *o.shape[2:], dtype=dt, device=o.device)
    out[at[live]] = o[live].to(dt)
    return out.view(rows, c["T"], *o.shape[2:])


def _run_plain(s):
    c = s["case"]
    op, dt = c["op"], TYPES[c["dtype"]]
    if op == "att_step":
        H, K = c["H"], c["K"]
        q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
        live = s["slots"] >= 0
        at = s["slots"].clamp(min=0).long()
        old = s["state"][at].unflatten(1, (K, H // K))
        new = torch.exp(s["g"]).view(K, H // K, 1, 1) * old + (k.unsqueeze(-1) * v.unsqueeze(-2)).unsqueeze(2)
        o = (q.unflatten(1, (K, H // K)).unsqueeze(-2) @ new).squeeze(-2).flatten(1, 2) * s["scale"]
        s["o"].copy_(torch.where(live[:, None, None], o, torch.zeros_like(o)))
        s["state"][at[live]] = new.flatten(1, 2)[live]
        return {"o": s["o"], "state": s["state"]}
    if op.startswith("att"):
        o, last, at, live = _attend(s, s["q"], s["k"], s["v"], s["s0"], False, s["scale"])
        out = {"o": _place(s, o, at, live, c["H"], dt), "s_last": last}
        if op == "att_fwd":
            return out
        t = lambda x: x.transpose(-1, -2)   # noqa: E731
        o, _, at, live = _attend(s, s["do"], s["v"], s["k"], t(s["s0"]), False, s["scale"])
        out["dq"] = _place(s, o, at, live, c["H"], dt)
        o, out["ds0"], at, live = _attend(s, s["k"], s["q"], s["do"], s["ds_last"], True, s["scale"])
        out["dv"] = _place(s, o, at, live, c["K"], dt)
        o, _, at, live = _attend(s, s["v"], s["do"], s["q"], t(s["ds_last"]), True, s["scale"])
        out["dk"] = _place(s, o, at, live, c["K"], dt)
        return out
    if op == "rotary":
        R = c["R"]
        angle = s["positions"].double()[..., None, None] * s["freq"]
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        sin = -sin if c["inverse"] else sin
        x = s["x"][..., :R].float()
        a, b = (x[..., ::2], x[..., 1::2]) if c["interleaved"] else (x[..., :R // 2], x[..., R // 2:])
        pair = (a * cos - b * sin, a * sin + b * cos)
        x = torch.stack(pair, dim=-1).flatten(-2) if c["interleaved"] else torch.cat(pair, dim=-1)
        s["out"][..., :R] = x.to(dt)
        if not c["inplace"]:
            s["out"][..., R:] = s["x"][..., R:]
        return {"out": s["out"]}
    groups = c["groups"]
    split = lambda t: t.float().unflatten(-1, (groups, -1))   # noqa: E731
    x, weight = split(s["x"]), split(s["weight"])
    act = slope = 1.0
    if s["gate"] is not None:
        u = split(s["gate"])
        sig = 1 / (1 + torch.exp(-u))
        act, slope = (u * sig, sig * (1 + u * (1 - sig))) if c["gate"] == "silu" else (sig, sig * (1 - sig))
    if op == "norm_fwd":
        rstd = torch.rsqrt(x.square().mean(dim=-1) + EPS)
        y = (s["scale"] * act * (x * rstd.unsqueeze(-1)) * weight).flatten(-2)
        if s["residual"] is not None:
            y = s["residual"].float() + y
        out = {"y": y.to(dt), "rstd": rstd}
        if s["follow"] is not None:
            out["rstd2"] = torch.rsqrt(y.square().mean(dim=-1) + EPS)
            out["z"] = (y * out["rstd2"].unsqueeze(-1) * s["follow"]).to(dt)
        return out
    d, out = s["dy"].float(), {}
    if s["follow"] is not None:
        r2 = s["rstd2"].unsqueeze(-1)
        n, u = s["y"].float() * r2, s["dz"].float() * s["follow"]
        d = d + r2 * (u - n * (u * n).mean(dim=-1, keepdim=True))
        out["dfollow"] = (s["dz"].float() * n).sum(dim=0)
        if s["dresidual"] is not None:
            out["dresidual"] = d.to(dt)
    rstd = s["rstd"].unsqueeze(-1)
    d, n = split(d) * s["scale"], x * rstd
    if s["gate"] is not None:
        out["dgate"] = (d * n * weight * slope).flatten(-2).to(dt)
    out["dweight"] = (d * act * n).sum(dim=0).flatten()
    dn = d * act * weight
    out["dx"] = (rstd * (dn - n * (dn * n).mean(dim=-1, keepdim=True))).flatten(-2).to(dt)
    return out


# ---- the definition in 64 bits ----------------------------------------------------------------

def _exact_attention(case, s, f64):
    B, H, K, dk, dv = (case[k] for k in ("B", "H", "K", "dk", "dv"))
    dev, group = s["q"].device, H // K
    decay = torch.exp(s["g"].to(f64)).view(1, H, 1, 1)
    if case["op"] == "att_step":
        state, o = s["state"].to(f64), torch.zeros(B, H, dv, dtype=f64, device=dev)
        slots = s["slots"].tolist()
        for b in range(B):
            if slots[b] >= 0:
                kb, vb = (s[n][b].to(f64).repeat_interleave(group, 0) for n in ("k", "v"))
                state[slots[b]] = decay[0] * state[slots[b]] + torch.einsum("hd,he->hde", kb, vb)
                o[b] = s["scale"] * torch.einsum("hd,hde->he", s["q"][b].to(f64), state[slots[b]])
        return {"o": o, "state": state}
    rows, T = s["q"].shape[:2]
    if s["offsets"] is not None:
        cuts = s["offsets"].tolist()
        spans = [(0, cuts[b], cuts[b + 1]) for b in range(B)]
    else:
        n = [T] * B if s["lengths"] is None else s["lengths"].tolist()
        spans = [(b, 0, n[b]) for b in range(B)]
    most = max(e - a for _, a, e in spans)
    index = torch.zeros(B, max(most, 1), dtype=torch.long)
    alive = torch.zeros(B, max(most, 1), dtype=torch.bool)
    for b, (r, a, e) in enumerate(spans):
        index[b, :e - a] = torch.arange(r * T + a, r * T + e)
        alive[b, :e - a] = True
    index, alive = index.to(dev), alive.to(dev)

    def rows_of(name):      # [tokens][B][H][D], zero past a sequence's end
        x = s[name].reshape(rows * T, -1, s[name].shape[-1])[index].to(f64) * alive[..., None, None]
        return x.repeat_interleave(H // x.shape[2], dim=2).transpose(0, 1).contiguous()

    def back_in_place(x, heads):
        x = x.transpose(0, 1).unflatten(2, (heads, -1)).sum(3)
        out = torch.zeros(rows * T, heads, x.shape[-1], dtype=f64, device=dev)
        out[index[alive]] = x[alive]
        return out.view(rows, T, heads, -1)

    q, k, v = rows_of("q") * s["scale"], rows_of("k"), rows_of("v")
    mul = torch.where(alive.t()[..., None, None, None], decay.unsqueeze(0), torch.ones_like(decay))
    train = case["op"] == "att_train"
    do = rows_of("do") if train else None
    S, o = s["s0"].to(f64), torch.empty_like(v)
    dq = torch.empty_like(q)
    for t in range(most):
        S = torch.addcmul(mul[t] * S, k[t].unsqueeze(-1), v[t].unsqueeze(-2))
        o[t] = (q[t].unsqueeze(-2) @ S).squeeze(-2)
        if train:
            dq[t] = (S @ do[t].unsqueeze(-1)).squeeze(-1) * s["scale"]
    out = {"o": back_in_place(o, H), "s_last": S}
    if train:
        D, dkt, dvt = s["ds_last"].to(f64), torch.empty_like(k), torch.empty_like(v)
        for t in range(most - 1, -1, -1):
            D = torch.addcmul(D, q[t].unsqueeze(-1), do[t].unsqueeze(-2))
            dkt[t] = (D @ v[t].unsqueeze(-1)).squeeze(-1)
            dvt[t] = (k[t].unsqueeze(-2) @ D).squeeze(-2)
            D = mul[t] * D
        out.update(dq=back_in_place(dq, H), dk=back_in_place(dkt, K), dv=back_in_place(dvt, K), ds0=D)
    return out


def exact(case, seed):
    s, f64 = prepare(case, seed), torch.float64
    if case["op"].startswith("att"):
        B, T, state = case["B"], case["T"], case["H"] * case["dk"] * case["dv"]
        longest = 1 if case["op"] == "att_step" else min(T, 6 * T // B + 2) if case["mask"] == "packed" else T
        most = (3 if case["op"] == "att_train" else 1) * longest * (4e-5 + B * state * 1e-11)
        return None if most > 12 else _exact_attention(case, s, f64)
    if case["op"] == "rotary":
        R, D = case["R"], case["D"]
        first = (lambda j: 2 * j) if case["interleaved"] else (lambda j: j)
        other = (lambda j: 2 * j + 1) if case["interleaved"] else (lambda j: j + R // 2)
        out = s["x"].to(f64).clone(memory_format=torch.contiguous_format)
        sign = -1.0 if case["inverse"] else 1.0
        for j in range(R // 2):
            turn = sign * s["positions"].to(f64) * s["freq"][j]
            c, n = torch.cos(turn)[..., None], torch.sin(turn)[..., None]
            a, b = s["x"][..., first(j)].to(f64), s["x"][..., other(j)].to(f64)
            out[..., first(j)], out[..., other(j)] = c * a - n * b, c * b + n * a
        return {"out": out}
    groups = case["groups"]
    kind = {"silu": lambda u: u * torch.sigmoid(u), "sigmoid": torch.sigmoid, "none": lambda u: 1.0}[case["gate"]]
    leaves = {k: s[k].detach().to(f64) for k in ("x", "gate", "weight") if s[k] is not None}
    rows, cols = s["x"].shape
    back = case["op"] == "norm_bwd"
    if back:
        for t in leaves.values():
            t.requires_grad_()
    x = leaves["x"].view(rows, groups, -1)
    if back:   # the stored 1 / sqrt(mean of squares + eps) stands for the value and moves as it does
        r = s["rstd"].to(f64).unsqueeze(-1)
        r = r - (r ** 3) * ((x * x).mean(dim=2, keepdim=True) - (x.detach() ** 2).mean(dim=2, keepdim=True)) / 2
    else:
        r = 1 / torch.sqrt((x * x).mean(dim=2, keepdim=True) + EPS)
    branch = s["scale"] * kind(leaves.get("gate")) * ((x * r).view(rows, cols) * leaves["weight"])
    if not back:
        y = branch if s["residual"] is None else branch + s["residual"].to(f64)
        out = {"y": y, "rstd": r.squeeze(-1)}
        if case["follow"]:
            r2 = 1 / torch.sqrt((y * y).sum(dim=1) / cols + EPS)
            out.update(z=y * r2[:, None] * s["follow"].to(f64), rstd2=r2)
        return out
    d, out = s["dy"].to(f64), {}
    if case["follow"]:
        y, dz, k = s["y"].to(f64), s["dz"].to(f64), s["rstd2"].to(f64)[:, None]
        out["dfollow"] = (dz * y * k).sum(dim=0)
        dz = dz * s["follow"].to(f64)
        d = d + k * dz - y * k ** 3 * (dz * y).sum(dim=1, keepdim=True) / cols
        if s["dresidual"] is not None:
            out["dresidual"] = d.clone()
    grads = torch.autograd.grad(branch, list(leaves.values()), d)
    out.update({"d" + k: g for k, g in zip(leaves, grads)})
    return out
