"""The calls around attention in a transformer block whose speed is measured, and its gradients.

Operators, each through its public entry point:
  rope      queries and keys of every head, root-mean-square normalised (where there are weights) and rotated by
            their token's positions on three axes (time, height, width), in one pass
  rope_bwd  its gradients: of queries, keys and the norms' weights
  attn_bwd  the gradients of packed attention (each session's queries over its own keys), from its result and
            log-sum-exp; the probabilities are computed again
Tokens are packed, bfloat16 [tokens, heads, width]. Sizes are latent grids of streaming video models: 30 x 52 =
1560 tokens a frame, chunks of one or three frames against up to 21 cached ones, whole clips of 21 frames, single
tokens of an autoregressive head; 2 to 40 heads of width 64 or 128. Lengths that are no multiple of anything stand
for cropped clips. Queries and keys that come out of one projection lie beside the values in rows of one tensor.
"""
import math

import torch

own = False

GRID = (30, 52)  # a frame's latent tokens
EPS = 1e-6


def listed():
    return [
        # one token each of four sessions that have streamed for long, grouped heads: launches and latency are all it is
        {"name": "rope_token", "op": "rope", "T": 4, "Hq": 40, "Hk": 8, "d": 128, "norm": True, "pairs": True, "fused": False, "far": 4000000},
        # one frame of the small model, in rows of the fused projection
        {"name": "rope_frame", "op": "rope", "T": 1560, "Hq": 12, "Hk": 12, "d": 128, "norm": True, "pairs": True, "fused": True, "far": 1000},
        # an odd crop at head width 64, rotation by halves of a head and no norm
        {"name": "rope_odd", "op": "rope", "T": 20011, "Hq": 24, "Hk": 24, "d": 64, "norm": False, "pairs": False, "fused": False, "far": 100},
        # a coalesced batch of five chunks of three frames, the large model: as fast as memory takes it
        {"name": "rope_chunk", "op": "rope", "T": 23400, "Hq": 40, "Hk": 40, "d": 128, "norm": True, "pairs": True, "fused": True, "far": 1000},
        # training on an odd crop at head width 64, grouped heads
        {"name": "rope_bwd_odd", "op": "rope_bwd", "T": 2731, "Hq": 24, "Hk": 12, "d": 64, "norm": True, "pairs": False, "fused": False, "far": 100},
        # training on a clip of 21 frames, the large model
        {"name": "rope_bwd_clip", "op": "rope_bwd", "T": 32760, "Hq": 40, "Hk": 40, "d": 128, "norm": True, "pairs": True, "fused": True, "far": 0},
        # the smallest training step: one short clip, two heads
        {"name": "attn_bwd_tiny", "op": "attn_bwd", "lq": "1024", "lk": "1024", "H": 2, "d": 64},
        # cropped clips of odd sizes at head width 64, one of them without keys and one without queries
        {"name": "attn_bwd_odd", "op": "attn_bwd", "lq": "777,1,0,131,2047,64", "lk": "777,333,100,0,2500,1", "H": 12, "d": 64},
        # training a streaming model: one frame against 21, the small model
        {"name": "attn_bwd_frame", "op": "attn_bwd", "lq": "1560", "lk": "32760", "H": 12, "d": 128},
        # clips of four sessions of unequal length in one call
        {"name": "attn_bwd_batch", "op": "attn_bwd", "lq": "8190,8190,16380,2730", "lk": "8190,8190,16380,2730", "H": 12, "d": 128},
        # head width 64
        {"name": "attn_bwd_clip64", "op": "attn_bwd", "lq": "16380", "lk": "16380", "H": 24, "d": 64},
        # a whole clip of 21 frames, the small model: the largest, bound by the matrix cores
        {"name": "attn_bwd_clip", "op": "attn_bwd", "lq": "32760", "lk": "32760", "H": 12, "d": 128},
    ]


_MOST_FLOPS = 10.0 * 32760 * 32760 * 12 * 128
_MOST_SCORES = 12.9e9  # of the padded batch that the plain form holds
_MOST_BYTES = 2.1e9


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _ints(text):
    return [int(x) for x in text.split(",")]


def _text(values):
    return ",".join(str(x) for x in values)


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        if case["op"] == "attn_bwd":
            lq, lk = _ints(case["lq"]), _ints(case["lk"])
            # (one key a query has no gradient but rounding)
            if sum(a * b for a, b in zip(lq, lk) if b > 1) < 64 or len(lq) * max(lq) * max(lk) * case["H"] > _MOST_SCORES:
                continue
        if w["flops"] <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES:
            return case


def _draw(rng):
    op = rng.choice(["rope", "rope_bwd", "attn_bwd", "attn_bwd"])
    d = rng.choice([64, 128, 128])
    if op != "attn_bwd":
        Hq, Hk = rng.choice([(2, 2), (4, 4), (12, 12), (24, 24), (40, 40), (40, 8), (24, 12), (16, 4), (7, 1)])
        return {"op": op, "T": _log(rng, 1 if op == "rope" else 100, 32760), "Hq": Hq, "Hk": Hk, "d": d, "norm": op == "rope_bwd" or rng.random() < 0.7,
                "pairs": rng.random() < 0.5, "fused": rng.random() < 0.5, "far": rng.choice([0, 100, 1000, 4000000])}
    H = rng.choice([2, 4, 12, 12, 24, 40])
    n = _log(rng, 1, 12)
    frame = rng.choice([256, 1560, _log(rng, 30, 1560)])
    lq = [frame * rng.choice([1, 1, 3]) + rng.choice([0, 0, rng.randrange(64)]) for _ in range(n)]
    if rng.random() < 0.5:  # clips that attend to themselves
        top = _log(rng, 30, 32760)
        lq = [rng.choice([top, rng.randrange(top + 1)]) for _ in range(n - 1)] + [top]
        lk = lq
    else:  # chunks against a cache
        lk = [a + frame * _log(rng, 1, 20) for a in lq]
    return {"op": op, "lq": _text(lq), "lk": _text(lk), "H": H, "d": d}


def work(case):
    d = case["d"]
    if case["op"] == "attn_bwd":  # q, o, do and dq; k, v, dk and dv; the log-sum-exp
        lq, lk, H = _ints(case["lq"]), _ints(case["lk"]), case["H"]
        return {"bytes": 8 * (sum(lq) + sum(lk)) * H * d + 4 * sum(lq) * H, "flops": 10 * sum(a * b for a, b in zip(lq, lk)) * H * d}
    heads = case["T"] * (case["Hq"] + case["Hk"])
    if case["op"] == "rope":
        return {"bytes": 4 * heads * d + 12 * case["T"], "flops": 0}
    return {"bytes": (6 if case["norm"] else 4) * heads * d + 12 * case["T"], "flops": 0}


# ---- inputs


def _offsets(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32, device="cuda")


def _axes(d):
    """How many of a head's d / 2 rotated pairs go by time, height and width."""
    n = d // 6
    return d // 2 - 2 * n, n, n


def prepare(case, seed):
    """Positions are a latent grid's, from a frame on that the stream has come to. Queries and keys carry an offset per
    head and channel, as the channel outliers of a trained model's keys."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    d = case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    if case["op"] == "attn_bwd":
        lq, lk, H = _ints(case["lq"]), _ints(case["lk"]), case["H"]
        state = {"case": case, "cu_q": _offsets(lq), "cu_k": _offsets(lk), "max_q": max(lq), "max_k": max(lk), "scale": 1.0 / math.sqrt(d)}
        state["q"], state["v"], state["do"] = (normal(n, H, d).bfloat16() for n in (sum(lq), sum(lk), sum(lq)))
        state["k"] = (normal(sum(lk), H, d) + normal(H, d)).bfloat16()
        state["o"], state["lse"] = _forward(state)
        return state
    T, Hq, Hk = case["T"], case["Hq"], case["Hk"]
    at = torch.arange(T, device="cuda") + torch.randint(0, GRID[0] * GRID[1], (1,), generator=g, device="cuda")
    frame = torch.randint(0, case["far"] + 1, (1,), generator=g, device="cuda") + at // (GRID[0] * GRID[1])
    state = {"case": case, "pos": torch.stack([frame, at // GRID[1] % GRID[0], at % GRID[1]], 1).int(),
             "freq": torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n) for n in _axes(d)])}
    offset = normal(1, Hq + 2 * Hk, d)
    if case["fused"]:  # rows of queries, keys and values
        rows = (normal(T, Hq + 2 * Hk, d) + offset).bfloat16()
        state["q"], state["k"] = rows[:, :Hq], rows[:, Hq:Hq + Hk]
    else:
        state["q"], state["k"] = (normal(T, Hq, d) + offset[:, :Hq]).bfloat16(), (normal(T, Hk, d) + offset[:, Hq:Hq + Hk]).bfloat16()
    state["q_weight"], state["k_weight"] = (1 + 0.2 * normal(d) if case["norm"] else None for _ in range(2))
    if case["op"] == "rope_bwd":
        state["dq"], state["dk"] = normal(T, Hq, d).bfloat16(), normal(T, Hk, d).bfloat16()
    return state


# ---- the operators


def run(state):
    if own:
        return _own(state)
    return {"rope": _rope, "rope_bwd": _rope_bwd, "attn_bwd": _attn_bwd}[state["case"]["op"]](state)


def _own(state):
    import paper_2606_19271_amd as ts

    case, s = state["case"], state
    if case["op"] == "attn_bwd":
        return list(ts.ts_attn_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["cu_q"], s["cu_k"], s["max_q"], s["max_k"]))
    rope = ts.Rope(s["freq"], _axes(case["d"]), case["pairs"])
    if case["op"] == "rope":
        return list(ts.ts_qk_rope(s["q"], s["k"], s["pos"], rope, s["q_weight"], s["k_weight"], eps=EPS))
    return list(ts.ts_qk_rope_bwd(s["dq"], s["dk"], s["q"], s["k"], s["pos"], rope, s["q_weight"], s["k_weight"], eps=EPS))


def _angles(state):
    """cos and sin [T, 1, d / 2] of each pair's angle, its axis' position times its frequency."""
    axis = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(_axes(state["case"]["d"]), device="cuda"))
    angle = state["pos"][:, axis].double() * state["freq"]
    return angle.cos().float()[:, None], angle.sin().float()[:, None]


def _split(state, x):
    """The two members of every pair: neighbouring channels, or the two halves of a head."""
    return (x[..., 0::2], x[..., 1::2]) if state["case"]["pairs"] else x.chunk(2, -1)


def _join(state, a, b):
    return torch.stack([a, b], -1).flatten(-2) if state["case"]["pairs"] else torch.cat([a, b], -1)


def _rope_one(state, x, weight, cos, sin):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight
    a, b = _split(state, x)
    return _join(state, a * cos - b * sin, a * sin + b * cos).bfloat16()


def _rope(state):
    cos, sin = _angles(state)
    return [_rope_one(state, state["q"], state["q_weight"], cos, sin), _rope_one(state, state["k"], state["k_weight"], cos, sin)]


def _rope_bwd_one(state, dy, x, weight, cos, sin):
    a, b = _split(state, dy.float())
    dy = _join(state, a * cos + b * sin, b * cos - a * sin)
    if weight is None:
        return dy.bfloat16(), None
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    x, g = x * r, dy * weight
    dx = r * (g - x * (g * x).mean(-1, keepdim=True))
    return dx.bfloat16(), (dy * x).sum((0, 1), dtype=torch.float64).float()


def _rope_bwd(state):
    cos, sin = _angles(state)
    dq, dqw = _rope_bwd_one(state, state["dq"], state["q"], state["q_weight"], cos, sin)
    dk, dkw = _rope_bwd_one(state, state["dk"], state["k"], state["k_weight"], cos, sin)
    return [dq, dk, dqw, dkw]


def _places(cu, total):
    """Where each row lies in the padded batch: its session and its place there."""
    t = torch.arange(total, device="cuda")
    s = torch.searchsorted(cu.long(), t, right=True) - 1
    return s, t - cu.long()[s]


def _padded(x, cu, most, at):
    """[tokens, H, ...] to [nseq, H, most, ...], zeros past each session's end."""
    out = torch.zeros(cu.numel() - 1, most, *x.shape[1:], device="cuda")
    out[at] = x.float()
    return out.transpose(1, 2).contiguous()


def _weights(state, lse):
    """exp(scale q k - lse) [nseq, H, rows, keys], or without an lse the scores; past a session's last key 0, or -inf."""
    at_q, at_k = (_places(state["cu_" + c], state[c].shape[0]) for c in "qk")
    q, k = _padded(state["q"], state["cu_q"], state["max_q"], at_q), _padded(state["k"], state["cu_k"], state["max_k"], at_k)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(state["scale"])
    len_k = (state["cu_k"][1:] - state["cu_k"][:-1]).long()
    if state["cu_k"].numel() > 2:
        x.masked_fill_((torch.arange(state["max_k"], device="cuda") >= len_k[:, None])[:, None, None], -math.inf)
    if lse is not None:
        x = x.sub_(_padded(lse, state["cu_q"], state["max_q"], at_q)[..., None]).exp_()
        x = x.masked_fill_((len_k == 0)[:, None, None, None], 0) if state["cu_k"].numel() > 2 else x
    return x, q, k, at_q, at_k


def _forward(state):
    """The result of attention and its log-sum-exp, as the backward pass is given them."""
    x, _, _, at_q, at_k = _weights(state, None)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(top == -math.inf, 0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    v = _padded(state["v"], state["cu_k"], state["max_k"], at_k)
    o = torch.matmul(x, v) / torch.where(total > 0, total, 1)
    return o.transpose(1, 2)[at_q].bfloat16(), (top + total.log()).squeeze(-1).transpose(1, 2)[at_q].contiguous()


def _attn_bwd(state):
    x, q, k, at_q, at_k = _weights(state, state["lse"])
    do, o = (_padded(state[c], state["cu_q"], state["max_q"], at_q) for c in ("do", "o"))
    v = _padded(state["v"], state["cu_k"], state["max_k"], at_k)
    dv = torch.matmul(x.transpose(2, 3), do)
    x = x.mul_(torch.matmul(do, v.transpose(2, 3)).sub_((do * o).sum(-1, keepdim=True)))
    dq, dk = torch.matmul(x, k).mul_(state["scale"]), torch.matmul(x.transpose(2, 3), q).mul_(state["scale"])
    return [g.transpose(1, 2)[at].bfloat16() for g, at in ((dq, at_q), (dk, at_k), (dv, at_k))]


# ---- the definition in 64 bits


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "attn_bwd":
        return _exact_attn(state)
    T, d = case["T"], case["d"]
    n = torch.tensor(_axes(d), device="cuda").cumsum(0)
    pos = state["pos"].double()
    angle = torch.empty(T, d // 2, dtype=torch.float64, device="cuda")
    for axis, (lo, hi) in enumerate(((0, n[0]), (n[0], n[1]), (n[1], n[2]))):
        angle[:, lo:hi] = torch.outer(pos[:, axis], state["freq"][lo:hi])
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def forward(x, weight):
        if weight is not None:
            x = x * weight / torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS)
        z = torch.view_as_complex(x.unflatten(-1, (d // 2, 2) if case["pairs"] else (2, d // 2)).movedim(-1 if case["pairs"] else -2, -1).contiguous())
        y = torch.view_as_real(z * turn)
        return (y if case["pairs"] else y.transpose(-1, -2)).flatten(-2)

    got = []
    for c in "qk":
        x, w = state[c].double(), None if state[c + "_weight"] is None else state[c + "_weight"].double()
        if case["op"] == "rope":
            got.append(forward(x, w))
            continue
        x.requires_grad_()
        leaves = [x] if w is None else [x, w.requires_grad_()]
        got.append(list(torch.autograd.grad(forward(x, w), leaves, state["d" + c].double())) + [None] * (2 - len(leaves)))
    return got if case["op"] == "rope" else [got[0][0], got[1][0], got[0][1], got[1][1]]


def _exact_attn(state):
    lq, lk, scale = _ints(state["case"]["lq"]), _ints(state["case"]["lk"]), state["scale"]
    dq, dk, dv = (torch.zeros(state[c].shape, dtype=torch.float64, device="cuda") for c in "qkv")
    a = b = 0
    for m, n in zip(lq, lk):
        for h in range(state["case"]["H"] if m and n else 0):
            q, o, do = (state[c][a:a + m, h].double() for c in ("q", "o", "do"))
            k, v = (state[c][b:b + n, h].double() for c in "kv")
            p = torch.exp(scale * (q @ k.T) - state["lse"][a:a + m, h, None].double())
            dv[b:b + n, h] = p.T @ do
            p = p * (do @ v.T - (do * o).sum(1, keepdim=True))
            dq[a:a + m, h], dk[b:b + n, h] = p @ k * scale, p.T @ q * scale
        a, b = a + m, b + n
    return [dq, dk, dv]
