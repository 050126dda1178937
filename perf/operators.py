"""The calls of the 8-bit session cache whose speed is measured.

A session's keys and values live in pages of 64 tokens: e4m3 bytes k, v [P, H, 64, d], one power-of-two
scale per page and head (k_exp, v_exp [P, H], the exponent biased by 127), and per token and head the
attention weight it has collected (weight [P, H, 64]). Sessions find their pages in table [nseq, width].

Operators, each through its public entry point:
  append  a chunk's (or a token's) keys and values, bfloat16, into the sessions' pages
  attn    new queries against the cached keys and values
  weigh   the weight that these queries gave to each cached token, added to what it had
  evict   per head, the tokens of most weight (and the first and the newest) into new pages
Sizes are latent grids of streaming video models: 16 x 16 = 256 tokens a frame, 30 x 52 = 1560, chunks of
one or three frames against up to 21 cached ones, single tokens of an autoregressive head; 4 to 40 heads of
width 64 or 128, alone or in groups that share a cached head. Lengths that are no multiple of anything
stand for cropped clips.
"""
import math

import torch

own = False

PAGE = 64


def listed():
    return [
        # one token each of four young sessions, the small model: launches and latency are all it is
        {"name": "attn_token", "op": "attn", "lq": "1,1,1,1", "lk": "1000,1,333,2047", "H": 12, "G": 1, "d": 128, "lse": False},
        # one token each of 32 long sessions, five query heads to a cached head: bound by reading the cache
        {"name": "attn_tokens", "op": "attn", "lq": ",".join(["1"] * 32),
         "lk": ",".join(str(32760 - 857 * i) for i in range(32)), "H": 8, "G": 5, "d": 128, "lse": False},
        # one session's frame against 21 frames, the small model: fewer query tiles than compute units
        {"name": "attn_frame", "op": "attn", "lq": "1560", "lk": "32760", "H": 12, "G": 1, "d": 128, "lse": True},
        # the frames of six sessions of unequal length in one call
        {"name": "attn_batch", "op": "attn", "lq": "1560,1560,1560,1560,1560,1560", "lk": "8190,8190,16380,32760,32760,2730",
         "H": 12, "G": 1, "d": 128, "lse": False},
        # three frames against 21, the large model: the largest call, bound by the matrix cores
        {"name": "attn_chunk", "op": "attn", "lq": "4680", "lk": "32760", "H": 40, "G": 1, "d": 128, "lse": False},
        # cropped chunks of odd sizes at head width 64, with their log-sum-exp
        {"name": "attn_odd", "op": "attn", "lq": "257,31,100,640", "lk": "777,4097,129,20011", "H": 12, "G": 2, "d": 64, "lse": True},
        # one token each of eight sessions into the middle of a page
        {"name": "append_token", "op": "append", "lq": "1,1,1,1,1,1,1,1", "lk": "5,77,1000,129,2047,333,700,64", "H": 12, "G": 1, "d": 128},
        # three frames of five sessions, the large model: as fast as memory takes them
        {"name": "append_chunk", "op": "append", "lq": "4680,4680,4680,4680,4680", "lk": "0,1560,4680,100,3121", "H": 40, "G": 1, "d": 128},
        # small odd chunks at head width 64, grouped heads
        {"name": "weigh_odd", "op": "weigh", "lq": "100,37,256", "lk": "513,1200,64", "H": 4, "G": 2, "d": 64},
        # one session's frame against 21 frames, the small model
        {"name": "weigh_frame", "op": "weigh", "lq": "1560", "lk": "32760", "H": 12, "G": 1, "d": 128},
        # three short sessions, odd lengths, one of them shorter than what is kept
        {"name": "evict_odd", "op": "evict", "lq": "0,0,0", "lk": "1000,411,2304", "H": 4, "G": 1, "d": 64, "keep": 513, "first": 64, "last": 100},
        # five sessions of 21 frames cut down to half, the large model; the first and the newest frames stay
        {"name": "evict_half", "op": "evict", "lq": "0,0,0,0,0", "lk": "32760,32760,32760,32760,32760", "H": 40, "G": 1, "d": 128,
         "keep": 16380, "first": 1560, "last": 4680},
    ]


_MOST_FLOPS = 4.0 * 4680 * 32760 * 40 * 128
_MOST_BYTES = 1.74e9
_MOST_SCORES = 4680 * 32760 * 40  # of the padded batch that the plain form holds


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
        lq, lk = _ints(case["lq"]), _ints(case["lk"])
        scores = len(lq) * max(lq) * max(lk) * case["H"] * case["G"] if case["op"] in ("attn", "weigh") else 0
        padded = len(lk) * max(lk) * case["H"] * case["d"]
        if w["flops"] <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES and scores <= _MOST_SCORES and padded <= 1.1e9:
            return case


def _draw(rng):
    op = rng.choice(["attn", "attn", "attn", "append", "weigh", "evict"])
    d = rng.choice([64, 128, 128])
    H, G = rng.choice([(4, 1), (12, 1), (24, 1), (40, 1), (8, 5), (12, 2), (4, 4)])
    n = _log(rng, 1, 12)
    if op == "attn" and rng.random() < 0.4:  # single tokens
        n = _log(rng, 1, 32)
        return {"op": op, "lq": _text([1] * n), "lk": _text(_log(rng, 1, 32760) for _ in range(n)), "H": H, "G": G, "d": d,
                "lse": rng.random() < 0.5}
    if op in ("attn", "weigh"):
        frame = rng.choice([256, 1560, _log(rng, 30, 1560)])
        lq = [frame * rng.choice([1, 1, 3]) for _ in range(n)]
        lk = [a + frame * _log(rng, 1, 20) + rng.choice([0, 0, rng.randrange(64)]) for a in lq]
        case = {"op": op, "lq": _text(lq), "lk": _text(lk), "H": H, "G": G, "d": d}
        return {**case, "lse": rng.random() < 0.5} if op == "attn" else case
    if op == "append":
        top = _log(rng, 1, 4680)
        return {"op": op, "lq": _text(rng.choice([top, rng.randrange(top + 1)]) for _ in range(n - 1)) + ("," if n > 1 else "") + str(top),
                "lk": _text(_log(rng, 1, 8190) - 1 for _ in range(n)), "H": H, "G": 1, "d": d}
    lk = [_log(rng, 200, 32760) for _ in range(n)]
    keep = rng.randrange(64, max(65, max(lk)))
    return {"op": op, "lq": _text([0] * n), "lk": _text(lk), "H": H, "G": 1, "d": d, "keep": keep,
            "first": rng.randrange(keep // 4 + 1), "last": rng.randrange(keep // 4 + 1)}


def work(case):
    lq, lk, H, d = _ints(case["lq"]), _ints(case["lk"]), case["H"], case["d"]
    Hq = H * case["G"]
    pairs = sum(a * b for a, b in zip(lq, lk))
    if case["op"] == "attn":  # queries and results in 16 bits, keys and values in 8
        return {"bytes": 4 * sum(lq) * Hq * d + 2 * sum(lk) * H * d + (4 * sum(lq) * Hq if case["lse"] else 0),
                "flops": 4 * pairs * Hq * d}
    if case["op"] == "append":  # 16 bits in, 8 out, the new tokens' weights cleared
        return {"bytes": sum(lq) * H * (2 * d * 3 + 4), "flops": 0}
    if case["op"] == "weigh":  # queries and their lse, keys, the weights before and after
        return {"bytes": sum(lq) * Hq * (2 * d + 4) + sum(lk) * H * (d + 8), "flops": 2 * pairs * Hq * d}
    kept = sum(min(b, case["keep"]) for b in lk)  # weights, the kept rows in and out, their weights and positions
    return {"bytes": 4 * sum(lk) * H + kept * H * (4 * d + 8), "flops": 0}


# ---- inputs


def _scale_exp(amax):
    """The least n >= -100 with amax <= 448 * 2^n, plus 127 (amax = m * 2^x, 448 = 0.875 * 2^9)."""
    m, x = torch.frexp(amax)
    n = x - 9 + (m > 0.875).to(x.dtype)
    return torch.where(amax > 0, n, -100).clamp(min=-100) + 127


def _power(exp):
    """2^(exp - 127), exactly: exp2 and ldexp are a last bit off on some devices."""
    return (exp.to(torch.int32) << 23).view(torch.float32)


def _e4m3(x, exp):
    return (x * _power(254 - exp.to(torch.int32))).to(torch.float8_e4m3fn)


def _numbers(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return _numbers(cu)


def prepare(case, seed):
    """The sessions' pages lie anywhere in the pool: those that the call only reads in its first part, those
    that it writes in its last one. Keys carry an offset per head and channel, as the channel outliers of a
    trained model's keys; weights are uneven, and those of the newest tokens still zero."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    lq, lk, H, G, d, op = _ints(case["lq"]), _ints(case["lk"]), case["H"], case["G"], case["d"], case["op"]
    n = len(lq)
    total = [b + (a if op == "append" else 0) for a, b in zip(lq, lk)]
    pages = [-(-t // PAGE) for t in total]
    width = max(1, max(pages))
    written = [p - b // PAGE if op == "append" and a else 0 for a, b, p in zip(lq, lk, pages)]
    keep_pages = -(-case["keep"] // PAGE) if op == "evict" else 0
    read = sum(pages) - sum(written)
    new = sum(written) + n * keep_pages
    order = torch.cat([torch.randperm(read, generator=g, device="cuda"), read + torch.randperm(new, generator=g, device="cuda")]).tolist()
    at, table, a0, b0 = 0, [], 0, read
    for p, w in zip(pages, written):
        row = order[a0:a0 + p - w] + order[b0:b0 + w]
        a0, b0 = a0 + p - w, b0 + w
        table.append(row + [-1] * (width - p))
    pool = read + new + 1  # the last page belongs to nobody
    new_table = [order[b0 + i * keep_pages:b0 + (i + 1) * keep_pages] for i in range(n)]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    offset = normal(H, 1, d) * math.sqrt(2.0)
    state = {"case": case, "read": read, "table": _numbers(table), "lens": _numbers(lk), "cu": _offsets(lq), "max_q": max(lq),
             "max_k": max(lk), "scale": 1.0 / math.sqrt(d)}
    for name, x in (("k", normal(pool, H, PAGE, d) + offset), ("v", normal(pool, H, PAGE, d))):
        exp = _scale_exp(x.abs().amax((2, 3)))
        state[name], state[name + "_exp"] = _e4m3(x, exp[:, :, None, None]), exp.to(torch.uint8)
    state["weight"] = normal(pool, H, PAGE).square() * torch.exp(2 * normal(pool, H, PAGE))
    if op == "append":
        state["new_k"], state["new_v"] = (normal(sum(lq), H, d) * 2 + offset[:, 0]).bfloat16(), normal(sum(lq), H, d).bfloat16()
    if op in ("attn", "weigh"):
        state["q"] = normal(sum(lq), H * G, d).bfloat16()
    if op == "weigh":
        state["lse"] = torch.empty(sum(lq), H * G, device="cuda")
        state["after"] = state["weight"].clone()
        for s, (a, b) in enumerate(zip(lq, lk)):
            t = sum(lq[:s])
            k, _ = _tokens(state, "k", s, b, torch.float32)
            for h in range(H):
                q = state["q"][t:t + a, h * G:(h + 1) * G].float()
                state["lse"][t:t + a, h * G:(h + 1) * G] = torch.logsumexp(q @ k[h].T * state["scale"], -1)
    if op == "evict":
        state["new_table"] = _numbers(new_table)
        for row, b in zip(table, lk):
            newest = b - b // 16
            for j in range(newest // PAGE, -(-b // PAGE)):
                state["weight"][row[j], :, max(0, newest - j * PAGE):] = 0
    if op == "attn":
        del state["weight"]
        state["weight"] = torch.zeros(pool, H, PAGE, device="cuda")
    return state


def _tokens(state, name, s, length, dtype):
    """Session s's cached keys or values [H, length, d] and, beside them, where each token lies."""
    at = torch.arange(length, device="cuda")
    page = state["table"][s].long()[at // PAGE]
    x = state[name][page, :, at % PAGE].to(dtype)
    scale = _power(state[name + "_exp"][page]).to(dtype)
    return (x * scale[:, :, None]).transpose(0, 1).contiguous(), (page, at % PAGE)


# ---- the operators


def run(state):
    if own:
        return _own(state)
    return {"attn": _attn, "append": _append, "weigh": _weigh, "evict": _evict}[state["case"]["op"]](state)


def _own(state):
    import paper_2606_19271_amd as ts

    case = state["case"]
    cache = ts.SessionCache(state["k"], state["v"], state["k_exp"], state["v_exp"], state["weight"])
    if case["op"] == "attn":
        r = ts.ts_cache_attn(state["q"], cache, state["cu"], state["max_q"], state["table"], state["lens"], state["max_k"],
                             return_lse=case["lse"])
        return list(r) if case["lse"] else [r]
    if case["op"] == "append":
        lens = ts.ts_cache_append(cache, state["new_k"], state["new_v"], state["cu"], state["max_q"], state["table"], state["lens"])
        n = state["read"]
        return [lens, cache.k[n:], cache.v[n:], cache.k_exp[n:], cache.v_exp[n:], cache.weight[n:]]
    if case["op"] == "weigh":
        return [ts.ts_cache_weigh(state["q"], state["lse"], cache, state["cu"], state["max_q"], state["table"], state["lens"],
                                  state["max_k"], out=state["after"])]
    lens, kept = ts.ts_cache_evict(cache, state["table"], state["lens"], state["max_k"], state["new_table"], case["keep"],
                                   first=case["first"], last=case["last"])
    n = state["read"]
    return [lens, kept, cache.k[n:], cache.v[n:], cache.k_exp[n:], cache.v_exp[n:], cache.weight[n:]]


def _padded(state, name):
    """Every session's cached keys or values, padded to the longest: [nseq, H, max_k, d], zeros past the end."""
    page = state["table"].long().clamp(min=0)[:, :-(-state["max_k"] // PAGE)]
    scale = _power(state[name + "_exp"])
    x = (state[name][page].float() * scale[page][..., None, None]).transpose(1, 2).flatten(2, 3)[:, :, :state["max_k"]]
    live = torch.arange(state["max_k"], device="cuda")[None] < state["lens"][:, None]
    return torch.where(live[:, None, :, None], x, 0), live


def _rows(state):
    """Where each query row lies in the padded batch: its session and its place there."""
    t = torch.arange(state["q"].shape[0], device="cuda")
    s = torch.searchsorted(state["cu"].long(), t, right=True) - 1
    return s, t - state["cu"].long()[s]


def _scores(state, k, live):
    """[nseq, H, rows, max_k], the rows of a cached head being its query heads' tokens one after the other."""
    q, n, H = state["q"], len(state["lens"]), k.shape[1]
    G, d, rows = q.shape[1] // H, q.shape[2], state["max_q"]
    s, at = _rows(state)
    padded = torch.zeros(n, rows, H, G, d, device="cuda")
    padded[s, at] = q.float().view(-1, H, G, d)
    padded = padded.permute(0, 2, 1, 3, 4).reshape(n, H, rows * G, d)
    x = torch.matmul(padded, k.transpose(2, 3)).mul_(state["scale"])
    return x.masked_fill_(~live[:, None, None, :], -math.inf)


def _unpadded(state, x):
    """[nseq, H, rows, ...] back to [Tq, Hq, ...]."""
    n, H = x.shape[:2]
    s, at = _rows(state)
    x = x.reshape(n, H, state["max_q"], -1, *x.shape[3:]).transpose(1, 2)[s, at]
    return x.reshape(x.shape[0], -1, *x.shape[3:])


def _attn(state):
    k, live = _padded(state, "k")
    x = _scores(state, k, live)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    v, _ = _padded(state, "v")
    o = _unpadded(state, torch.matmul(x, v) / total).bfloat16()
    return [o, _unpadded(state, (top + total.log()).squeeze(-1))] if state["case"]["lse"] else [o]


def _weigh(state):
    k, live = _padded(state, "k")
    x = _scores(state, k, live)
    n, H, rows, _ = x.shape
    s, at = _rows(state)
    lse = torch.full((n, state["max_q"], H, rows // state["max_q"]), math.inf, device="cuda")
    lse[s, at] = state["lse"].view(-1, H, lse.shape[3])
    got = x.sub_(lse.transpose(1, 2).reshape(n, H, rows, 1)).exp_().sum(2)  # [nseq, H, max_k]
    got = torch.nn.functional.pad(got, (0, -got.shape[2] % PAGE)).unflatten(2, (-1, PAGE)).transpose(1, 2)
    page = state["table"].long()[:, :got.shape[1]]
    spare = state["weight"].shape[0] - 1
    live = torch.nn.functional.pad(live, (0, -live.shape[1] % PAGE)).unflatten(1, (-1, PAGE))[:, :, None]
    page = torch.where(live.any(-1).squeeze(-1), page, spare)
    after = state["after"]
    after[page] = torch.where(live, state["weight"][page] + got, after[page])
    return [after]


def _append(state):
    t = torch.arange(state["new_k"].shape[0], device="cuda")
    cu, lens, table = state["cu"].long(), state["lens"].long(), state["table"].long()
    s = torch.searchsorted(cu, t, right=True) - 1
    at = lens[s] + t - cu[s]
    page, slot = table[s, at // PAGE], at % PAGE
    pool = state["k"].shape[0]
    touched = torch.zeros(pool, dtype=torch.bool, device="cuda").index_fill(0, page, True)
    # the page that holds a session's last tokens, where new ones come into it
    tail = table.gather(1, (lens // PAGE).clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    tail = torch.where((lens % PAGE > 0) & (cu[1:] > cu[:-1]), tail, pool - 1)
    older = torch.zeros(pool, dtype=torch.bool, device="cuda").index_fill(0, tail, True)
    older[pool - 1] = False
    is_old = (torch.arange(PAGE, device="cuda") < (lens % PAGE)[:, None])[:, None, :, None]
    for name in ("k", "v"):
        x, exp = state["new_" + name].float(), state[name + "_exp"]
        amax = torch.zeros(pool, x.shape[1], device="cuda")
        amax.scatter_reduce_(0, page[:, None].expand(-1, x.shape[1]), x.abs().amax(2), "amax")
        e = torch.maximum(_scale_exp(amax), torch.where(older[:, None], exp.int(), 0))
        e = torch.where(touched[:, None], e, exp.int())
        old = state[name][tail]
        again = _e4m3(old.float() * _power(exp[tail])[:, :, None, None], e[tail][:, :, None, None])
        state[name][tail] = torch.where(is_old, again.view(torch.uint8), old.view(torch.uint8)).view(old.dtype)
        state[name][page, :, slot] = _e4m3(x, e[page][:, :, None])
        exp.copy_(e)
    state["weight"][page, :, slot] = 0
    n = state["read"]
    return [(lens + cu[1:] - cu[:-1]).int(), *(state[x][n:] for x in ("k", "v", "k_exp", "v_exp", "weight"))]


def _evict(state):
    case, lens = state["case"], state["lens"].long()
    keep, pool = case["keep"], state["k"].shape[0]
    page = state["table"].long().clamp(min=0)[:, :-(-state["max_k"] // PAGE)]
    w = state["weight"][page].transpose(1, 2).flatten(2)  # [nseq, H, tokens]
    at = torch.arange(w.shape[2], device="cuda")
    length = lens[:, None, None]
    w = torch.where((at < case["first"]) | (at >= length - case["last"]), math.inf, w).masked_fill(at >= length, -math.inf)
    kept = torch.sort(w, dim=2, descending=True, stable=True).indices[:, :, :keep].sort(2).values
    new_lens = lens.clamp(max=keep)
    kept = torch.nn.functional.pad(kept, (0, keep - kept.shape[2]), value=w.shape[2])
    gone = torch.arange(keep, device="cuda") >= new_lens[:, None, None]
    kept = kept.masked_fill(gone, 0)
    n, H = kept.shape[:2]
    src = page.unsqueeze(1).expand(-1, H, -1).gather(2, kept // PAGE)
    head = torch.arange(H, device="cuda")[None, :, None]
    pages = -(-keep // PAGE)
    more = pages * PAGE - keep
    first_slot = torch.arange(pages, device="cuda") * PAGE
    to = torch.where(first_slot < new_lens[:, None], state["new_table"].long(), pool - 1)  # [nseq, pages]
    live = ~torch.nn.functional.pad(gone, (0, more), value=True).view(n, 1, pages, PAGE).transpose(1, 2)

    def paged(x):
        x = torch.nn.functional.pad(x, (0, 0) * (x.dim() - 3) + (0, more))
        return x.unflatten(2, (pages, PAGE)).transpose(1, 2)

    for name in ("k", "v"):
        exp = state[name + "_exp"]
        x = state[name][src, head, kept % PAGE].float() * _power(exp[src, head])[..., None]
        x = torch.where(live[..., None], paged(x), 0)
        e = _scale_exp(x.abs().amax((3, 4)))
        was = state[name][to]
        state[name][to] = torch.where(live[..., None], _e4m3(x, e[..., None, None]).view(torch.uint8), was.view(torch.uint8)).view(was.dtype)
        exp[to] = torch.where(live.any(-1), e.to(torch.uint8), exp[to])
    state["weight"][to] = torch.where(live, paged(state["weight"][src, head, kept % PAGE]), state["weight"][to])
    r = state["read"]
    return [new_lens.int(), kept.masked_fill(gone, -1).int(), *(state[x][r:] for x in ("k", "v", "k_exp", "v_exp", "weight"))]


# ---- the definition in 64 bits, session by session


def _two(n):
    """2^n in 64 bits, exactly."""
    return ((n.to(torch.int64) + 1023) << 52).view(torch.float64)


def _round_e4m3(x):
    """The nearest e4m3 value (ties to even): 4 significant bits from 2^-6 on, steps of 2^-9 below."""
    _, e = torch.frexp(x)
    step = _two((e - 4).clamp(min=-9))
    return torch.round(x / step) * step


def exact(case, seed):
    state = prepare(case, seed)
    lq, lk, H, G = _ints(case["lq"]), _ints(case["lk"]), case["H"], case["G"]
    scale, r = state["scale"], state["read"]
    if case["op"] in ("attn", "weigh"):
        o = torch.zeros(sum(lq), H * G, case["d"], dtype=torch.float64, device="cuda")
        lse = torch.zeros(sum(lq), H * G, dtype=torch.float64, device="cuda")
        after = state["weight"].double()
        t = 0
        for s, (a, b) in enumerate(zip(lq, lk)):
            k, (page, slot) = _tokens(state, "k", s, b, torch.float64)
            v, _ = _tokens(state, "v", s, b, torch.float64)
            for hq in range(H * G):
                h = hq // G
                x = state["q"][t:t + a, hq].double() @ k[h].T * scale
                if case["op"] == "attn":
                    lse[t:t + a, hq] = torch.logsumexp(x, 1)
                    o[t:t + a, hq] = torch.softmax(x, 1) @ v[h]
                else:
                    after[page, h, slot] += torch.exp(x - state["lse"][t:t + a, hq, None].double()).sum(0)
            t += a
        return [after] if case["op"] == "weigh" else [o, lse] if case["lse"] else [o]
    pools = {}
    for name in ("k", "v"):
        pools[name], pools[name + "_exp"] = state[name].double(), state[name + "_exp"].double()
    weight = state["weight"].double()

    def put(name, page, slots, x, least):
        """x [H, slots, d] into the slots of a page, at the least exponent that holds x and not under `least` [H]."""
        ratio = x.abs().amax((1, 2)) / 448
        n = torch.where(ratio > 0, torch.ceil(torch.log2(ratio)), -100.0).clamp(min=-100)
        n = torch.where(ratio > _two(n), n + 1, torch.where(ratio <= _two(n - 1), n - 1, n)).clamp(min=-100)
        n = torch.maximum(n, least)
        pools[name][page, :, slots] = _round_e4m3(x * _two(-n)[:, None, None])
        pools[name + "_exp"][page] = n + 127
        return n

    if case["op"] == "append":
        t = 0
        for s, (a, b) in enumerate(zip(lq, lk)):
            row = state["table"][s].tolist()
            for j in range(b // PAGE, -(-(b + a) // PAGE) if a else 0):
                lo, hi = max(b, j * PAGE), min(b + a, (j + 1) * PAGE)
                page, old = row[j], lo - j * PAGE
                for name in ("k", "v"):
                    was = pools[name + "_exp"][page].clone() - 127
                    x = state["new_" + name][t + lo - b:t + hi - b].double().transpose(0, 1)
                    before = pools[name][page, :, :old] * _two(was)[:, None, None]
                    n = put(name, page, slice(old, old + hi - lo), x, was if old else torch.full_like(was, -100))
                    pools[name][page, :, :old] = _round_e4m3(before * _two(-n)[:, None, None])
                weight[page, :, old:old + hi - lo] = 0
            t += a
        return [None, pools["k"][r:], pools["v"][r:], None, None, weight[r:]]
    if sum(lk) * H > 2_000_000:
        return None
    for s, b in enumerate(lk):
        row, n = state["table"][s].long(), min(b, case["keep"])
        at = torch.arange(b, device="cuda")
        w = state["weight"][row[at // PAGE], :, at % PAGE].double()  # [tokens, H]
        rank = w.clone()
        rank[:case["first"]] = math.inf
        rank[max(0, b - case["last"]):] = math.inf
        # the n first by weight and then by place, in order of place
        kept = [sorted(sorted(range(b), key=lambda i, v=r: (-v[i], i))[:n]) for r in rank.T.tolist()]
        for j in range(-(-n // PAGE)):
            page, live = int(state["new_table"][s, j]), min(PAGE, n - j * PAGE)
            ids = torch.tensor([x[j * PAGE:j * PAGE + live] for x in kept], device="cuda")  # [H, live]
            src, head = row[ids // PAGE], torch.arange(H, device="cuda")[:, None]
            for name in ("k", "v"):
                x = state[name].view(torch.uint8)[src, head, ids % PAGE].view(torch.float8_e4m3fn).double()
                x = x * _two(state[name + "_exp"][src, head].long() - 127)[..., None]
                put(name, page, slice(0, live), x, torch.full((H,), -100.0, dtype=torch.float64, device="cuda"))
            weight[page, :, :live] = w.T.gather(1, ids)
    return [None, None, pools["k"][r:], pools["v"][r:], None, None, weight[r:]]
