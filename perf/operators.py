"""The operators for serving many sequences from one pool of cache pages, as measurable cases.

``kind`` names the operator:

    rope     rotation of queries and keys by positions with several axes (time, row, column), forward, or the gradient (``grad``)
    append   new keys, rotated by their positions, and values enter the pages of their sequences; the queries are rotated beside them
    attend   attention of every sequence's new tokens over its pages

Sizes: ``seqs`` sequences with up to ``ctx`` tokens in the cache each and up to ``new`` new ones (``spread``: the lengths are spread
below these, otherwise all alike), ``heads`` query heads that share ``heads_kv`` key and value heads of ``head_dim`` features, pages
of ``page`` tokens.  ``causal``, ``window`` and ``sink`` say which keys a token sees; a chunk of video frames sees all of itself.
``pairs``: feature pairs of the axes, as text; ``halves``: pair p is features (p, p + P) instead of (2 p, 2 p + 1); ``shared``: one
spectrum of frequencies over all axes; ``packed``: the operands are views into the rows of a joint projection.  Inputs are Gaussian.
"""
import math
import random

import torch

own = False

DEV = "cuda"
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, kind, **kw):
    base = dict(name=name, kind=kind, dtype="bf16", heads=32, heads_kv=8, head_dim=128, seqs=1, new=1, ctx=0, spread=False, page=64,
                causal=True, window=0, sink=0, pairs="64", halves=True, shared=True, theta=10000.0, grad=False, packed=False)
    base.update(kw)
    return base


def listed():
    return [
        # one token's queries and keys: what a decoding step pays for the rotation alone
        _case("rope_one", "rope", heads=40, pairs="16,24,24"),
        # queries and keys of a chunk of three 1280x720 frames in the rows of the joint projection
        _case("rope_1280x720", "rope", heads=80, new=10800, pairs="22,21,21", halves=False, shared=False, packed=True),
        # the gradient of a rotation that leaves part of the features alone, in fp32, odd sizes
        _case("rope_grad_f32", "rope", dtype="f32", heads=7, head_dim=64, seqs=5, new=1111, pairs="8,8,8", grad=True),
        # one token each of 64 sequences
        _case("append_decode", "append", seqs=64, ctx=4000, spread=True, page=16),
        # a chunk of three 832x480 frames of two streams, a frame a page
        _case("append_832x480", "append", heads=12, heads_kv=12, seqs=2, new=4680, ctx=9360, page=1560, pairs="22,21,21", halves=False,
              shared=False),
        # prompts of different lengths in fp32
        _case("append_prompts_f32", "append", dtype="f32", heads=16, heads_kv=4, head_dim=64, seqs=7, new=1500, ctx=700, spread=True,
              page=48, pairs="32"),
        # one token over a short context: the least that a call costs
        _case("attend_one", "attend", heads=12, heads_kv=12, ctx=117),
        # one token each of 64 sequences of different lengths
        _case("attend_decode", "attend", seqs=64, ctx=8191, spread=True, page=16),
        # four tokens (a draft to be checked) at the end of one long context
        _case("attend_long", "attend", new=4, ctx=131071),
        # a chunk of three 832x480 frames over sink frame and sliding window
        _case("attend_832x480", "attend", heads=12, heads_kv=12, new=4680, ctx=9360, page=1560, causal=False, window=9360, sink=1560),
        # chunks of prompts, causal, in groups of four heads
        _case("attend_prompts", "attend", seqs=4, new=2048, ctx=6100, spread=True),
        # single tokens and chunks of prompts in one batch, in fp32
        _case("attend_mixed_f32", "attend", dtype="f32", heads=8, heads_kv=2, head_dim=64, seqs=6, new=700, ctx=2000, spread=True, page=40,
              window=1000, sink=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"], c["dtype"]] = max(most.get((c["kind"], c["dtype"]), 0.0), w["bytes"] / 5e12 + w["flops"] / (1e15 if c["dtype"] == "bf16" else 1e14))
    most["rope", "f32"] = most["append", "f32"] = most["append", "bf16"]
    while True:
        kind = rng.choice(["rope", "append", "attend", "attend", "attend"])
        group, heads_kv = rng.choice([1, 1, 2, 3, 4, 4, 8]), _log_int(rng, 1, 16)
        d = rng.choice([64, 128, 128])
        c = _case("", kind, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), heads_kv=heads_kv, heads=group * heads_kv, head_dim=d,
                  page=rng.choice([16, 32, 64, 128, 256, 1560, _log_int(rng, 8, 200)]), spread=rng.random() < 0.7)
        del c["name"]
        full = d // 2
        c.update(rng.choice([dict(pairs="%d,%d,%d" % (full - 2 * (full // 3), full // 3, full // 3), halves=False, shared=False),
                             dict(pairs="%d,%d,%d" % (full // 4, full // 4 + full // 8, full // 4 + full // 8)), dict(pairs=str(full)),
                             dict(pairs=str(full // 2)), dict(pairs="%d,%d" % (full // 2, full // 2), halves=False)]))
        if kind == "rope":
            c.update(seqs=rng.choice([1, 1, 2, 5]), new=_log_int(rng, 1, 20000), grad=rng.random() < 0.3, packed=rng.random() < 0.4)
        elif rng.random() < 0.5:   # single tokens, or a few
            c.update(seqs=_log_int(rng, 1, 128), new=rng.choice([1, 1, 1, 2, 4]), ctx=_log_int(rng, 1, 100000))
        else:
            c.update(seqs=_log_int(rng, 1, 8), new=_log_int(rng, 16, 6000), ctx=rng.choice([0, _log_int(rng, 1, 16000)]))
        if kind == "attend":
            if rng.random() < 0.3:
                c.update(window=_log_int(rng, 100, 10000), sink=rng.choice([0, 4, c["page"]]))
            c["causal"] = rng.random() < 0.7
        w = work(c)
        cost = w["bytes"] / 5e12 + w["flops"] / (1e15 if c["dtype"] == "bf16" else 1e14)
        held = max(1, c["seqs"]) * (c["ctx"] + c["new"]) * c["heads_kv"] * d
        scores = c["seqs"] * c["heads"] * c["new"] * (c["ctx"] + c["new"])
        if cost <= most[kind, c["dtype"]] and held <= 5e8 and (kind != "attend" or scores <= 2.5e9):
            return c


def _lengths(case):
    """New tokens and tokens before them of every sequence: the same for every seed."""
    n, new, ctx = case["seqs"], case["new"], case["ctx"]
    if not case["spread"]:
        return [new] * n, [ctx] * n
    rng = random.Random(1000003 * n + 1009 * new + ctx)
    part = [1.0] + [rng.uniform(0.05, 1.0) for _ in range(n - 1)]
    few = [1.0] + [rng.choice([0.0, rng.uniform(0.1, 1.0), rng.uniform(0.1, 1.0)]) for _ in range(n - 1)]
    return [max(1, round(new * f)) for f in few], [round(ctx * f) for f in part]


def _pairs(case):
    return [int(p) for p in case["pairs"].split(",")]


def _seen(case, p, length):
    """Keys that the token at place p sees, as ranges (sink, window)."""
    end = min(length, p + 1) if case["causal"] else length
    first = max(0, p - case["window"] + 1) if case["window"] else 0
    sink = min(case["sink"], end, first) if case["window"] else 0
    return sink, min(first, end), end


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    new, ctx = _lengths(case)
    d, H, Hk = case["head_dim"], case["heads"], case["heads_kv"]
    n, axes = sum(new), len(_pairs(case))
    rot = 6 * sum(_pairs(case))
    if case["kind"] == "rope":
        n = case["seqs"] * case["new"]
        return {"bytes": n * (2 * H * d * es + 4 * axes), "flops": n * H * rot}
    tables = 4 * (2 * case["seqs"] + 1)
    if case["kind"] == "append":
        pages = sum((c + m - 1) // case["page"] - c // case["page"] + 1 for m, c in zip(new, ctx))
        return {"bytes": n * (2 * (H + 2 * Hk) * d * es + 4 * axes) + 4 * pages + tables, "flops": n * (H + Hk) * rot}
    keys = see = pages = 0
    for m, c in zip(new, ctx):
        sink, first, _ = _seen(case, c, c + m)           # the first token's window reaches back the furthest
        held = sink + (c + m - first)
        keys += held
        pages += -(-held // case["page"])
        if case["window"]:
            see += sum(s + e - f for s, f, e in (_seen(case, c + i, c + m) for i in range(m)))
        else:
            see += m * c + m * (m + 1) // 2 if case["causal"] else m * (c + m)
    return {"bytes": 2 * n * H * d * es + 2 * keys * Hk * d * es + 4 * pages + tables, "flops": 4 * d * H * see}


def _positions(case, new, ctx, axes):
    """Every new token's place on every axis: text counts on, frames of a chunk are a grid of up to 30 x 52."""
    at = torch.cat([torch.arange(c, c + m, device=DEV) for m, c in zip(new, ctx)])
    if axes == 1 or case["halves"]:
        return torch.stack([at // (1 + a) for a in range(axes)]).to(torch.int32)
    grid = [at // 1560, at % 1560 // 52, at % 52]
    return torch.stack(grid[:axes]).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t, d, H, Hk, P = _TYPES[case["dtype"]], case["head_dim"], case["heads"], case["heads_kv"], case["page"]
    new, ctx = _lengths(case)
    normal = lambda *shape: torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(t)  # noqa: E731
    s = {"case": case}
    if case["kind"] == "rope":
        B, n, axes = case["seqs"], case["new"], len(_pairs(case))
        start = int(torch.randint(0, 1000, (1,), generator=g, device=DEV))
        s["pos"] = _positions(case, [n], [start], axes)
        if case["packed"]:   # rows of a joint projection of which the last third is left alone
            s["X"] = normal(B, n, H + (H + 1) // 2, d)[:, :, :H].transpose(1, 2)
        else:
            s["X"] = normal(B, H, n, d)
        s["Y"] = torch.empty((B, H, n, d), dtype=t, device=DEV)
        return s
    n_pages = [-(-(m + c) // P) for m, c in zip(new, ctx)]
    width, total = max(n_pages), sum(n_pages) + 3
    order = torch.randperm(total, generator=g, device=DEV)[:sum(n_pages)].to(torch.int32)
    s["table"] = torch.zeros((case["seqs"], width), dtype=torch.int32, device=DEV)
    at = 0
    for i, k in enumerate(n_pages):
        s["table"][i, :k] = order[at:at + k]
        at += k
    s["K_pages"], s["V_pages"] = normal(total, Hk, P, d), normal(total, Hk, P, d)
    cu = [0]
    for m in new:
        cu.append(cu[-1] + m)
    s["n"], s["longest"], s["new"] = cu[-1], max(m + c for m, c in zip(new, ctx)), max(new)
    s["cu"] = torch.tensor(cu, dtype=torch.int32, device=DEV)
    s["lens"] = torch.tensor([m + c for m, c in zip(new, ctx)], dtype=torch.int32, device=DEV)
    rows = normal(s["n"], H + 2 * Hk, d)   # the joint projection's output
    s["Q"], s["K"], s["V"] = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    if case["kind"] == "append":
        s["pos"] = _positions(case, new, ctx, len(_pairs(case)))
        s["Q_out"] = torch.empty((s["n"], H, d), dtype=t, device=DEV)
    else:
        s["O"] = torch.empty((s["n"], H, d), dtype=t, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _turn(case, X, pos):
    """Rotated rows of X [..., tokens, d] (fp32 arithmetic, angles in 64 bits); pos [axes, tokens]."""
    pairs = _pairs(case)
    P = sum(pairs)
    axis = torch.cat([torch.full((n,), a) for a, n in enumerate(pairs)]).to(DEV)
    if case["shared"]:
        power = torch.arange(P, dtype=torch.float64, device=DEV) / P
    else:
        power = torch.cat([torch.arange(n, dtype=torch.float64, device=DEV) / n for n in pairs])
    angle = pos.to(torch.float64)[axis].T * case["theta"] ** -power
    c, s = torch.cos(angle).float(), torch.sin(angle).float()
    if case["grad"]:
        s = -s
    x = X.float()
    a, b = (x[..., :P], x[..., P:2 * P]) if case["halves"] else (x[..., 0:2 * P:2], x[..., 1:2 * P:2])
    u, v = a * c - b * s, a * s + b * c
    turned = torch.cat([u, v], -1) if case["halves"] else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * P:]], -1).to(X.dtype)


def _rows(s):
    """Sequence and index within it of every packed row."""
    at = torch.arange(s["n"], dtype=torch.int32, device=DEV)
    seq = torch.searchsorted(s["cu"], at, right=True) - 1
    return seq, at - s["cu"][seq]


def _plain_append(s):
    case, P = s["case"], s["case"]["page"]
    seq, i = _rows(s)
    slot = (s["lens"] - (s["cu"][1:] - s["cu"][:-1]))[seq] + i
    page, inside = s["table"][seq, slot // P].long(), (slot % P).long()
    s["K_pages"][page, :, inside] = _turn(case, s["K"].transpose(0, 1), s["pos"]).transpose(0, 1)
    s["V_pages"][page, :, inside] = s["V"]
    return s["K_pages"], s["V_pages"], _turn(case, s["Q"].transpose(0, 1), s["pos"]).transpose(0, 1).contiguous()


def _plain_attend(s):
    case = s["case"]
    S, H, Hk, d, L, m = case["seqs"], case["heads"], case["heads_kv"], case["head_dim"], s["longest"], s["new"]
    lens, count = s["lens"][:, None], (s["cu"][1:] - s["cu"][:-1])[:, None]
    i = torch.arange(m, device=DEV)
    Q = s["Q"][torch.clamp(s["cu"][:-1, None] + i, max=s["n"] - 1)].float()                 # [S, m, H, d]
    Q = Q.view(S, m, Hk, H // Hk, d).permute(0, 2, 3, 1, 4).reshape(S * Hk, H // Hk * m, d)
    kv = lambda pages: pages[s["table"]].transpose(1, 2).flatten(2, 3)[:, :, :L].float().reshape(S * Hk, L, d)  # noqa: E731
    score = torch.bmm(Q, kv(s["K_pages"]).transpose(1, 2).contiguous()).view(S, Hk, H // Hk, m, L)
    score *= 1.0 / math.sqrt(d)
    p, j = (lens - count + i)[:, :, None], torch.arange(L, device=DEV)
    sees = (j < lens[:, :, None]) & (i < count)[:, :, None]
    if case["causal"]:
        sees = sees & (j <= p)
    if case["window"]:
        sees = sees & ((j > p - case["window"]) | (j < case["sink"]))
    score.masked_fill_(~sees[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    total = score.sum(-1)
    out = torch.bmm(score.view(S * Hk, H // Hk * m, L), kv(s["V_pages"])).view(S, Hk, H // Hk, m, d)
    out = torch.where(total[..., None] > 0, out / total[..., None], 0.0).permute(0, 3, 1, 2, 4).reshape(S, m, H, d)
    seq, at = _rows(s)
    return out[seq, at].to(s["Q"].dtype)


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own(s):
    import paper_2604_10103_amd as hf

    case = s["case"]
    if "hf" not in s:   # what a program keeps for all its steps
        t = case["dtype"]
        rope = cache = ws = None
        if case["kind"] != "attend":
            rope = hf.make_rope_axes(_pairs(case), theta=case["theta"], layout=hf.HF_ROPE_HALVES if case["halves"] else hf.HF_ROPE_ADJACENT,
                                     spectrum=hf.HF_ROPE_SHARED if case["shared"] else hf.HF_ROPE_PER_AXIS)
        if case["kind"] != "rope":
            cache = hf.make_paged(case["heads"], case["heads_kv"], case["head_dim"], t, case["page"], s["K_pages"].shape[0],
                                  case["seqs"], s["table"].shape[1], causal=case["causal"], window=case["window"], n_sink=case["sink"])
        if case["kind"] == "attend":
            ws = torch.empty(hf.hf_paged_workspace_bytes(cache, s["n"]), dtype=torch.uint8, device=DEV)
        s["hf"] = rope, cache, ws
    rope, cache, ws = s["hf"]
    if case["kind"] == "rope":
        hf.hf_rope_axes_apply(rope, s["X"], s["pos"], s["Y"], inverse=case["grad"])
        return s["Y"]
    if case["kind"] == "append":
        hf.hf_paged_append(cache, s["K"], s["V"], s["cu"], s["lens"], s["K_pages"], s["V_pages"], s["table"], rope=rope,
                           positions=s["pos"], Q=s["Q"], Q_out=s["Q_out"])
        return s["K_pages"], s["V_pages"], s["Q_out"]
    hf.hf_paged_attn_fwd(cache, s["Q"], s["cu"], s["lens"], s["K_pages"], s["V_pages"], s["table"], s["O"], ws)
    return s["O"]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "rope":
        return _turn(state["case"], state["X"], state["pos"])
    return _plain_append(state) if kind == "append" else _plain_attend(state)


# ------------------------------------------------------------------------------------------------ 64 bits, from the definitions
def _turned64(case, x, pos):
    """x [tokens, heads, d] in 64 bits as complex numbers times e^(i angle)."""
    pairs, y, first = _pairs(case), x.clone(), 0
    P = sum(pairs)
    for a, n in enumerate(pairs):
        for i in range(n):
            p = first + i
            w = case["theta"] ** (-(p / P) if case["shared"] else -(i / n))
            re, im = (p, p + P) if case["halves"] else (2 * p, 2 * p + 1)
            angle = (pos[a].double() * w * (-1.0 if case["grad"] else 1.0))[:, None]
            z = torch.complex(x[..., re], x[..., im]) * torch.polar(torch.ones_like(angle), angle)
            y[..., re], y[..., im] = z.real, z.imag
        first += n
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return torch.stack([_turned64(case, x.transpose(0, 1).double(), s["pos"]).transpose(0, 1) for x in s["X"]])
    new, ctx = _lengths(case)
    P, group, row = case["page"], case["heads"] // case["heads_kv"], 0
    if case["kind"] == "append":
        K, V = s["K_pages"].double(), s["V_pages"].double()
        turned = _turned64(case, s["K"].double(), s["pos"])
        for q, (m, c) in enumerate(zip(new, ctx)):
            while m:   # a page at a time
                k = min(m, P - c % P)
                page = int(s["table"][q, c // P])
                K[page, :, c % P:c % P + k] = turned[row:row + k].transpose(0, 1)
                V[page, :, c % P:c % P + k] = s["V"][row:row + k].double().transpose(0, 1)
                row, m, c = row + k, m - k, c + k
        return K, V, _turned64(case, s["Q"].double(), s["pos"])
    O = torch.zeros((s["n"], case["heads"], case["head_dim"]), dtype=torch.float64, device=DEV)
    for q, (m, c) in enumerate(zip(new, ctx)):
        pages = s["table"][q, :-(-(m + c) // P)].long()
        p, j = torch.arange(c, c + m, device=DEV)[:, None], torch.arange(c + m, device=DEV)[None]
        hidden = torch.zeros((m, c + m), dtype=torch.bool, device=DEV)
        if case["causal"]:
            hidden |= j > p
        if case["window"]:
            hidden |= (j <= p - case["window"]) & (j >= case["sink"])
        for h in range(case["heads"]):
            k = s["K_pages"][pages, h // group].flatten(0, 1)[:c + m].double()
            v = s["V_pages"][pages, h // group].flatten(0, 1)[:c + m].double()
            logit = (s["Q"][row:row + m, h].double() @ k.T) / math.sqrt(case["head_dim"])
            O[row:row + m, h] = torch.softmax(logit.masked_fill(hidden, -math.inf), -1) @ v
        row += m
    return O
