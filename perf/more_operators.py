"""The operators around a cache of pages in 8 bits, as measurable cases.

``kind`` names the operator:

    norm     queries or keys of a layer: every head's row brought to unit mean square, weighted, and rotated by its positions, forward, or
             the gradients of rows and weights (``grad``)
    append   new keys (normalised, rotated) and values enter the pages of their sequences as e4m3 with a scale for each row; the queries are
             normalised and rotated beside them
    attend   attention of every sequence's new tokens over such pages

Sizes: ``seqs`` sequences (``norm``: batches) with up to ``ctx`` tokens in the cache each and up to ``new`` new ones (``spread``: the lengths
are spread below these, otherwise all alike), ``heads`` query heads that share ``heads_kv`` key and value heads of ``head_dim`` features,
pages of ``page`` tokens.  ``causal``, ``window`` and ``sink`` say which keys a token sees; a chunk of video frames sees all of itself.
``pairs``: feature pairs of the axes, as text (none: no rotation); ``halves``: pair p is features (p, p + P) instead of (2 p, 2 p + 1);
``shared``: one spectrum of frequencies over all axes; ``factor``: how many times longer than the ``trained`` one the first axis may get;
``weights``: of the norm, one row for all heads, one for each head, or none; ``packed``: the rows are a view into those of a joint
projection.  Rows are Gaussian, their sizes and the weights spread.
"""
import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SLOW, FAST = 1.0, 32.0   # turns over the trained length: pairs with fewer are slowed by the whole factor, with more not at all


def _case(name, kind, **kw):
    base = dict(name=name, kind=kind, dtype="bf16", heads=32, heads_kv=8, head_dim=128, seqs=1, new=1, ctx=0, spread=False, page=64,
                causal=True, window=0, sink=0, pairs="64", halves=True, shared=True, theta=10000.0, factor=1.0, trained=4096,
                weights="one", grad=False, packed=False)
    base.update(kw)
    return base


def listed():
    return [
        # one token's queries: what a decoding step pays for norm and rotation alone
        _case("norm_one", "norm", heads=40, pairs="16,24,24"),
        # queries of a chunk of three 1280x720 frames in the rows of the joint projection
        _case("norm_1280x720", "norm", heads=40, new=10800, pairs="22,21,21", halves=False, shared=False, packed=True),
        # training: the gradients for a chunk of three 832x480 frames of two streams
        _case("norm_grad_832x480", "norm", heads=12, seqs=2, new=4680, pairs="22,21,21", halves=False, shared=False, grad=True),
        # gradients in fp32, odd sizes, weights for each head, a rotation of part of the features
        _case("norm_grad_f32", "norm", dtype="f32", heads=7, head_dim=64, seqs=5, new=1111, pairs="8,8,8", weights="each", grad=True),
        # one token each of 64 sequences
        _case("append_decode", "append", seqs=64, ctx=4000, spread=True, page=16),
        # a chunk of three 832x480 frames of two streams, a frame a page
        _case("append_832x480", "append", heads=12, heads_kv=12, seqs=2, new=4680, ctx=9360, page=1560, pairs="22,21,21", halves=False,
              shared=False),
        # prompts of different lengths in fp32, rotation scaled for a context four times as long as the trained one
        _case("append_prompts_f32", "append", dtype="f32", heads=16, heads_kv=4, head_dim=64, seqs=7, new=1500, ctx=700, spread=True,
              page=48, pairs="32", factor=4.0),
        # one token over a short context: the least that a call costs
        _case("attend_one", "attend", heads=12, heads_kv=12, ctx=117),
        # one token each of 64 sequences of different lengths
        _case("attend_decode", "attend", seqs=64, ctx=8191, spread=True, page=16),
        # four tokens (a draft to be checked) at the end of one long context
        _case("attend_long", "attend", new=4, ctx=131071),
        # a chunk of three 832x480 frames over sink frame and sliding window
        _case("attend_832x480", "attend", heads=12, heads_kv=12, new=4680, ctx=9360, page=1560, causal=False, window=9360, sink=1560),
        # single tokens and chunks of prompts in one batch, in fp32
        _case("attend_mixed_f32", "attend", dtype="f32", heads=8, heads_kv=2, head_dim=64, seqs=6, new=700, ctx=2000, spread=True, page=40,
              window=1000, sink=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / (1e15 if case["dtype"] == "bf16" else 1e14)


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    while True:
        kind = rng.choice(["norm", "append", "attend", "attend"])
        group, heads_kv = rng.choice([1, 1, 2, 3, 4, 4, 8]), _log_int(rng, 1, 16)
        d = rng.choice([64, 128, 128])
        c = _case("", kind, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), heads_kv=heads_kv, heads=group * heads_kv, head_dim=d,
                  page=rng.choice([16, 32, 64, 128, 256, 1560, _log_int(rng, 8, 200)]), spread=rng.random() < 0.7)
        del c["name"]
        full = d // 2
        c.update(rng.choice([dict(pairs="%d,%d,%d" % (full - 2 * (full // 3), full // 3, full // 3), halves=False, shared=False),
                             dict(pairs="%d,%d,%d" % (full // 4, full // 4 + full // 8, full // 4 + full // 8)), dict(pairs=str(full)),
                             dict(pairs=str(full // 2)), dict(pairs="%d,%d" % (full // 2, full // 2), halves=False), dict(pairs="")]))
        if c["pairs"] and rng.random() < 0.4:
            c.update(factor=round(rng.uniform(1.5, 16.0), 3), trained=rng.choice([512, 4096, 8192]))
        c["weights"] = rng.choice(["one", "one", "each", "none"])
        if kind == "norm":
            c.update(seqs=rng.choice([1, 1, 2, 5]), new=_log_int(rng, 1, 20000), grad=rng.random() < 0.5, packed=rng.random() < 0.4)
        elif rng.random() < 0.5:   # single tokens, or a few
            c.update(seqs=_log_int(rng, 1, 128), new=rng.choice([1, 1, 1, 2, 4]), ctx=_log_int(rng, 1, 100000))
        else:
            c.update(seqs=_log_int(rng, 1, 8), new=_log_int(rng, 16, 6000), ctx=rng.choice([0, _log_int(rng, 1, 16000)]))
        if kind == "attend":
            if rng.random() < 0.3:
                c.update(window=_log_int(rng, 100, 10000), sink=rng.choice([0, 4, c["page"]]))
            c["causal"] = rng.random() < 0.7
        held = max(1, c["seqs"]) * (c["ctx"] + c["new"]) * c["heads_kv"] * d
        scores = c["seqs"] * c["heads"] * c["new"] * (c["ctx"] + c["new"])
        if _cost(c) <= most[kind] and held <= 5e8 and (kind != "attend" or scores <= 2.5e9):
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
    return [int(p) for p in case["pairs"].split(",") if p]


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
    each = 6 * sum(_pairs(case)) + 4 * d
    weights = {"one": 4 * d, "each": 4 * d * H, "none": 0}[case["weights"]]
    if case["kind"] == "norm":
        n = case["seqs"] * case["new"]
        if case["grad"]:
            return {"bytes": n * (3 * H * d * es + 4 * axes) + 2 * weights, "flops": n * H * (each + 8 * d)}
        return {"bytes": n * (2 * H * d * es + 4 * axes) + weights, "flops": n * H * each}
    tables = 4 * (2 * case["seqs"] + 1)
    if case["kind"] == "append":
        pages = sum((c + m - 1) // case["page"] - c // case["page"] + 1 for m, c in zip(new, ctx))
        return {"bytes": n * ((2 * H + 2 * Hk) * d * es + 2 * Hk * (d + 4) + 4 * axes) + 4 * pages + tables + 2 * weights,
                "flops": n * (H + Hk) * each + 4 * n * Hk * d}
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
    return {"bytes": 2 * n * H * d * es + 2 * keys * Hk * (d + 4) + 4 * pages + tables, "flops": 4 * d * H * see}


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
    normal = lambda *shape: torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)  # noqa: E731
    rows_of = lambda *shape: (normal(*shape, d) * (0.5 * normal(*shape, 1)).exp()).to(t)  # noqa: E731
    weight = lambda heads: (None if case["weights"] == "none" else  # noqa: E731
                            1.0 + 0.3 * (normal(heads, d) if case["weights"] == "each" else normal(d)))
    s = {"case": case}
    if case["kind"] == "norm":
        B, n, axes = case["seqs"], case["new"], len(_pairs(case))
        start = int(torch.randint(0, 1000, (1,), generator=g, device=DEV))
        s["pos"] = _positions(case, [n], [start], axes) if axes else None
        if case["packed"]:   # rows of a joint projection of which the last third is left alone
            s["X"] = rows_of(B, n, H + (H + 1) // 2)[:, :, :H].transpose(1, 2)
        else:
            s["X"] = rows_of(B, H, n)
        s["w"] = weight(H)
        if case["grad"]:
            s["dY"] = normal(B, H, n, d).to(t)
        s["out"] = torch.empty((B, H, n, d), dtype=t, device=DEV)
        return s
    n_pages = [-(-(m + c) // P) for m, c in zip(new, ctx)]
    width, total = max(n_pages), sum(n_pages) + 3
    order = torch.randperm(total, generator=g, device=DEV)[:sum(n_pages)].to(torch.int32)
    s["table"] = torch.zeros((case["seqs"], width), dtype=torch.int32, device=DEV)
    at = 0
    for i, k in enumerate(n_pages):
        s["table"][i, :k] = order[at:at + k]
        at += k
    for name in ("K", "V"):   # a pool in use: rows of unit mean square, weighted (K), or of spread sizes (V)
        pages = normal(total, Hk, P, d)
        pages = pages * (1.0 + 0.3 * normal(d)) if name == "K" else pages.mul_((0.5 * normal(total, Hk, P, 1)).exp())
        scale = pages.abs().amax(-1) / 448.0
        s[name + "_pages"], s[name + "_scales"] = pages.div_(scale[..., None]).to(torch.float8_e4m3fn), scale
    cu = [0]
    for m in new:
        cu.append(cu[-1] + m)
    s["n"], s["longest"], s["new"] = cu[-1], max(m + c for m, c in zip(new, ctx)), max(new)
    s["cu"] = torch.tensor(cu, dtype=torch.int32, device=DEV)
    s["lens"] = torch.tensor([m + c for m, c in zip(new, ctx)], dtype=torch.int32, device=DEV)
    rows = normal(s["n"], H + 2 * Hk, d).to(t) if case["kind"] == "attend" else rows_of(s["n"], H + 2 * Hk)   # the joint projection's output
    s["Q"], s["K"], s["V"] = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    if case["kind"] == "append":
        s["pos"] = _positions(case, new, ctx, len(_pairs(case))) if _pairs(case) else None
        s["wq"], s["wk"] = weight(H), weight(Hk)
        s["Q_out"] = torch.empty((s["n"], H, d), dtype=t, device=DEV)
    else:
        s["O"] = torch.empty((s["n"], H, d), dtype=t, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _angles(case, pos):
    """cos and sin [tokens, P] in fp32; the angles in 64 bits, pairs of the first axis slowed as ``factor`` says."""
    pairs = _pairs(case)
    P = sum(pairs)
    axis = torch.cat([torch.full((n,), a) for a, n in enumerate(pairs)]).to(DEV)
    if case["shared"]:
        power = torch.arange(P, dtype=torch.float64, device=DEV) / P
    else:
        power = torch.cat([torch.arange(n, dtype=torch.float64, device=DEV) / n for n in pairs])
    rate = case["theta"] ** -power
    if case["factor"] != 1.0:
        keep = ((rate * (case["trained"] / (2 * math.pi)) - SLOW) / (FAST - SLOW)).clamp(0.0, 1.0)
        rate = torch.where(axis == 0, rate * (keep + (1.0 - keep) / case["factor"]), rate)
    angle = pos.to(torch.float64)[axis].T * rate
    a = _amplitude(case)
    return (a * torch.cos(angle)).float(), (a * torch.sin(angle)).float()


def _amplitude(case):
    return 1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0


def _turn(case, x, c, s):
    P = c.shape[-1]
    a, b = (x[..., :P], x[..., P:2 * P]) if case["halves"] else (x[..., 0:2 * P:2], x[..., 1:2 * P:2])
    u, v = a * c - b * s, a * s + b * c
    turned = torch.cat([u, v], -1) if case["halves"] else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * P:]], -1)


def _unit(X):
    """Rows at unit mean square, and what they were multiplied with."""
    x = X.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _norm_turn(case, X, w, cs):
    """fp32 rows [..., heads, tokens, d], normalised, weighted (w [d] or [heads, d]) and turned."""
    y = _unit(X)[0]
    if w is not None:
        y = y * (w[:, None] if w.dim() == 2 else w)
    return _turn(case, y, *cs) if cs is not None else y


def _plain_norm(s):
    case, w = s["case"], s["w"]
    cs = _angles(case, s["pos"]) if s["pos"] is not None else None
    if not case["grad"]:
        return _norm_turn(case, s["X"], w, cs).to(s["X"].dtype)
    x, r = _unit(s["X"])
    g = s["dY"].float()
    if cs is not None:
        g = _turn(case, g, cs[0], -cs[1])
    h = g if w is None else g * (w[:, None] if w.dim() == 2 else w)
    dX = (r * (h - x * (h * x).mean(-1, keepdim=True))).to(s["X"].dtype)
    if w is None:
        return dX
    return dX, (g * x).sum((0, 2) if w.dim() == 2 else (0, 1, 2), dtype=torch.float64).float()


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
    cs = _angles(case, s["pos"]) if s["pos"] is not None else None
    for name, x in (("K", _norm_turn(case, s["K"].transpose(0, 1), s["wk"], cs).transpose(0, 1)), ("V", s["V"].float())):
        scale = x.abs().amax(-1) / 448.0
        s[name + "_pages"].view(torch.uint8)[page, :, inside] = (x / scale[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        s[name + "_scales"][page, :, inside] = scale
    q = _norm_turn(case, s["Q"].transpose(0, 1), s["wq"], cs).transpose(0, 1).to(s["Q"].dtype).contiguous()
    return s["K_pages"], s["V_pages"], s["K_scales"], s["V_scales"], q


def _plain_attend(s):
    case = s["case"]
    S, H, Hk, d, L, m = case["seqs"], case["heads"], case["heads_kv"], case["head_dim"], s["longest"], s["new"]
    lens, count = s["lens"][:, None], (s["cu"][1:] - s["cu"][:-1])[:, None]
    i = torch.arange(m, device=DEV)
    Q = s["Q"][torch.clamp(s["cu"][:-1, None] + i, max=s["n"] - 1)].float()                 # [S, m, H, d]
    Q = Q.view(S, m, Hk, H // Hk, d).permute(0, 2, 3, 1, 4).reshape(S * Hk, H // Hk * m, d)

    def kv(name):
        codes = s[name + "_pages"].view(torch.uint8)[s["table"]].transpose(1, 2).flatten(2, 3)[:, :, :L].contiguous().view(torch.float8_e4m3fn)
        scale = s[name + "_scales"][s["table"]].transpose(1, 2).flatten(2, 3)[:, :, :L]
        return (codes.float() * scale[..., None]).reshape(S * Hk, L, d)

    score = torch.bmm(Q, kv("K").transpose(1, 2).contiguous()).view(S, Hk, H // Hk, m, L)
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
    out = torch.bmm(score.view(S * Hk, H // Hk * m, L), kv("V")).view(S, Hk, H // Hk, m, d)
    out = torch.where(total[..., None] > 0, out / total[..., None], 0.0).permute(0, 3, 1, 2, 4).reshape(S, m, H, d)
    seq, at = _rows(s)
    return out[seq, at].to(s["Q"].dtype)


# ------------------------------------------------------------------------------------------------ the framework's calls
def _kept(s):
    """What a program keeps for all its steps."""
    import paper_2604_10103_amd as hf

    case = s["case"]
    rope = scaling = cache = ws = None
    norm = hf.make_head_norm(eps=EPS, per_head=case["weights"] == "each")
    if case["kind"] != "attend" and _pairs(case):
        rope = hf.make_rope_axes(_pairs(case), theta=case["theta"], layout=hf.HF_ROPE_HALVES if case["halves"] else hf.HF_ROPE_ADJACENT,
                                 spectrum=hf.HF_ROPE_SHARED if case["shared"] else hf.HF_ROPE_PER_AXIS)
        if case["factor"] != 1.0:
            scaling = hf.make_rope_scaling(case["factor"], case["trained"], slow=SLOW, fast=FAST, amplitude=_amplitude(case), axes=[0])
    if case["kind"] == "norm" and case["grad"] and s["w"] is not None:
        B, H, n, d = s["X"].shape
        s["dw"] = torch.empty_like(s["w"])
        ws = torch.empty(hf.hf_norm_rope_bwd_workspace_bytes(norm, d, B, H, n), dtype=torch.uint8, device=DEV)
    if case["kind"] != "norm":
        cache = hf.make_paged(case["heads"], case["heads_kv"], case["head_dim"], case["dtype"], case["page"], s["K_pages"].shape[0],
                              case["seqs"], s["table"].shape[1], causal=case["causal"], window=case["window"], n_sink=case["sink"])
    if case["kind"] == "attend":
        ws = torch.empty(hf.hf_paged_e4m3_workspace_bytes(cache, s["n"]), dtype=torch.uint8, device=DEV)
    return norm, rope, scaling, cache, ws


def _own(s):
    import paper_2604_10103_amd as hf

    case = s["case"]
    if "hf" not in s:
        s["hf"] = _kept(s)
    norm, rope, scaling, cache, ws = s["hf"]
    if case["kind"] == "norm" and case["grad"]:
        hf.hf_norm_rope_bwd(s["X"], s["dY"], s["out"], norm=norm, weight=s["w"], rope=rope, positions=s["pos"], scaling=scaling,
                            dweight=s.get("dw"), workspace=ws)
        return s["out"] if s["w"] is None else (s["out"], s["dw"])
    if case["kind"] == "norm":
        hf.hf_norm_rope_fwd(s["X"], s["out"], norm=norm, weight=s["w"], rope=rope, positions=s["pos"], scaling=scaling)
        return s["out"]
    if case["kind"] == "append":
        hf.hf_paged_append_e4m3(cache, s["K"], s["V"], s["cu"], s["lens"], s["K_pages"], s["V_pages"], s["K_scales"], s["V_scales"],
                                s["table"], norm=norm, k_weight=s["wk"], q_weight=s["wq"], rope=rope, positions=s["pos"],
                                scaling=scaling, Q=s["Q"], Q_out=s["Q_out"])
        return s["K_pages"], s["V_pages"], s["K_scales"], s["V_scales"], s["Q_out"]
    hf.hf_paged_attn_e4m3_fwd(cache, s["Q"], s["cu"], s["lens"], s["K_pages"], s["V_pages"], s["K_scales"], s["V_scales"], s["table"],
                              s["O"], ws)
    return s["O"]


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "append": _plain_append, "attend": _plain_attend}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------ 64 bits, from the definitions
def _turned64(case, x, pos, way=1.0):
    """x [tokens, heads, d] in 64 bits as complex numbers times e^(i angle), and the amplitude."""
    pairs, y, first = _pairs(case), x.clone(), 0
    P = sum(pairs)
    long = case["factor"] != 1.0
    size = 1.0 + 0.1 * math.log(case["factor"]) if long else 1.0
    for a, n in enumerate(pairs):
        for i in range(n):
            p = first + i
            w = case["theta"] ** (-(p / P) if case["shared"] else -(i / n))
            if long and a == 0:
                turns = case["trained"] * w / (2.0 * math.pi)
                part = min(1.0, max(0.0, (turns - SLOW) / (FAST - SLOW)))
                w = part * w + (1.0 - part) * w / case["factor"]
            re, im = (p, p + P) if case["halves"] else (2 * p, 2 * p + 1)
            angle = (pos[a].double() * w * way)[:, None]
            z = torch.complex(x[..., re], x[..., im]) * torch.polar(torch.full_like(angle, size), angle)
            y[..., re], y[..., im] = z.real, z.imag
        first += n
    return y


def _normed64(case, X, w, pos):
    """X [tokens, heads, d] -> normalised, weighted and turned, in 64 bits."""
    x = X.double()
    y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["head_dim"] + EPS)
    return _turned64(case, y * w.double() if w is not None else y, pos)


def _exact_norm(s):
    case, w, d = s["case"], s["w"], s["case"]["head_dim"]
    if not case["grad"]:
        return torch.stack([_normed64(case, x.transpose(0, 1), w, s["pos"]).transpose(0, 1) for x in s["X"]])
    dX, dw = [], 0.0
    for X, dY in zip(s["X"], s["dY"]):
        x, g = X.transpose(0, 1).double(), _turned64(case, dY.transpose(0, 1).double(), s["pos"], way=-1.0)
        size = torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS)
        h = g * w.double() if w is not None else g
        dX.append((h / size - x * (h * x).sum(-1, keepdim=True) / (d * size ** 3)).transpose(0, 1))
        dw = dw + (g * x / size).sum(0)
    if w is None:
        return torch.stack(dX)
    return torch.stack(dX), dw if case["weights"] == "each" else dw.sum(0)


def _e4m3(x):
    """The nearest value of 4 significant bits, at least 2^-9 apart, ties to the even one; |x| <= 448."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s)
    new, ctx = _lengths(case)
    P, group, row = case["page"], case["heads"] // case["heads_kv"], 0
    if case["kind"] == "append":
        out = {}
        for name, x in (("K", _normed64(case, s["K"], s["wk"], s["pos"])), ("V", s["V"].double())):
            scale = x.abs().amax(-1) / 448
            code = _e4m3((x / scale[..., None]).clamp(-448, 448))
            codes, scales, row = s[name + "_pages"].double(), s[name + "_scales"].double(), 0
            for q, (m, c) in enumerate(zip(new, ctx)):
                while m:   # a page at a time
                    k = min(m, P - c % P)
                    page = int(s["table"][q, c // P])
                    codes[page, :, c % P:c % P + k] = code[row:row + k].transpose(0, 1)
                    scales[page, :, c % P:c % P + k] = scale[row:row + k].T
                    row, m, c = row + k, m - k, c + k
            out[name] = codes, scales
        return out["K"][0], out["V"][0], out["K"][1], out["V"][1], _normed64(case, s["Q"], s["wq"], s["pos"])
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
            held = lambda name: (s[name + "_pages"].view(torch.uint8)[pages, h // group].view(torch.float8_e4m3fn).double() *  # noqa: E731
                                 s[name + "_scales"][pages, h // group].double()[..., None]).flatten(0, 1)[:c + m]
            logit = (s["Q"][row:row + m, h].double() @ held("K").T) / math.sqrt(case["head_dim"])
            O[row:row + m, h] = torch.softmax(logit.masked_fill(hidden, -math.inf), -1) @ held("V")
        row += m
    return O
