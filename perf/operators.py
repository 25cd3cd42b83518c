"""What a program does with a compressed clip next, as cases that can be timed: queries and keys are normed per head and
rotated by the emitted positions, keys and values go into the pages of a cache, and the new tokens attend to what the
cache holds; later the same with one token per sequence.

Sizes: heads of 128 channels, 32 / 16 of them, are the widths C = 4096 / 2048 of the synthetic clips, 16 heads of 72
channels C = 1152; 2703 is L' of the 8B-shaped clip, 8192 the capacity of its buffers.  Lengths of a batch follow from the
case alone (spread evenly over the logarithm between two bounds), their order and all values from the seed.
"""
import math

import torch

own = False

GOLDEN = 0.6180339887498949


def _rotation(heads, kv_heads, dim, dtype="bf16", rot=None, layout="half", axes=3, norm=True, factor=1.0, far=0):
    return {"dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": dim if rot is None else rot,
            "layout": layout, "axes": axes, "norm": norm, "factor": factor, "far": far}


def _batch(seqs, new, before, page):
    return {"seqs": seqs, "new_lo": new[0], "new_hi": new[1], "before_lo": before[0], "before_hi": before[1], "page": page}


def _attend(heads, kv_heads, dim, batch, dtype="bf16", causal=True, window=0, spare=0):
    return dict(batch, kind="attend", dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, causal=causal, window=window,
                spare=spare)


def listed():
    return [
        # one generated token for each of 32 requests: what a call costs
        dict(_rotation(32, 8, 128), kind="rotate", rows=32, count=32, name="rotate_decode"),
        # the prefill of one compressed clip: buffers of worst-case capacity, the number of rows known on the device alone
        dict(_rotation(32, 8, 128), kind="rotate", rows=8192, count=2703, name="rotate_clip"),
        # fp32 tokens at the width of a vision encoder: adjacent pairs, half of the head, far scalar positions of a scaled
        # long context, no norm
        dict(_rotation(16, 16, 72, "f32", 36, "interleaved", 1, False, 1.1, 1_000_000), kind="rotate", rows=1153, count=1153,
             name="rotate_f32_part"),
        # one token for each of 64 requests joins the cache
        dict(_rotation(32, 8, 128), kind="append", spare=0, **_batch(64, (1, 1), (500, 6000), 16), name="append_decode"),
        # a compressed clip behind the text of its prompt
        dict(_rotation(32, 8, 128), kind="append", spare=5489, **_batch(1, (2703, 2703), (35, 35), 64), name="append_clip"),
        # new frames of several streams, each of another length, pages that are no power of two, scalar positions
        dict(_rotation(16, 2, 128, axes=1, far=40_000), kind="append", spare=77, **_batch(9, (60, 900), (1, 5000), 48),
             name="append_streams"),
        # decoding one request behind a clip: 2703 visual tokens, 57 of text
        dict(_attend(32, 8, 128, _batch(1, (1, 1), (2759, 2759), 16)), name="decode_one"),
        # a decoding batch, ragged
        dict(_attend(32, 8, 128, _batch(64, (1, 1), (500, 16000), 64)), name="decode_batch"),
        # the prefill of a clip and its prompt, into an empty cache
        dict(_attend(32, 8, 128, _batch(1, (2760, 2760), (0, 0), 64), spare=5432), name="prefill_clip"),
        # new frames of several streams behind what they hold
        dict(_attend(16, 2, 128, _batch(6, (60, 900), (400, 12000), 32)), name="segment_streams"),
        # a long prompt in pieces: 4096 new tokens over 16384
        dict(_attend(32, 8, 128, _batch(1, (4096, 4096), (12288, 12288), 128)), name="chunk_long"),
        # fp32 at the width of a vision encoder, short ragged chunks, a sliding window
        dict(_attend(16, 16, 72, _batch(5, (1, 50), (1, 700), 48), "f32", window=100), name="attend_f32"),
    ]


MOST_SCORES = 32 * 4096 * 16384          # the plain form's score matrix, in values
MOST_PAIRS = 1.8e9                       # visible (query head, slot) pairs: those of the largest listed case
MOST_CACHE = 64 * 16384 * 8 * 128        # values of one gathered cache


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotate", "append", "attend", "attend", "attend"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    kv_heads = log_int(1, 16)
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 8])
    dim = rng.choice([64, 128, 128, 128, 8 * rng.randint(4, 16), rng.choice([80, 96, 192, 256])])
    page = rng.choice([16, 16, 32, 64, 128, 256, rng.randint(1, 100)])
    if kind == "rotate":
        rot = dim if rng.random() < 0.6 else 4 * rng.randint(2, dim // 4)
        rows = log_int(1, 12000)
        return dict(_rotation(kv_heads * group, kv_heads, dim, dtype, rot, rng.choice(["half", "interleaved"]),
                              rng.choice([1, 3]), rng.random() < 0.7, rng.choice([1.0, 1.0, 1.2]), log_int(100, 4_000_000)),
                    kind=kind, rows=rows, count=rows if rng.random() < 0.5 else rng.randint(0, rows))
    if rng.random() < 0.4:
        batch = _batch(log_int(1, 100), (1, 1), (log_int(1, 400), log_int(400, 16000)), page)
    else:
        hi = log_int(2, 4096)
        batch = _batch(log_int(1, 8), (max(1, hi // rng.choice([1, 3, 20])), hi), (0, log_int(1, 12000)), page)
    spare = rng.choice([0, 0, log_int(1, 3000)])
    if kind == "append":
        while batch["seqs"] * (batch["new_hi"] + batch["before_hi"]) * kv_heads * dim > MOST_CACHE:
            batch["before_hi"] = max(batch["before_lo"], batch["before_hi"] // 2)
            batch["seqs"] = max(1, batch["seqs"] * 3 // 4)
        rot = dim if rng.random() < 0.7 else 4 * rng.randint(2, dim // 4)
        return dict(_rotation(kv_heads * group, kv_heads, dim, dtype, rot, rng.choice(["half", "interleaved"]),
                              rng.choice([1, 3]), rng.random() < 0.7, 1.0, log_int(100, 4_000_000)),
                    kind=kind, spare=spare, **batch)
    c = _attend(kv_heads * group, kv_heads, dim, batch, dtype, rng.random() < 0.85,
                log_int(16, 4000) if rng.random() < 0.25 else 0, spare)

    def too_large():
        s = c["new_hi"] + c["before_hi"]
        pairs = c["seqs"] * c["heads"] * c["new_hi"] * s
        return (pairs > MOST_SCORES or c["seqs"] * s * c["kv_heads"] * c["dim"] > MOST_CACHE or
                pairs * c["dim"] > (MOST_PAIRS * 128 if dtype == "bf16" else MOST_PAIRS * 4))

    while too_large():
        if c["new_hi"] > 64 and c["new_hi"] * 2 > c["before_hi"]:
            c["new_hi"] = c["new_hi"] * 2 // 3
            c["new_lo"] = min(c["new_lo"], c["new_hi"])
        elif c["seqs"] > 1:
            c["seqs"] = c["seqs"] * 2 // 3
        else:
            c["before_hi"] = c["before_hi"] * 2 // 3
            c["before_lo"] = min(c["before_lo"], c["before_hi"])
    return c


def _spread(n, lo, hi, shift):
    """n lengths between lo and hi, evenly over the logarithm"""
    return [int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** (((s + shift) * GOLDEN) % 1.0))) - 1 for s in range(n)]


def _lengths(case):
    """new tokens of every sequence, and the tokens its cache held before them"""
    n = case["seqs"]
    if n == 1:
        return [case["new_hi"]], [case["before_hi"]]
    return _spread(n, case["new_lo"], case["new_hi"], 0.5), _spread(n, case["before_lo"], case["before_hi"], 0.8)


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _rotation_state(case, rows, g, dev):
    """What a layer holds for its rotation: the table of frequencies and the two norms' weights; and the rows' positions."""
    dim, rot, dt = case["dim"], case["rot"], _dtype(case)
    pairs = rot // 2
    j = torch.arange(pairs, device=dev, dtype=torch.float64)
    freq = 1e6 ** (-j / pairs)
    if case["factor"] != 1.0:                                   # a long context: the slow pairs turn four times as slowly
        freq = torch.where(freq < 1e-3, freq / 4, freq)
    s = {"freq": freq.float(), "q_weight": None, "k_weight": None}
    if case["norm"]:
        s["q_weight"] = (1 + 0.2 * torch.randn(dim, generator=g, device=dev)).to(dt)
        s["k_weight"] = (1 + 0.2 * torch.randn(dim, generator=g, device=dev)).to(dt)
    if case["axes"] == 3:                                       # (frame, row, column) of a grid behind a text
        cell = torch.randint(0, 32 * 256, (rows,), generator=g, device=dev).sort().values
        s["pos"] = (torch.stack((cell // 256, cell // 16 % 16, cell % 16), 1) + 35 + case["far"]).int()
        h = pairs * 5 // 16
        s["sections"] = (pairs - 2 * h, h, h)
    else:
        s["pos"] = (case["far"] + torch.arange(rows, device=dev)).int().view(rows, 1)
        s["sections"] = None
    return s


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    host = torch.Generator()
    host.manual_seed(seed)
    dt, D, Hq, Hk = _dtype(case), case["dim"], case["heads"], case["kv_heads"]

    def rand(*shape, scale=1.0):
        return (scale * torch.randn(shape, generator=g, device=dev)).to(dt)

    s = {"case": case}
    if case["kind"] == "rotate":
        rows = case["rows"]
        s.update(_rotation_state(case, rows, g, dev))
        qkv = rand(rows, (Hq + 2 * Hk) * D)                     # one projection's output: q, k and v of a token side by side
        s["q"], s["k"] = qkv[:, :Hq * D].view(rows, Hq, D), qkv[:, Hq * D:(Hq + Hk) * D].view(rows, Hk, D)
        s["count"] = torch.tensor([case["count"]], dtype=torch.int32, device=dev)
        s["out_q"], s["out_k"] = torch.zeros((rows, Hq, D), dtype=dt, device=dev), torch.zeros((rows, Hk, D), dtype=dt, device=dev)
        return s
    new, before = _lengths(case)
    order = torch.randperm(case["seqs"], generator=host).tolist()
    new, before = [new[o] for o in order], [before[o] for o in order]
    ctx, page = [a + b for a, b in zip(new, before)], case["page"]
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    rows = start[-1] + case["spare"]
    used = [-(-c // page) for c in ctx]
    pages = sum(used) + 3
    ids = torch.randperm(pages, generator=host)[:sum(used)]
    table = torch.full((case["seqs"], max(1, max(used))), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = ids[at:at + n]
        at += n
    s["table"], s["rows"], s["new_most"], s["ctx_most"] = table.to(dev), rows, max(new), max(ctx)
    s["start"] = torch.tensor(start, dtype=torch.int32, device=dev)
    s["ctx"] = torch.tensor(ctx, dtype=torch.int32, device=dev)
    if case["kind"] == "append":
        s.update(_rotation_state(case, rows, g, dev))
        qkv = rand(rows, (Hq + 2 * Hk) * D).view(rows, Hq + 2 * Hk, D)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
        s["k_cache"] = torch.zeros((pages, page, Hk, D), dtype=dt, device=dev)
        s["v_cache"] = torch.zeros((pages, page, Hk, D), dtype=dt, device=dev)
        s["out_q"] = torch.zeros((rows, Hq, D), dtype=dt, device=dev)
        return s
    s["q"], s["out"] = rand(rows, Hq, D, scale=1.5), torch.zeros((rows, Hq, D), dtype=dt, device=dev)
    s["k_cache"], s["v_cache"] = rand(pages, page, Hk, D, scale=1.5), rand(pages, page, Hk, D)
    s["scale"] = D ** -0.5
    return s


def run(s):
    case = s["case"]
    if own:
        import paper_2605_07355_b200 as P
        if case["kind"] == "attend":
            return P.ttf_attend(s["q"], s["k_cache"], s["v_cache"], s["start"], s["ctx"], s["table"], s["scale"],
                                causal=case["causal"], window=case["window"], out=s["out"])
        turn = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], rot_dim=case["rot"], factor=case["factor"],
                    interleaved=case["layout"] == "interleaved", sections=s["sections"], cyclic=True)
        if case["kind"] == "rotate":
            return P.ttf_rotate(s["q"], s["k"], s["pos"], s["freq"], count=s["count"], out_q=s["out_q"], out_k=s["out_k"], **turn)
        q = P.ttf_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["start"], s["ctx"], s["table"], s["pos"], s["freq"],
                               q=s["q"], out_q=s["out_q"], **turn)
        return q, s["k_cache"], s["v_cache"]
    if case["kind"] == "attend":
        return _plain_attend(s)
    if case["kind"] == "rotate":
        valid = (torch.arange(case["rows"], device=s["q"].device) < s["count"]).view(-1, 1, 1)
        cos, sin = _plain_turns(s)
        q = _plain_rotated(s, s["q"], s["q_weight"], cos, sin)
        k = _plain_rotated(s, s["k"], s["k_weight"], cos, sin)
        return torch.where(valid, q, s["out_q"]), torch.where(valid, k, s["out_k"])
    return _plain_append(s)


def _plain_turns(s):
    """cosine and sine of every (row, pair); the angle in 64 bits (32 lose the turns of far positions)"""
    case = s["case"]
    j = torch.arange(case["rot"] // 2, device=s["pos"].device)
    if s["sections"] is None:
        pos = s["pos"].double()
    else:
        _, h, w = s["sections"]
        axis = torch.where((j % 3 == 1) & (j // 3 < h), 1, torch.where((j % 3 == 2) & (j // 3 < w), 2, 0))
        pos = s["pos"].double()[:, axis]
    angle = pos * s["freq"].double()
    return angle.cos().float()[:, None] * case["factor"], angle.sin().float()[:, None] * case["factor"]


def _plain_rotated(s, x, weight, cos, sin):
    rot, x = s["case"]["rot"], x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.float()
    if s["case"]["layout"] == "half":
        u, v = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((u * cos - v * sin, v * cos + u * sin, x[..., rot:]), -1)
    else:
        u, v = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.cat((torch.stack((u * cos - v * sin, v * cos + u * sin), -1).flatten(-2), x[..., rot:]), -1)
    return y.to(_dtype(s["case"]))


def _plain_append(s):
    rows, page = s["rows"], s["case"]["page"]
    cos, sin = _plain_turns(s)
    i = torch.arange(rows, device=s["q"].device)
    valid = i < s["start"][-1]
    seq = torch.searchsorted(s["start"][1:].long(), i, right=True).clamp(max=s["case"]["seqs"] - 1)
    slot = (s["ctx"][seq] - s["start"][seq + 1] + i)[valid]
    at = s["table"][seq[valid], slot // page].long(), slot % page
    s["k_cache"][at] = _plain_rotated(s, s["k"], s["k_weight"], cos, sin)[valid]
    s["v_cache"][at] = s["v"][valid]
    q = _plain_rotated(s, s["q"], s["q_weight"], cos, sin)
    return torch.where(valid.view(-1, 1, 1), q, s["out_q"]), s["k_cache"], s["v_cache"]


def _plain_attend(s):
    case = s["case"]
    B, n, S, D, Hk = case["seqs"], s["new_most"], s["ctx_most"], case["dim"], case["kv_heads"]
    G, dev = case["heads"] // Hk, s["q"].device
    i, j = torch.arange(n, device=dev), torch.arange(S, device=dev)
    new = s["start"][1:] - s["start"][:-1]
    row = (s["start"][:-1, None] + i).long()                    # [B, n]
    valid = i < new[:, None]
    q = s["q"][row.clamp(max=s["rows"] - 1)].float().view(B, n, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * n, D)
    pages = s["table"].clamp(min=0).long()
    k = s["k_cache"][pages].flatten(1, 2)[:, :S].float().permute(0, 2, 3, 1)            # [B, Hk, D, S]
    v = s["v_cache"][pages].flatten(1, 2)[:, :S].float().permute(0, 2, 1, 3)            # [B, Hk, S, D]
    here = s["ctx"][:, None] - new[:, None] + i                 # the new tokens' own slots
    seen = (j < s["ctx"][:, None, None]).expand(B, n, S)
    if case["causal"]:
        seen = seen & (j <= here[..., None])
    if case["window"]:
        seen = seen & (j > here[..., None] - case["window"])
    v = torch.where((j < s["ctx"][:, None])[:, None, :, None], v, 0.0)
    p = torch.matmul(q * s["scale"], k).view(B, Hk, G, n, S).masked_fill_(~seen[:, None, None], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hk, G * n, S), v).view(B, Hk, G, n, D) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, n, Hk * G, D).to(s["out"].dtype)
    s["out"][row[valid]] = o[valid]
    return s["out"]


def work(case):
    item = 4 if case["dtype"] == "f32" else 2
    D, Hq, Hk = case["dim"], case["heads"], case["kv_heads"]
    if case["kind"] == "rotate":
        n = case["count"]
        return {"bytes": 2 * n * (Hq + Hk) * D * item + n * case["axes"] * 4 + case["rot"] * 2 + (2 * D * item if case["norm"] else 0),
                "flops": n * (Hq + Hk) * (3 * case["rot"] + (4 * D if case["norm"] else 0))}
    new, before = _lengths(case)
    n = sum(new)
    table = sum(-(-(a + b) // case["page"]) for a, b in zip(new, before)) * 4 + case["seqs"] * 8
    if case["kind"] == "append":
        return {"bytes": 2 * n * (Hq + 2 * Hk) * D * item + n * case["axes"] * 4 + n * 4 + case["rot"] * 2 + (2 * D * item if case["norm"] else 0),
                "flops": n * (Hq + Hk) * (3 * case["rot"] + (4 * D if case["norm"] else 0))}
    w, pairs, slots = case["window"], 0, 0
    for a, b in zip(new, before):
        c = a + b
        first = max(0, b - w + 1) if w else 0                   # the first slot that the first new token sees
        slots += c - first if a else 0
        for i in range(a):                                      # (integers alone: a few thousand at most)
            top = b + i + 1 if case["causal"] else c
            pairs += top - (max(0, b + i - w + 1) if w else 0)
    return {"bytes": 2 * n * Hq * D * item + 2 * slots * Hk * D * item + table, "flops": 4.0 * D * Hq * pairs}


def exact(case, seed):
    """The definitions in 64 bits, token by token or head by head."""
    s = prepare(case, seed)
    D, Hq, Hk = case["dim"], case["heads"], case["kv_heads"]
    group = Hq // Hk
    start, ctx, table = (s[k].tolist() if k in s else None for k in ("start", "ctx", "table"))
    if case["kind"] == "attend":
        out = s["out"].double()
        for b in range(case["seqs"]):
            n, c = start[b + 1] - start[b], ctx[b]
            if n == 0 or c == 0:
                continue
            page_ids = torch.tensor(table[b][:-(-c // case["page"])], device=out.device)
            kb, vb = (s[x][page_ids].reshape(-1, Hk, D)[:c].double() for x in ("k_cache", "v_cache"))
            here = torch.arange(c - n, c, device=out.device).view(n, 1)
            slot = torch.arange(c, device=out.device).view(1, c)
            hidden = torch.zeros((n, c), dtype=torch.bool, device=out.device)
            if case["causal"]:
                hidden |= slot > here
            if case["window"]:
                hidden |= slot <= here - case["window"]
            for h in range(Hq):
                score = s["q"][start[b]:start[b + 1], h].double() @ kb[:, h // group].T * s["scale"]
                score[hidden] = -math.inf
                out[start[b]:start[b + 1], h] = torch.softmax(score, -1) @ vb[:, h // group]
        return out

    pairs = case["rot"] // 2
    axis = [0] * pairs
    if s["sections"] is not None:
        for a in (1, 2):
            for m in range(s["sections"][a]):
                axis[3 * m + a] = a
    first = [j if case["layout"] == "half" else 2 * j for j in range(pairs)]
    second = [j + pairs if case["layout"] == "half" else 2 * j + 1 for j in range(pairs)]

    def turned(x, weight):
        y = x.double()
        if weight is not None:
            y = y / (y.pow(2).sum(-1, keepdim=True) / D + 1e-6).sqrt() * weight.double()
        z = y.clone()
        turn = torch.polar(torch.full((1,), case["factor"], dtype=torch.float64, device=y.device),
                           s["pos"][:, axis].double() * s["freq"].double())[:, None]
        w = torch.complex(y[..., first], y[..., second]) * turn
        z[..., first], z[..., second] = w.real, w.imag
        return z

    q, k = turned(s["q"], s["q_weight"]), turned(s["k"], s["k_weight"])
    if case["kind"] == "rotate":
        n = case["count"]
        out_q, out_k = s["out_q"].double(), s["out_k"].double()
        out_q[:n], out_k[:n] = q[:n], k[:n]
        return out_q, out_k
    out_q, k_cache, v_cache = s["out_q"].double(), s["k_cache"].double(), s["v_cache"].double()
    out_q[:start[-1]] = q[:start[-1]]
    page = case["page"]
    for b in range(case["seqs"]):
        n = start[b + 1] - start[b]
        slot = torch.arange(ctx[b] - n, ctx[b])
        ids = torch.tensor(table[b])[slot // page].to(out_q.device)
        slot = (slot % page).to(out_q.device)
        k_cache[ids, slot] = k[start[b]:start[b + 1]]
        v_cache[ids, slot] = s["v"][start[b]:start[b + 1]].double()
    return out_q, k_cache, v_cache
