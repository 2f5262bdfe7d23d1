"""The operators around the reduction, as cases whose time can be measured: the normalised and rotated queries and keys that
the reduction reads, the kept rows' way into a paged cache, and the attention that reads the cache, with a prompt that many
sequences share.

A case is one call by a serving engine that keeps its cache, its tables and its output buffers.  Query and key rows are
unit-variance rows with a few outlying channels, as projections give them; caches are full of older tokens.  Sequences' lengths
are part of a case (drawn from its ``mix``), their tokens and pages come from the seed.
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---- cases ------------------------------------------------------------------------------------------------------------------

def _rope(rows, Hq, Hk, D=128, dtype="bf16", rot=None, interleaved=False, axes=1, norm=True):
    return dict(op="norm_rope", rows=rows, Hq=Hq, Hk=Hk, D=D, dtype=dtype, rot=rot or D, interleaved=interleaved, axes=axes, norm=norm)


def _append(B, Hk, lo, hi, S=0, start=0, page=16, D=128, dtype="bf16", rope=True, norm=False, mix=0):
    return dict(op="append", B=B, Hk=Hk, lo=lo, hi=hi, S=S, start=start, page=page, D=D, dtype=dtype, rope=rope, norm=norm, mix=mix)


def _attend(B, Hq, Hk, lo, hi, q=1, groups=0, prefix=0, page=16, D=128, dtype="bf16", mix=0):
    return dict(op="attend", B=B, Hq=Hq, Hk=Hk, lo=lo, hi=hi, q=q, groups=groups, prefix=prefix, page=page, D=D, dtype=dtype, mix=mix)


def listed():
    cases = {
        # one decoding step of 16 sequences: nothing but latency
        "rope_token_b16": _rope(16, 28, 4),
        # the prefill of 64 ordinary images with their text, 32 heads of queries and keys
        "rope_image_b64": _rope(64 * 676, 32, 32),
        # four videos: shared key heads, positions in time, height and width
        "rope_video_b4": _rope(4 * 4708, 28, 4, dtype="fp16", axes=3),
        # the new token's key and value of 16 sequences
        "append_token_b16": _append(16, 4, 1, 1, start=700),
        # the kept rows of 64 reduced images out of their layer's 676 rows
        "append_image_b64": _append(64, 32, 164, 164, S=676, page=64),
        # independent pivots: every sample keeps another number of rows, odd ones among them; high-resolution images
        "append_union_b32": _append(32, 8, 201, 420, S=2980, norm=True, mix=1),
        # one sequence answers, token by token, over one image
        "attend_token_b1": _attend(1, 28, 4, 676, 676),
        # 64 sequences decode, each over its own reduced prompt and what it has said so far
        "attend_token_b64": _attend(64, 32, 32, 164, 676, page=64, mix=2),
        # two sequences decode over hours of video
        "attend_long_b2": _attend(2, 28, 4, 99000, 131072, page=64, mix=3),
        # 48 questions about one long video, answered token by token
        "attend_shared_b48": _attend(48, 28, 4, 5, 200, groups=1, prefix=18432, mix=4),
        # eight high-resolution images with eight questions each: the questions' prefill behind the shared prompts
        "attend_questions_b64": _attend(64, 32, 8, 21, 77, q=77, groups=8, prefix=2980, mix=5),
        # the prefill of four high-resolution prompts that nothing has shortened
        "attend_prefill_b4": _attend(4, 32, 8, 2600, 2980, q=2980, page=64, mix=6),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    return rng.choice(((32, 32), (28, 4), (32, 8), (40, 40), (12, 2), (16, 16), (8, 1), (24, 8)))


def draw(rng):
    """1 to 65536 rows; 1 to 128 sequences of 1 to 4000 new rows or 1 to 131072 cached tokens, alone or 1 to 16 prefixes of up to
    32768 tokens shared by up to 64 sequences each; 8 to 80 heads; either type."""
    Hq, Hk = _heads(rng)
    dtype, D, page = rng.choice(("bf16", "bf16", "fp16")), rng.choice((64, 128, 128)), rng.choice((16, 32, 64, 128))
    op, mix = rng.choice(("rope", "append", "token", "shared", "prefill")), rng.randrange(1000)
    if op == "rope":
        rows = min(_log_uniform(rng, 1, 65536), int(350e6 / ((Hq + Hk) * D)))
        return _rope(rows, Hq, Hk, D, dtype, rng.choice((D, D, D // 2)), rng.random() < 0.3, rng.choice((1, 1, 3)), rng.random() < 0.7)
    if op == "append":
        B, hi = _log_uniform(rng, 1, 128), _log_uniform(rng, 1, 4000)
        hi = max(1, min(hi, int(60e6 / (B * Hk * D))))
        S = rng.randint(hi, min(4 * hi + 10, 5000)) if hi > 1 and rng.random() < 0.6 else 0
        return _append(B, Hk, rng.randint(1, hi), hi, S, rng.choice((0, rng.randint(1, 900))), page, D, dtype, rng.random() < 0.7, rng.random() < 0.5, mix)
    if op == "token":
        B = _log_uniform(rng, 1, 128)
        hi = max(1, min(_log_uniform(rng, 16, 131072), int(130e6 / (B * Hk * D))))
        return _attend(B, Hq, Hk, rng.randint(max(1, hi // 4), hi), hi, 1, 0, 0, page, D, dtype, mix)
    if op == "shared":
        groups = _log_uniform(rng, 1, 16)
        B = groups * _log_uniform(rng, 2, 64)
        q = rng.choice((1, 1, _log_uniform(rng, 2, 100)))
        prefix = max(64, min(_log_uniform(rng, 256, 32768), int(60e6 / (groups * Hk * D)), int(6e9 / (B * q * Hq * 4)), int(2e11 / (B * q * Hq * D * 4))))
        hi = max(q, min(_log_uniform(rng, 4, 600), int(60e6 / (B * Hk * D))))
        q = min(q, hi)
        return _attend(B, Hq, Hk, rng.randint(q, hi), hi, q, groups, prefix, page, D, dtype, mix)
    B = _log_uniform(rng, 1, 64)
    hi = max(16, min(_log_uniform(rng, 64, 4000), int(math.sqrt(4e9 / (B * Hq * 4))), int(60e6 / (B * Hk * D))))
    return _attend(B, Hq, Hk, rng.randint(hi // 2, hi), hi, hi, 0, 0, page, D, dtype, mix)


def _lengths(case):
    """(own cached tokens, query rows) of every sequence.  More than one query row: prompts or questions of ragged length, as many
    rows as own tokens where ``q`` is their largest length."""
    rng = random.Random(case["mix"])
    n = [rng.randint(case["lo"], case["hi"]) for _ in range(case["B"])]
    n[0] = case["hi"]
    if case["op"] == "append":
        return n, n
    return n, [min(x, case["q"]) for x in n]


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _rows(g, shape, dtype):
    x = torch.randn(shape, generator=g, device=g.device, dtype=torch.float32 if math.prod(shape) < 1e8 else dtype)
    x[..., :: shape[-1] // 4] *= 3.0  # the outlying channels of a head
    return x.to(dtype)


def _inv_freq(rot, dev):
    return (1.0 / 10000.0 ** (torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().to(dev)


def _sections(half):
    return (half // 4, (half - half // 4) // 2, half - half // 4 - (half - half // 4) // 2)


def _table(g, lengths, page, n_pages_before=0):
    """Pages in no order: [sequences, most pages], int32; entries behind a sequence's last page are 0."""
    dev = g.device
    need = torch.tensor([(n + page - 1) // page for n in lengths], device=dev)
    width, total = max(1, int(need.max())), int(need.sum())
    table = torch.zeros((len(lengths), width), dtype=torch.int32, device=dev)
    used = torch.arange(width, device=dev)[None, :] < need[:, None]
    table[used] = (torch.randperm(max(1, total), generator=g, device=dev)[:total] + n_pages_before).to(torch.int32)
    return table, total


def _cu(counts, dev):
    return torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device=dev)


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(seed)
    dtype, D, op = _TYPES[case["dtype"]], case["D"], case["op"]
    s = {"case": case}
    if op == "norm_rope":
        n, Hq, Hk, half = case["rows"], case["Hq"], case["Hk"], case["rot"] // 2
        # one projection's output: queries, keys and values of a row side by side, as the layer leaves them
        qkv = _rows(g, (n, Hq + 2 * Hk, D), dtype)
        s["q"], s["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
        s["pos"] = torch.randint(0, 40000, (case["axes"], n), generator=g, device=dev)
        s["inv_freq"] = _inv_freq(case["rot"], dev)
        s["sections"] = _sections(half) if case["axes"] == 3 else None
        s["wq"], s["wk"] = ((1 + 0.2 * torch.randn(D, generator=g, device=dev)).to(dtype) if case["norm"] else None for _ in range(2))
        s["out"] = (torch.empty((n, Hq, D), dtype=dtype, device=dev), torch.empty((n, Hk, D), dtype=dtype, device=dev))
        return s
    if op == "append":
        B, Hk, S, page = case["B"], case["Hk"], case["S"], case["page"]
        rows, _ = _lengths(case)
        n = sum(rows)
        src = B * S if S else n
        s["k"], s["v"] = _rows(g, (src, Hk, D), dtype), _rows(g, (src, Hk, D), dtype)
        s["cu"] = None if case["lo"] == case["hi"] else _cu(rows, dev)
        s["cu_all"] = _cu(rows, dev)
        s["seq"] = torch.repeat_interleave(torch.arange(B, device=dev), torch.tensor(rows, device=dev))
        s["idx"] = s["pos"] = None
        s["start"] = torch.randint(1, case["start"] + 1, (B,), generator=g, device=dev, dtype=torch.int32) if case["start"] else None
        if S:  # the rows a reduction kept, ascending, and their positions in the whole prompt
            kept = [torch.randperm(S, generator=g, device=dev)[:r].sort().values for r in rows]
            s["idx"] = torch.cat(kept).to(torch.int32)
            s["pos"] = torch.cat(kept)
        s["table"], pages = _table(g, [r + case["start"] for r in rows], page)
        s["inv_freq"] = _inv_freq(D, dev) if case["rope"] else None
        s["wk"] = (1 + 0.2 * torch.randn(D, generator=g, device=dev)).to(dtype) if case["norm"] else None
        s["k_cache"], s["v_cache"] = (_rows(g, (pages, Hk, page, D), dtype) for _ in range(2))
        return s
    B, Hq, Hk, page, G = case["B"], case["Hq"], case["Hk"], case["page"], case["groups"]
    kv, rows = _lengths(case)
    s["q"] = _rows(g, (sum(rows), Hq, D), dtype)
    s["cu_q"] = None if case["q"] == 1 else _cu(rows, dev)
    s["cu_all"] = _cu(rows, dev)
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device=dev)
    s["table"], pages = _table(g, kv, page)
    s["prefix"] = None
    if G:
        prefix_table, more = _table(g, [case["prefix"]] * G, page, pages)
        pages += more
        s["prefix"] = (prefix_table, torch.full((G,), case["prefix"], dtype=torch.int32, device=dev), _cu([B // G] * G, dev))
    s["k_cache"], s["v_cache"] = (_rows(g, (pages, Hk, page, D), dtype) for _ in range(2))
    s["out"] = torch.empty_like(s["q"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------

def _norm_rope(x, w, eps, pos, inv_freq, sections, interleaved):
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + eps) * w.float()
    if inv_freq is not None:
        half = inv_freq.numel()
        axis = torch.zeros(half, dtype=torch.long, device=x.device)
        if sections is not None:
            i = torch.arange(half, device=x.device)
            axis = (i >= sections[0]).long() + (i >= sections[0] + sections[1]).long()
        angle = pos[axis].t().double() * inv_freq.double()
        c, s = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
        if interleaved:
            a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
            turned = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
        else:
            a, b = y[..., :half], y[..., half:2 * half]
            turned = torch.cat((a * c - b * s, b * c + a * s), -1)
        y = torch.cat((turned, y[..., 2 * half:]), -1)
    return y.to(x.dtype)


def _slots(s):
    """(source row, page, place in the page, slot) of every appended row."""
    case = s["case"]
    n = s["seq"].numel()
    t = torch.arange(n, device=s["seq"].device) - s["cu_all"].long()[s["seq"]]
    slot = t if s["start"] is None else t + s["start"].long()[s["seq"]]
    page = s["table"].long()[s["seq"], slot // case["page"]]
    source = torch.arange(n, device=t.device) if s["idx"] is None else s["seq"] * case["S"] + s["idx"].long()
    return source, page, slot % case["page"], slot


def _plain_append(s):
    source, page, place, slot = _slots(s)
    pos = (slot if s["pos"] is None else s["pos"])[None]
    s["k_cache"][page, :, place] = _norm_rope(s["k"][source], s["wk"], 1e-6, pos, s["inv_freq"], None, False)
    s["v_cache"][page, :, place] = s["v"][source]
    return s["k_cache"], s["v_cache"]


def _pages(cache, table):
    n, w = table.shape
    x = cache[table.long()]  # [n, w, heads, page, D]
    return x.permute(0, 2, 1, 3, 4).reshape(n, cache.shape[1], w * cache.shape[2], cache.shape[3]).float()


def _plain_attend(s):
    case = s["case"]
    B, Hq, Hk, D, q, dev = case["B"], case["Hq"], case["Hk"], case["D"], case["q"], s["q"].device
    cu = s["cu_all"].long()
    lq = cu[1:] - cu[:-1]
    t = torch.arange(q, device=dev)
    row = (cu[:-1, None] + t).clamp(max=s["q"].shape[0] - 1)
    R = Hq // Hk
    x = s["q"][row].float().view(B, q, Hk, R, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, q * R, D) * (D ** -0.5)
    k, v = _pages(s["k_cache"], s["table"]), _pages(s["v_cache"], s["table"])
    sees = (s["kv_len"].long() - lq)[:, None] + t + 1  # how many own tokens a row sees
    seen = torch.arange(k.shape[2], device=dev) < sees[:, :, None]
    seen = seen[:, None, :, None, :].expand(B, 1, q, R, k.shape[2]).reshape(B, 1, q * R, k.shape[2])
    a = (x @ k.transpose(2, 3)).masked_fill_(~seen, -math.inf)
    top = a.amax(-1, keepdim=True)
    if s["prefix"] is not None:
        table, length, _ = s["prefix"]
        G, Lp = table.shape[0], case["prefix"]
        kp, vp = _pages(s["k_cache"], table)[:, :, :Lp], _pages(s["v_cache"], table)[:, :, :Lp]
        xp = x.view(G, B // G, Hk, q * R, D).transpose(1, 2).reshape(G, Hk, (B // G) * q * R, D)
        ap = xp @ kp.transpose(2, 3)
        back = lambda y: y.view(G, Hk, B // G, q * R, -1).transpose(1, 2).reshape(B, Hk, q * R, -1)  # noqa: E731
        top = torch.maximum(top, back(ap.amax(-1, keepdim=True)))
        there = top.view(G, B // G, Hk, q * R, 1).transpose(1, 2).reshape(G, Hk, -1, 1)
        ap = ap.sub_(there).exp_()
    top = top.masked_fill(top == -math.inf, 0.0)  # rows behind a short sequence
    a = a.sub_(top).exp_()
    o, total = a @ v, a.sum(-1, keepdim=True)
    if s["prefix"] is not None:
        o, total = o + back(ap @ vp), total + back(ap.sum(-1, keepdim=True))
    o = (o / total).view(B, Hk, q, R, D).permute(0, 2, 1, 3, 4).reshape(B, q, Hq, D)
    return o[t < lq[:, None]].to(s["q"].dtype)


def _handles(s):
    """The engine's cache and rotation, made once."""
    from paper_2502_11494_b200 import dart

    s["rope"] = dart.Rope(s["inv_freq"], interleaved=s["case"].get("interleaved", False), sections=s.get("sections")) if s.get("inv_freq") is not None else None
    s["cache"] = dart.PagedCache(s["k_cache"], s["v_cache"]) if "k_cache" in s else None
    s["norm_rope"] = dart.norm_rope


def _own(s):
    if "norm_rope" not in s:
        _handles(s)
    case = s["case"]
    if case["op"] == "norm_rope":
        return s["norm_rope"](s["q"], s["k"], pos=s["pos"], rope=s["rope"], q_weight=s["wq"], k_weight=s["wk"], eps=1e-6, out=s["out"])
    if case["op"] == "append":
        s["cache"].append(s["k"], s["v"], s["table"], start=s["start"], cu_rows=s["cu"], idx=s["idx"], S=case["S"], pos=s["pos"],
                          rope=s["rope"], k_weight=s["wk"], eps=1e-6)
        return s["k_cache"], s["v_cache"]
    return s["cache"].attend(s["q"], s["table"], s["kv_len"], cu_q=s["cu_q"], prefix=s["prefix"], out=s["out"])


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "norm_rope":
        s = state
        more = (s["pos"], s["inv_freq"], s["sections"], s["case"]["interleaved"])
        return _norm_rope(s["q"], s["wq"], 1e-6, *more), _norm_rope(s["k"], s["wk"], 1e-6, *more)
    return _plain_append(state) if op == "append" else _plain_attend(state)


def work(case):
    """Every row, every cached token and every page's share of it once; the visible (row, token) pairs' two products."""
    D, op = case["D"], case["op"]
    if op == "norm_rope":
        n, H = case["rows"], case["Hq"] + case["Hk"]
        return {"bytes": n * (4 * D * H + 8 * case["axes"]), "flops": 8.0 * n * H * D}
    kv, rows = _lengths(case)
    if op == "append":
        n, Hk = sum(rows), case["Hk"]
        index = (4 if case["S"] else 0) + (8 if case["rope"] and case["S"] else 0)
        return {"bytes": n * (8 * D * Hk + index), "flops": 6.0 * n * Hk * D}
    Hq, Hk, shared = case["Hq"], case["Hk"], case["prefix"] if case["groups"] else 0
    pairs = sum(r * (L - r) + r * (r + 1) // 2 + r * shared for L, r in zip(kv, rows))
    return {"bytes": 4 * D * Hk * (sum(kv) + case["groups"] * shared) + 4 * D * Hq * sum(rows), "flops": 4.0 * D * Hq * pairs}


# ---- the definition, in 64 bits, one head or one sequence at a time ------------------------------------------------------------

def _exact_rows(x, w, eps, positions, inv_freq, sections, interleaved):
    """x [rows, heads, D] -> float64; the rotation as a product of complex numbers."""
    y = x.to(torch.float64)
    if w is not None:
        y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / y.shape[-1] + eps) * w.to(torch.float64)
    if inv_freq is None:
        return y
    half = inv_freq.shape[0]
    which = [0] * half if sections is None else [a for a, n in enumerate(sections) for _ in range(n)]
    theta = torch.stack([positions[a].to(torch.float64) * f for a, f in zip(which, inv_freq.to(torch.float64))], dim=1)
    turn = torch.polar(torch.ones_like(theta), theta)
    z = y.clone()
    first, second = (range(0, 2 * half, 2), range(1, 2 * half, 2)) if interleaved else (range(half), range(half, 2 * half))
    first, second = (torch.tensor(list(r), device=x.device) for r in (first, second))
    for h in range(x.shape[1]):
        pair = torch.complex(y[:, h, first], y[:, h, second]) * turn
        z[:, h, first], z[:, h, second] = pair.real, pair.imag
    return z


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm_rope":
        more = (s["pos"], s["inv_freq"], s["sections"], case["interleaved"])
        return _exact_rows(s["q"], s["wq"], 1e-6, *more), _exact_rows(s["k"], s["wk"], 1e-6, *more)
    page = case["page"]
    if case["op"] == "append":
        K, V = s["k_cache"].to(torch.float64), s["v_cache"].to(torch.float64)
        cu = s["cu_all"].tolist()
        for b in range(case["B"]):
            r = torch.arange(cu[b], cu[b + 1], device=K.device)
            source = r if s["idx"] is None else b * case["S"] + s["idx"][r].long()
            first = 0 if s["start"] is None else int(s["start"][b])
            slot = torch.arange(first, first + len(r), device=K.device)
            where = s["table"][b].long()[torch.div(slot, page, rounding_mode="floor")]
            pos = slot if s["pos"] is None else s["pos"][r]
            K[where, :, slot % page] = _exact_rows(s["k"][source], s["wk"], 1e-6, [pos], s["inv_freq"], None, False)
            V[where, :, slot % page] = s["v"][source].to(torch.float64)
        return K, V
    kv, rows = _lengths(case)
    Hq, Hk, D, G = case["Hq"], case["Hk"], case["D"], case["groups"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)

    def tokens(cache, pages, n, h):
        return cache[pages.long(), h].reshape(-1, D)[:n].to(torch.float64)

    at = 0
    for b in range(case["B"]):
        t = torch.arange(rows[b], device=out.device)
        for h in range(Hk):
            k, v = (tokens(c, s["table"][b, :(kv[b] + page - 1) // page], kv[b], h) for c in (s["k_cache"], s["v_cache"]))
            hidden = torch.arange(kv[b], device=out.device)[None, :] > (kv[b] - rows[b] + t)[:, None]
            if G:
                table = s["prefix"][0][b // (case["B"] // G)]
                k = torch.cat((tokens(s["k_cache"], table, case["prefix"], h), k))
                v = torch.cat((tokens(s["v_cache"], table, case["prefix"], h), v))
                hidden = torch.cat((torch.zeros((rows[b], case["prefix"]), dtype=torch.bool, device=out.device), hidden), 1)
            for r in range(h * (Hq // Hk), (h + 1) * (Hq // Hk)):
                logits = s["q"][at:at + rows[b], r].to(torch.float64) @ k.T / math.sqrt(D)
                out[at:at + rows[b], r] = torch.softmax(logits.masked_fill(hidden, -math.inf), dim=1) @ v
        at += rows[b]
    return out
