"""Operators of a paged FP16 cache and of windowed prompts: what a serving program does with its requests until a prompt
becomes codes.

    page_map              block tables and slot maps of a step, made on the GPU from the requests' lengths
    page_store            new K and V rows to their slots of the pages
    page_load             a sequence's rows out of the pages, dense, as anchor selection and encoding read them
    page_attn             attention of each request's new tokens (one to thousands) over its pages, with row statistics
    prefill_attn_window   attention over a dense prompt in which a query sees a window of recent keys and a few first ones

    listed()  the fixed cases            prepare(case, seed)  inputs on the GPU
    draw(rng) one more of their ranges   run(state)           one pass: plain torch operations, or the package's calls if `own`
    work(case)  bytes and operations     exact(case, seed)    the same outputs from the definition, in 64 bits
"""
from __future__ import annotations

import math
import random

import torch

own = False
D = 128                       # head dim


def _attn(name, R, T, longest, Hq=32, Hkv=8, page=64, window=0, sinks=0, kind="chunk", stats=False):
    return dict(name=name, op="attn", R=R, T=T, longest=longest, Hq=Hq, Hkv=Hkv, page=page, window=window, sinks=sinks, kind=kind, stats=stats)


def listed():
    return [
        # a decode step of 256 requests: a token each, a new page for one in sixteen
        dict(name="map_decode_256", op="map", R=256, T=256, longest=8192, page=16),
        # prompts of uneven length admitted together: 65536 tokens, all of their pages new but the partly filled ones
        dict(name="map_prompts_64k", op="map", R=48, T=65536, longest=16384, page=64),
        # the rows of a decode step of 64 requests
        dict(name="store_64", op="store", T=64, Hkv=8, page=16),
        # the rows of a prompt's chunk, out of a fused projection
        dict(name="store_32k", op="store", T=32768, Hkv=8, page=64),
        # a finished prompt of odd length on its way to anchor selection
        dict(name="load_4099", op="load", R=1, N=4099, Hkv=8, page=16),
        # four long ones
        dict(name="load_4x32k", op="load", R=4, N=32768, Hkv=8, page=64),
        # one chat, one token: latency
        _attn("attn_decode_4k", 1, 1, 4096, page=16, kind="decode"),
        # a decode step of 64 requests with contexts from a few tokens to 32768
        _attn("attn_decode_64", 64, 64, 32768, kind="decode"),
        # chunked prefill beside decoding: one token for most requests, hundreds for a few
        _attn("attn_mixed_16", 16, 2048, 8192, page=32, kind="mixed"),
        # a chunk of a long prompt, with the statistics that the Anchor Score takes
        _attn("attn_chunk_2k_of_32k", 1, 2048, 32768, stats=True),
        # short prompts of uneven length under a small window, a KV head per query head
        dict(name="window_1531_b2_mha", op="window", B=2, N=1531, Nq=1531, Hq=32, Hkv=32, window=256, sinks=4),
        # a long prompt under the usual window
        dict(name="window_8k", op="window", B=1, N=8192, Nq=8192, Hq=32, Hkv=8, window=1024, sinks=4),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["map", "store", "load", "attn", "attn", "attn", "attn", "window", "window"])
    Hq, Hkv = rng.choice([(32, 8), (32, 8), (32, 32), (16, 8), (28, 7)])
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "map":
        R = _log_uniform(rng, 1, 512)
        return dict(op=op, R=R, T=_log_uniform(rng, R, 65536), longest=_log_uniform(rng, 64, 16384), page=page)
    if op == "store":
        return dict(op=op, T=_log_uniform(rng, 1, 32768 * 8 // Hkv), Hkv=Hkv, page=page)
    if op == "load":
        R = _log_uniform(rng, 1, 8)
        return dict(op=op, R=R, N=_log_uniform(rng, 1, 32768 * 32 // (R * Hkv)), Hkv=Hkv, page=page)
    window, sinks = (0, 0) if rng.random() < 0.5 else (_log_uniform(rng, 1, 4096), rng.choice([0, 1, 4, 37]))
    if op == "window":
        B = rng.choice([1, 1, 2, 3])
        N = _log_uniform(rng, 1, int(8192 * math.sqrt(32 / (B * Hq))))
        Nq = N if rng.random() < 0.7 else rng.randint(1, N)
        return dict(op=op, B=B, N=N, Nq=Nq, Hq=Hq, Hkv=Hkv, window=window or _log_uniform(rng, 1, 4096), sinks=sinks)
    kind = rng.choice(["decode", "decode", "mixed", "chunk"])
    R = 1 if kind == "chunk" else _log_uniform(rng, 1, 64 if kind == "decode" else 16)
    T = R if kind == "decode" else _log_uniform(rng, R, 2048)
    longest = _log_uniform(rng, 16, min(32768, 32768 * 512 // (R * Hkv)))
    if kind != "decode":
        longest = min(longest, max(16, 67_000_000 // (R * max(T, 64))))      # scores of the padded batch: as the longest chunk
    case = _attn("", R, T, longest, Hq, Hkv, page, window, sinks, kind, rng.random() < 0.3)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------ inputs

def _lengths(case):
    """Per request: tokens that its context has in all, and how many of them are new.  The first request has the longest
    context; contexts are spread over their logarithm.  The same for every seed, so that a case is always the same work."""
    rng = random.Random("%(R)d %(T)d %(longest)d" % case)
    R, T, most, kind = case["R"], case["T"], case["longest"], case.get("kind", "mixed")
    if kind == "decode":
        new = [1] * R
    elif kind == "chunk":
        new = [T]
    else:                                                        # a few requests share what is left behind one token each
        new, left = [1] * R, T - R
        busy = rng.sample(range(R), max(1, R // 4)) if case["op"] == "attn" else range(R)
        share = [rng.random() + 0.1 for _ in busy]
        for r, w in zip(busy, share):
            new[r] += int(left * w / sum(share))
        new[busy[0]] += T - sum(new)
    ctx = [most] + [_log_uniform(rng, 1, most) for _ in range(R - 1)]
    return [max(c, n) for c, n in zip(ctx, new)], new


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype).cuda()


def _pool(gen, n_pages, Hkv, page):
    shape = (n_pages, Hkv, page, D)
    return (torch.randn(shape, dtype=torch.float16, device="cuda", generator=gen), torch.randn(shape, dtype=torch.float16, device="cuda", generator=gen))


def _scattered(gen, counts, n_pages):
    """int32 [R, most] page numbers, no page twice, -1 behind a request's last one; and the pages that nobody holds."""
    order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    most, total = max(max(counts), 1), sum(counts)
    first = _ints([sum(counts[:r]) for r in range(len(counts))], torch.int64)
    at = torch.arange(most, device="cuda")
    held = at < _ints(counts, torch.int64)[:, None]
    table = torch.where(held, order[(first[:, None] + at).clamp(max=n_pages - 1)], -1)
    return table.to(torch.int32).contiguous(), order[total:].contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, s = case["op"], dict(case)
    if op == "window":
        B, N, Nq, Hq, Hkv = (case[x] for x in ("B", "N", "Nq", "Hq", "Hkv"))
        s["q"] = torch.randn((B, Hq, Nq, D), dtype=torch.float16, device="cuda", generator=gen)
        s["k"], s["v"] = (torch.randn((B, Hkv, N, D), dtype=torch.float16, device="cuda", generator=gen) for _ in "kv")
        return s
    page = case["page"]
    if op == "map":
        ctx, new = _lengths(case)
        held = [c - n for c, n in zip(ctx, new)]
        has, needs = [-(-h // page) for h in held], [-(-c // page) for c in ctx]
        n_pages = sum(needs) + 64
        table, s["free"] = _scattered(gen, has, n_pages)
        s["table"] = torch.full((case["R"], max(needs) + 8), -1, dtype=torch.int32, device="cuda")
        s["table"][:, :table.shape[1]] = table
        s["held"], s["new"], s["n_pages"] = _ints(held), _ints(new), n_pages
        return s
    Hkv = case["Hkv"]
    if op == "store":                                            # rows as a fused projection leaves them: token, then Q, K and V heads
        T = case["T"]
        qkv = torch.randn((T, 6 * Hkv, D), dtype=torch.float16, device="cuda", generator=gen)
        s["k"], s["v"] = qkv[:, 4 * Hkv:5 * Hkv], qkv[:, 5 * Hkv:]
        n_pages = -(-T // page) + 8
        s["k_pages"], s["v_pages"] = _pool(gen, n_pages, Hkv, page)
        s["slot"] = torch.randperm(n_pages * page, device="cuda", generator=gen)[:T].to(torch.int32)
        if T > 8:                                                # runs of rows within pages, as a prompt has them; a few rows without a slot
            pages = torch.randperm(n_pages, device="cuda", generator=gen)
            at = torch.arange(T, device="cuda") + 3
            s["slot"] = (pages[at // page] * page + at % page).to(torch.int32)
            s["slot"][-2:] = -1
        return s
    if op == "load":
        R, N = case["R"], case["N"]
        lens = [N] + [max(1, N - 37 * r) for r in range(1, R)]
        counts = [-(-n // page) for n in lens]
        n_pages = sum(counts) + 8
        s["table"], _ = _scattered(gen, counts, n_pages)
        s["ctx"] = _ints(lens)
        s["k_pages"], s["v_pages"] = _pool(gen, n_pages, Hkv, page)
        s["k"], s["v"] = (torch.zeros((R, Hkv, N, D), dtype=torch.float16, device="cuda") for _ in "kv")
        return s
    ctx, new = _lengths(case)
    counts = [-(-c // page) for c in ctx]
    n_pages = sum(counts) + 8
    s["table"], _ = _scattered(gen, counts, n_pages)
    s["k_pages"], s["v_pages"] = _pool(gen, n_pages, Hkv, page)
    s["ctx"], s["q_start"] = _ints(ctx), _ints([sum(new[:r]) for r in range(len(new) + 1)])
    s["most_new"], s["most_ctx"] = max(new), max(ctx)            # a server knows its lengths
    qkv = torch.randn((case["T"], case["Hq"] + 2 * Hkv, D), dtype=torch.float16, device="cuda", generator=gen)
    s["q"] = qkv[:, :case["Hq"]]
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_map(s):
    page, cap = s["page"], s["table"].shape[1]
    held, new = s["held"].long(), s["new"].long()
    has, needs = (held + page - 1) // page, (held + new + page - 1) // page
    take = needs - has
    first = torch.cumsum(take, 0) - take
    at = torch.arange(cap, device="cuda")
    fresh = (at >= has[:, None]) & (at < needs[:, None])
    entry = (first[:, None] + at - has[:, None]).clamp(0, s["free"].shape[0] - 1)
    s["table"].copy_(torch.where(fresh, s["free"][entry], s["table"]))
    q_start = torch.cat([torch.zeros_like(new[:1]), torch.cumsum(new, 0)])
    t = torch.arange(s["T"], device="cuda")
    r = torch.searchsorted(q_start[1:].contiguous(), t, right=True).clamp(max=s["R"] - 1)
    pos = held[r] + t - q_start[r]
    slot = s["table"][r, pos // page].long() * page + pos % page
    status = torch.stack([take.sum(), torch.zeros_like(take[0])])
    return {"ctx": (held + new).int(), "q_start": q_start.int(), "slot": slot.int(), "table": s["table"], "status": status.int()}


def _plain_store(s):
    page, Hkv = s["page"], s["Hkv"]
    slot = s["slot"].long()
    rows = torch.nonzero(slot >= 0)[:, 0]
    slot = slot[rows]
    for pages, x in ((s["k_pages"], s["k"]), (s["v_pages"], s["v"])):
        pages[slot // page, :, slot % page] = x[rows]
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_load(s):
    page, N = s["page"], s["N"]
    pos = torch.arange(N, device="cuda")
    ids = s["table"].long().clamp(min=0)[:, pos // page]                              # [R, N]
    there = (pos < s["ctx"][:, None])[:, None, :, None]
    for pages, x in ((s["k_pages"], s["k"]), (s["v_pages"], s["v"])):
        x.copy_(torch.where(there, pages[ids, :, pos % page].transpose(1, 2), x))     # [R, N, Hkv, D] -> [R, Hkv, N, D]
    return {"k": s["k"], "v": s["v"]}


def _plain_softmax(scores, seen, v):
    """scores [B, Hkv, G, n, C] and v [B, Hkv, C, D] in 32 bits -> outputs [B, Hkv, G, n, D], row maxima and row sums; a row
    that sees nothing is zero."""
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1)
    e = torch.exp(scores.sub_(torch.where(top.isfinite(), top, 0.0)[..., None]))
    total = e.sum(-1)
    out = (e.flatten(2, 3) @ v).view(*e.shape[:-1], D)
    return out / torch.where(total > 0, total, 1.0)[..., None], top, total


def _seen(pos, C, window, sinks):
    j = torch.arange(C, device="cuda")
    pos = pos[..., None]
    return (j <= pos) & ((j > pos - window) | (j < sinks)) if window else j <= pos


def _plain_attn(s):
    R, Hq, Hkv, page, n, C, T = s["R"], s["Hq"], s["Hkv"], s["page"], s["most_new"], s["most_ctx"], s["T"]
    G = Hq // Hkv
    pos = torch.arange(C, device="cuda")
    ids = s["table"].long().clamp(min=0)[:, pos // page]
    there = (pos < s["ctx"][:, None])[:, None, :, None]
    k, v = (torch.where(there, p[ids, :, pos % page].transpose(1, 2), 0).float() for p in (s["k_pages"], s["v_pages"]))    # [R, Hkv, C, D]
    start, new = s["q_start"][:-1].long(), (s["q_start"][1:] - s["q_start"][:-1]).long()
    i = torch.arange(n, device="cuda")
    at = (start[:, None] + i).clamp(max=T - 1)                                        # [R, n]
    q = s["q"][at].float().view(R, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(R, Hkv, G * n, D)
    scores = (q @ k.transpose(2, 3).contiguous()).mul_(D ** -0.5).view(R, Hkv, G, n, C)
    seen = _seen(s["ctx"].long()[:, None] - new[:, None] + i, C, s["window"], s["sinks"])[:, None, None]
    out, top, total = _plain_softmax(scores, seen, v)
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(s["q_start"][1:].long().contiguous(), t, right=True)
    real = r * n + t - start[r]                                                       # the tokens' rows of the padded batch
    res = {"out": out.permute(0, 3, 1, 2, 4).reshape(R * n, Hq, D)[real].half()}
    if s["stats"]:
        res["row_max"], res["row_sum"] = (x.permute(0, 3, 1, 2).reshape(R * n, Hq)[real].t().contiguous() for x in (top, total))
    return res


def _plain_window(s):
    B, N, Nq, Hq, Hkv = (s[x] for x in ("B", "N", "Nq", "Hq", "Hkv"))
    q = s["q"].float().view(B, Hkv, Hq // Hkv * Nq, D)
    scores = (q @ s["k"].float().transpose(2, 3).contiguous()).mul_(D ** -0.5).view(B, Hkv, Hq // Hkv, Nq, N)
    seen = _seen(torch.arange(N - Nq, N, device="cuda"), N, s["window"], s["sinks"])
    out, top, total = _plain_softmax(scores, seen, s["v"].float())
    return {"out": out.view(B, Hq, Nq, D).half(), "row_max": top.view(B, Hq, Nq), "row_sum": total.view(B, Hq, Nq)}


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    op = s["op"]
    if not own:
        return {"map": _plain_map, "store": _plain_store, "load": _plain_load, "attn": _plain_attn, "window": _plain_window}[op](s)
    import paper_2506_19505_amd as antkv

    if "geom" not in s and op != "map":
        s["geom"] = antkv.Geometry(s.get("B", s.get("R", 1)), s.get("Hq", s["Hkv"]), s["Hkv"], 8)
    if op == "map":
        ctx, q_start, slot, status = antkv.page_map(s["held"], s["new"], s["table"], s["page"], s["n_pages"], s["free"], s["T"])
        return {"ctx": ctx, "q_start": q_start, "slot": slot, "table": s["table"], "status": status}
    if op == "store":
        antkv.page_store(s["geom"], s["k"], s["v"], s["slot"], s["k_pages"], s["v_pages"])
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if op == "load":
        k, v = antkv.page_load(s["geom"], s["k_pages"], s["v_pages"], s["table"], s["N"], ctx_len=s["ctx"], k=s["k"], v=s["v"])
        return {"k": k, "v": v}
    if op == "window":
        out, row_max, row_sum = antkv.prefill_attn_window(s["geom"], s["q"], s["k"], s["v"], D ** -0.5, s["window"], s["sinks"])
        return {"out": out, "row_max": row_max, "row_sum": row_sum}
    if "workspace" not in s:                                     # kept for the next step, as a server keeps it
        s["workspace"] = antkv.page_attn_workspace(s["geom"], s["T"], s["q"].device)
    out, row_max, row_sum = antkv.page_attn(s["geom"], s["q"], D ** -0.5, s["q_start"], s["ctx"], s["table"], s["k_pages"], s["v_pages"],
                                            window=s["window"], n_sink=s["sinks"], want_stats=s["stats"], workspace=s["workspace"])
    return {"out": out, "row_max": row_max, "row_sum": row_sum} if s["stats"] else {"out": out}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits

def _exact_rows(q, k, v, first, window, sinks):
    """q [n, D] at positions first, first + 1, ..; k, v [C, D] in 64 bits."""
    out, top, total = [], [], []
    for a in range(0, q.shape[0], 1024):
        p = torch.arange(first + a, first + min(a + 1024, q.shape[0]), device="cuda")[:, None]
        x = q[a:a + 1024].mm(k.t().contiguous()) / math.sqrt(D)
        j = torch.arange(k.shape[0], device="cuda")[None]
        hidden = j > p
        if window:
            hidden |= (j <= p - window) & (j >= sinks)
        x[hidden] = -math.inf
        m = x.max(dim=1).values
        w = (x - m[:, None]).exp()
        z = w.sum(dim=1)
        out.append(w.mm(v) / z[:, None])
        top.append(m)
        total.append(z)
    return torch.cat(out), torch.cat(top), torch.cat(total)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op in ("map", "store", "load"):                           # numbers that are moved, none that are computed
        return None
    if op == "window":
        B, Hq, G = s["B"], s["Hq"], s["Hq"] // s["Hkv"]
        rows = [_exact_rows(s["q"][b, h].double(), s["k"][b, h // G].double(), s["v"][b, h // G].double(), s["N"] - s["Nq"], s["window"], s["sinks"])
                for b in range(B) for h in range(Hq)]
        shape = (B, Hq, s["Nq"])
        return {"out": torch.stack([x[0] for x in rows]).view(*shape, D), "row_max": torch.stack([x[1] for x in rows]).view(shape),
                "row_sum": torch.stack([x[2] for x in rows]).view(shape)}
    Hq, G, page = s["Hq"], s["Hq"] // s["Hkv"], s["page"]
    starts, ctx = s["q_start"].tolist(), s["ctx"].tolist()
    out = torch.empty((s["T"], Hq, D), dtype=torch.float64, device="cuda")
    top, total = (torch.empty((Hq, s["T"]), dtype=torch.float64, device="cuda") for _ in range(2))
    for r in range(s["R"]):
        a, b, c = starts[r], starts[r + 1], ctx[r]
        pages = s["table"][r, :-(-c // page)].tolist()
        for g in range(s["Hkv"]):
            k, v = (torch.cat([p[i, g] for i in pages])[:c].double() for p in (s["k_pages"], s["v_pages"]))
            for h in range(g * G, g * G + G):
                out[a:b, h], top[h, a:b], total[h, a:b] = _exact_rows(s["q"][a:b, h].double(), k, v, c - (b - a), s["window"], s["sinks"])
    return {"out": out, "row_max": top, "row_sum": total} if s["stats"] else {"out": out}


# ------------------------------------------------------------------------------------------------ bytes and operations

def _visible(first, n, window, sinks):
    """How many keys the queries at positions first .. first + n - 1 see in all, and how many different ones."""
    if not window:
        return n * (first + 1) + n * (n - 1) // 2, first + n
    pairs = 0
    for p in range(first, first + n):
        recent = min(window, p + 1)
        pairs += recent + min(sinks, p + 1 - recent)
    recent = min(first + n, n - 1 + window)
    return pairs, recent + min(sinks, first + n - recent)


def work(case):
    op = case["op"]
    if op == "map":
        R, T = case["R"], case["T"]
        return {"bytes": 16 * R + 4 * T + 8 * (T // case["page"]), "flops": 0}
    if op == "store":
        return {"bytes": case["T"] * (2 * 2 * case["Hkv"] * 2 * D + 4), "flops": 0}
    if op == "load":
        rows = sum(max(1, case["N"] - 37 * r) for r in range(case["R"]))
        return {"bytes": rows * 2 * 2 * case["Hkv"] * 2 * D, "flops": 0}
    Hq, Hkv = case["Hq"], case["Hkv"]
    if op == "window":
        pairs, keys = _visible(case["N"] - case["Nq"], case["Nq"], case["window"], case["sinks"])
        pairs, keys, rows = case["B"] * pairs, case["B"] * keys, case["B"] * case["Nq"]
        stats = 8
    else:
        seen = [_visible(c - n, n, case["window"], case["sinks"]) for c, n in zip(*_lengths(case))]
        pairs, keys, rows = sum(x[0] for x in seen), sum(x[1] for x in seen), case["T"]
        stats = 8 if case["stats"] else 0
    return {"bytes": rows * Hq * (2 * 2 * D + stats) + keys * Hkv * 2 * 2 * D, "flops": pairs * Hq * 4 * D}
